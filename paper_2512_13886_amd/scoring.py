"""The end of a model: the final norm, the output head and what they say of given tokens.

    s = x + r,   a = norm(s),   z = a W^T,   log p = z - lse(z)

score says how probable given tokens are under a head, with the entropy and the most probable
alternatives: the measure by which a pruned model is compared with the dense one (perplexity is
exp of minus the mean). prune_head runs the steps of Algorithm 1 (pipeline.py) on W; gradients and
recover go back from the tokens' loss to the norm's weight and the kept entries of W, and to the
hidden states, for what lies below. PackedHead holds W in microscaled 4-bit floating point and
scores out of buffers of its own.

This module sequences library calls and allocates with torch.
"""
from __future__ import annotations

import ctypes
from dataclasses import dataclass, replace
from typing import Callable

import torch

from . import _lib as L
from .feedforward import _product
from .pipeline import solve_layer, spectral_step_size


@dataclass
class Head:
    norm: torch.Tensor    # float32 [d]
    weight: torch.Tensor  # float32 [vocab, d]
    eps: float = 1e-6


@dataclass
class Scores:
    logits: torch.Tensor  # bfloat16 or float32 [n, vocab]
    logp: torch.Tensor    # float32 [n], 0 where the token is negative
    lse: torch.Tensor     # float32 [n]
    entropy: torch.Tensor  # float32 [n]
    top_index: torch.Tensor | None = None  # int64 [n, top]
    top_logp: torch.Tensor | None = None   # float32 [n, top]


def _scores(logits: torch.Tensor, top: int) -> Scores:
    n, dev = logits.shape[0], logits.device
    s = Scores(logits, *(torch.empty(n, dtype=torch.float32, device=dev) for _ in range(3)))
    if top:
        s.top_index = torch.empty((n, top), dtype=torch.int64, device=dev)
        s.top_logp = torch.empty((n, top), dtype=torch.float32, device=dev)
    return s


def _normed(head: Head, X: torch.Tensor, R: torch.Tensor | None):
    S, A = torch.empty_like(X), torch.empty_like(X)
    L.optima_rms_norm(X, head.norm, A, head.eps, R=R, S=S)
    return S, A


def score(head: Head, X: torch.Tensor, tokens: torch.Tensor, R: torch.Tensor | None = None,
          top: int = 0, scale: float = 1.0) -> Scores:
    """Scores of tokens (int64 [n], a negative one is none) after the hidden states X (+ R),
    bfloat16 [n, d], with logits of float32; scale is one over the temperature."""
    _, A = _normed(head, X, R)
    s = _scores(_product(A, head.weight, torch.float32), top)
    L.optima_token_logprobs(s.logits, tokens, s.logp, lse=s.lse, entropy=s.entropy,
                            top_index=s.top_index, top_logp=s.top_logp, scale=scale)
    return s


def prune_head(head: Head, X: torch.Tensor, R: torch.Tensor | None,
               start: Callable[[int], torch.Tensor], sparsity: float = 0.5,
               rel_damp: float = 0.01, opts: L.SolverOpts | None = None):
    """Algorithm 1 on the head's weight, on the hidden states X (+ R). start: width -> float32
    [block, width] start vectors of the step-size iteration. Returns (pruned head, mask, whether
    the skip rule kept the mask-only weights)."""
    d, dev = X.shape[1], X.device
    H = torch.empty((d, d), dtype=torch.float32, device=dev)
    L.optima_hessian_accumulate(_normed(head, X, R)[1], H)
    mask = torch.empty(head.weight.shape, dtype=torch.uint8, device=dev)
    L.optima_wanda_mask(head.weight, H, mask, L.MASK_UNSTRUCTURED, sparsity, col_sq_stride=d + 1)
    L.optima_hessian_damp(H, rel_damp, torch.empty(1, dtype=torch.float32, device=dev))
    lmax = torch.empty(1, dtype=torch.float32, device=dev)
    spectral_step_size(H, start(d), lmax)
    solved = solve_layer(H, lmax, head.weight, mask, opts)
    return replace(head, weight=solved.kept), mask, solved.skipped


def gradients(head: Head, X: torch.Tensor, tokens: torch.Tensor, R: torch.Tensor | None = None,
              mask: torch.Tensor | None = None):
    """(loss, gradients by name, the gradient of X and R) of loss = minus the mean log probability
    of the tokens that are given: float32 of the norm's weight and of W (exactly 0 where the mask
    is), bfloat16 of the hidden states."""
    n, d = X.shape
    S, A = _normed(head, X, R)
    # float32, as in score: in bfloat16 logits near 16 are 1/8 apart, and the loss would not be the score.
    s = _scores(_product(A, head.weight, torch.float32), 0)
    L.optima_token_logprobs(s.logits, tokens, s.logp, lse=s.lse)
    given = tokens >= 0
    count = given.sum().clamp_(min=1)
    dlogp = torch.where(given, -1.0 / count, 0.0).float()
    # The logits are not needed again: their gradient takes their place. It is rounded once, for the
    # 16-bit products.
    L.optima_token_logprobs_backward(s.logits, s.lse, s.logits, tokens=tokens, dlogp=dlogp)
    D = s.logits.bfloat16()
    dA = _product(D, head.weight.t().contiguous(), torch.bfloat16)
    g = {"weight": _product(D.t().contiguous(), A.t().float().contiguous(), torch.float32),
         "norm": torch.empty_like(head.norm)}
    if mask is not None:
        g["weight"].mul_(mask)
    dX = torch.empty_like(X)
    L.optima_rms_norm_backward(S, head.norm, dA, dX, head.eps, dweight=g["norm"])
    return float(-(s.logp.sum() / count).item()), g, dX


def recover(head: Head, mask: torch.Tensor, X: torch.Tensor, tokens: torch.Tensor,
            R: torch.Tensor | None = None, steps: int = 10, lr: float = 1e-2):
    """Gradient steps of the norm's weight and the kept entries of W from `head` on the tokens' loss,
    each of the gradient's size relative to its largest entry. Returns (head, losses before each
    step); pruned entries stay exactly 0."""
    out = replace(head, norm=head.norm.clone(), weight=head.weight.clone())
    losses = []
    for _ in range(steps):
        loss, g, _ = gradients(out, X, tokens, R, mask)
        losses.append(loss)
        for name in ("norm", "weight"):
            p = getattr(out, name)
            size = g[name].abs().amax().clamp_(min=1e-30) / p.abs().amax()
            p.sub_(lr * (g[name] / size))
    return out, losses


class PackedHead:
    """The head with W in microscaled 4-bit floating point, for up to max_tokens tokens a call, taken
    in 16 bits, or with packed_tokens in 4 bits too. Logits are kept in logits_dtype: bfloat16 halves
    what is written and read again of them, and its half step (1/16 at logits of 16 to 32) is below the
    4-bit weights' own error; the log probabilities, lse and entropy are those of the logits as they
    are kept. float32 keeps the products' sums as they are. All buffers are made here: step only
    launches and can be captured in a graph."""

    def __init__(self, head: Head, max_tokens: int = 1, top: int = 0, packed_tokens: bool = False,
                 logits_dtype: torch.dtype = torch.bfloat16):
        vocab, d = head.weight.shape
        dev = head.weight.device
        self.norm, self.eps = head.norm, head.eps

        def room(n):
            return (torch.empty((n, L.optima_mx4_row_bytes(d)), dtype=torch.uint8, device=dev),
                    torch.empty((n, L.optima_mx4_scale_bytes(d)), dtype=torch.uint8, device=dev))

        self.packed = room(vocab)
        L.optima_mx4_pack(head.weight, *self.packed)
        self.normed = torch.empty((max_tokens, d), dtype=torch.bfloat16, device=dev)
        self.codes = room(max_tokens) if packed_tokens else None
        self.out = _scores(torch.empty((max_tokens, vocab), dtype=logits_dtype, device=dev), top)
        space = max(L.optima_mx4_workspace_bytes(max_tokens, d, vocab),
                    L.optima_token_logprobs_workspace_bytes(max_tokens, vocab, top), 16)
        self.ws = torch.empty(space, dtype=torch.uint8, device=dev)

    def step(self, X: torch.Tensor, S: torch.Tensor, tokens: torch.Tensor,
             scale: float = 1.0) -> Scores:
        """S <- X + S, and the scores of `tokens` after it, in this object's buffers. X and S are
        [n, d], bfloat16 or float32 of one type. A call that is refused leaves S as it is."""
        n = X.shape[0]
        if n > self.normed.shape[0]:
            raise ValueError(f"{n} tokens, made for {self.normed.shape[0]}")
        A, o = self.normed[:n], self.out
        # What the calls after the norm would refuse. The norm refuses X and S itself, before it writes.
        L._need_one_device(None, X, S, tokens, A)
        if not (tokens.dtype == torch.int64 and tokens.is_cuda and tokens.shape == (n,) and
                tokens.is_contiguous()):
            raise ValueError(f"tokens must be contiguous int64 [{n}] on the device")
        if o.top_index is not None and \
                tokens.untyped_storage().data_ptr() == o.top_index.untyped_storage().data_ptr():
            raise ValueError("tokens lie in this object's alternatives, which the step writes")
        if not 0.0 < ctypes.c_float(scale).value < float("inf"):
            raise ValueError(f"scale must be positive and finite, got {scale}")
        out = Scores(o.logits[:n], o.logp[:n], o.lse[:n], o.entropy[:n],
                     None if o.top_index is None else o.top_index[:n],
                     None if o.top_logp is None else o.top_logp[:n])
        L.optima_rms_norm(X, self.norm, A, self.eps, R=S, S=S)
        if self.codes is None:
            L.optima_mx4_linear(A, *self.packed, out.logits, ws=self.ws)
        else:
            codes, scales = self.codes[0][:n], self.codes[1][:n]
            L.optima_mx4_pack(A, codes, scales)
            L.optima_mx4_linear(codes, *self.packed, out.logits, x_scales=scales, ws=self.ws)
        L.optima_token_logprobs(out.logits, tokens, out.logp, lse=out.lse, entropy=out.entropy,
                                top_index=out.top_index, top_logp=out.top_logp, scale=scale,
                                ws=self.ws)
        return out


def synthetic_head(d: int, vocab: int, seed: int = 0, device="cuda:0") -> Head:
    g = torch.Generator(device=device).manual_seed(seed)
    return Head(1 + 0.1 * torch.randn(d, generator=g, device=device),
                2.5 * d ** -0.5 * torch.randn((vocab, d), generator=g, device=device))
