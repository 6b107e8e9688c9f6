"""The feed-forward half of a decoder block: pruned, recovered and served.

    s = x + r,   a = norm(s),   h = act(a Wg^T) * (a Wu^T),   y = h Wd^T

with the root-mean-square norm and its weight. prune_feedforward runs the steps of
Algorithm 1 (pipeline.py) on its three matrices: gate and up share their inputs a, and so
their Hessian; down's inputs h are those of the pruned gate and up. recover then lowers
the output error with gradient steps on the norm's weight and on the kept entries of gate
and up; down stays as its solve left it, for the inputs that it had then. PackedFeedForward
holds the three matrices in 4 bits and runs a few tokens at a time.

Run as a program it does all three on a synthetic block and prints what each costs.
This module sequences library calls and allocates with torch; norms, products, their
gradients, the solves and the packing run in the HIP kernels.
"""
from __future__ import annotations

import argparse
from dataclasses import dataclass, replace
from typing import Callable

import torch
from torch.nn.functional import pad

from . import _lib as L
from .pipeline import solve_layer, spectral_step_size


@dataclass
class FeedForward:
    norm: torch.Tensor    # float32 [d]
    gate: torch.Tensor    # float32 [d_ff, d]
    up: torch.Tensor      # float32 [d_ff, d]
    down: torch.Tensor    # float32 [d, d_ff]
    eps: float = 1e-6
    act: int = L.ACT_SILU


@dataclass
class Activations:
    S: torch.Tensor       # bfloat16 [n_tok, d], x + r
    A: torch.Tensor       # bfloat16 [n_tok, d], its norm
    G: torch.Tensor       # bfloat16 [n_tok, d_ff]
    U: torch.Tensor       # bfloat16 [n_tok, d_ff]
    H: torch.Tensor       # bfloat16 [n_tok, d_ff]


def hidden(block: FeedForward, X: torch.Tensor, R: torch.Tensor | None = None) -> Activations:
    """The block up to down's inputs, with all that the gradient needs."""
    n, d = X.shape
    ff = block.gate.shape[0]

    def rows(width):
        return torch.empty((n, width), dtype=torch.bfloat16, device=X.device)

    t = Activations(rows(d), rows(d), rows(ff), rows(ff), rows(ff))
    L.optima_rms_norm(X, block.norm, t.A, block.eps, R=R, S=t.S)
    L.optima_gated_forward(t.A, block.gate.bfloat16(), block.up.bfloat16(), t.H, act=block.act,
                           G=t.G, U=t.U)
    return t


def _product(X: torch.Tensor, W: torch.Tensor, dtype: torch.dtype,
             ref: torch.Tensor | None = None, err: torch.Tensor | None = None) -> torch.Tensor:
    """X W^T. The forward product takes inputs in multiples of 64 and outputs in multiples of 4:
    other widths are filled up with zeros."""
    d_out, d_in = W.shape
    more_in, more_out = -d_in % 64, -d_out % 4
    if more_in:
        X = pad(X, (0, more_in))
    if more_in or more_out:
        W = pad(W, (0, more_in, 0, more_out))
    if more_out and ref is not None:
        ref = pad(ref, (0, more_out))
    Y = torch.empty((X.shape[0], d_out + more_out), dtype=dtype, device=X.device)
    L.optima_linear_forward(X, W, Y=Y, Y_ref=ref, err_out=err)
    return Y[:, :d_out].contiguous() if more_out else Y


def _down(H: torch.Tensor, down: torch.Tensor, ref: torch.Tensor | None = None):
    """H down^T in float32, and with ref the sum of squared differences."""
    err = None if ref is None else torch.zeros(1, dtype=torch.float64, device=H.device)
    return _product(H, down, torch.float32, ref, err), err


def output(block: FeedForward, X: torch.Tensor, R: torch.Tensor | None = None) -> torch.Tensor:
    """y, float32 [n_tok, d]."""
    return _down(hidden(block, X, R).H, block.down)[0]


def output_error(block: FeedForward, Y_dense: torch.Tensor, X: torch.Tensor,
                 R: torch.Tensor | None = None) -> float:
    """The sum of squared differences of the block's outputs from Y_dense (float32)."""
    return float(_down(hidden(block, X, R).H, block.down, Y_dense)[1].item())


@dataclass
class FeedForwardReport:
    skipped: dict         # matrix -> whether the skip rule kept the mask-only weights
    iterations: dict      # matrix -> iterations of its solve
    err_kept: float       # squared output error against the dense block
    err_wanda: float      # the same with the mask-only weights in all three


def prune_feedforward(block: FeedForward, X: torch.Tensor, R: torch.Tensor | None,
                      start: Callable[[int], torch.Tensor], sparsity: float = 0.5,
                      rel_damp: float = 0.01, opts: L.SolverOpts | None = None):
    """Algorithm 1 over gate, up and down on the calibration tokens X (+ R), bfloat16
    [n_tok, d]. start: width -> float32 [block, width] start vectors of the step-size
    iteration. Returns (pruned block, masks by matrix, report)."""
    dev = X.device
    Y_dense = output(block, X, R)
    pruned, wanda = replace(block), replace(block)
    masks, report = {}, FeedForwardReport({}, {}, 0.0, 0.0)

    def update(inputs, names):
        width = inputs.shape[1]
        H = torch.empty((width, width), dtype=torch.float32, device=dev)
        L.optima_hessian_accumulate(inputs, H)
        for name in names:
            W0 = getattr(block, name)
            masks[name] = torch.empty(W0.shape, dtype=torch.uint8, device=dev)
            L.optima_wanda_mask(W0, H, masks[name], L.MASK_UNSTRUCTURED, sparsity,
                                col_sq_stride=width + 1)
        lam = torch.empty(1, dtype=torch.float32, device=dev)
        L.optima_hessian_damp(H, rel_damp, lam)
        lmax = torch.empty(1, dtype=torch.float32, device=dev)
        spectral_step_size(H, start(width), lmax)
        for name in names:
            solved = solve_layer(H, lmax, getattr(block, name), masks[name], opts)
            setattr(pruned, name, solved.kept)
            setattr(wanda, name, solved.wanda)
            report.skipped[name] = solved.skipped
            report.iterations[name] = int(solved.info["iterations"])

    update(hidden(block, X, R).A, ("gate", "up"))
    update(hidden(pruned, X, R).H, ("down",))
    report.err_kept = output_error(pruned, Y_dense, X, R)
    report.err_wanda = output_error(wanda, Y_dense, X, R)
    return pruned, masks, report


def gradients(block: FeedForward, masks: dict, Y_dense: torch.Tensor, X: torch.Tensor,
              R: torch.Tensor | None = None, down_t: torch.Tensor | None = None):
    """(loss, gradients by name) of loss = mean over tokens of |y - y_dense|^2 / 2 in the
    norm's weight and the kept entries of gate and up; float32, exactly 0 elsewhere.
    down_t: block.down transposed, for callers that have it."""
    n, d = X.shape
    dev = X.device
    t = hidden(block, X, R)
    Y, err = _down(t.H, block.down, Y_dense)
    dY = Y.sub_(Y_dense).div_(n).bfloat16()
    if down_t is None:
        down_t = block.down.t().contiguous()
    dH = _product(dY, down_t, torch.bfloat16)
    g = {"gate": torch.empty_like(block.gate), "up": torch.empty_like(block.up),
         "norm": torch.empty_like(block.norm)}
    dA = torch.empty((n, d), dtype=torch.bfloat16, device=dev)
    L.optima_gated_backward(t.A, block.gate.bfloat16(), block.up.bfloat16(), t.G, t.U, dH, dX=dA,
                            dWg=g["gate"], dWu=g["up"], act=block.act, mask_g=masks["gate"],
                            mask_u=masks["up"])
    # dX is what blocks below would go on with; here it reuses dA.
    L.optima_rms_norm_backward(t.S, block.norm, dA, dA, block.eps, dweight=g["norm"])
    return float(err.item()) / (2 * n), g


def recover(block: FeedForward, masks: dict, Y_dense: torch.Tensor, X: torch.Tensor,
            R: torch.Tensor | None = None, steps: int = 20, lr: float = 1e-4,
            betas: tuple = (0.9, 0.99)):
    """Gradient steps with running first and second moments (each divided by its own
    sum of weights) from `block`, on the output error against Y_dense. Returns (block,
    losses before each step); pruned entries stay exactly 0."""
    out = replace(block, norm=block.norm.clone(), gate=block.gate.clone(), up=block.up.clone())
    params = {name: getattr(out, name) for name in ("norm", "gate", "up")}
    first = {k: torch.zeros_like(p) for k, p in params.items()}
    second = {k: torch.zeros_like(p) for k, p in params.items()}
    down_t = block.down.t().contiguous()
    losses = []
    for step in range(1, steps + 1):
        loss, g = gradients(out, masks, Y_dense, X, R, down_t)
        losses.append(loss)
        for k, p in params.items():
            first[k].lerp_(g[k], 1 - betas[0])
            second[k].lerp_(g[k].square_(), 1 - betas[1])
            size = (second[k] / (1 - betas[1] ** step)).sqrt_().add_(1e-30)
            p.addcdiv_(first[k], size, value=-lr / (1 - betas[0] ** step))
    return out, losses


class PackedFeedForward:
    """The block with its matrices in 4 bits, for up to max_tokens tokens a call.

    The norm writes 8-bit codes with one scale for each group of a token, so that gate
    and up multiply integers; down takes bfloat16. All buffers are made here: step only
    launches, three kernels for up to 16 tokens, and can be captured in a graph."""

    def __init__(self, block: FeedForward, group: int = 128, max_tokens: int = 1):
        dev = block.gate.device
        ff, d = block.gate.shape
        self.norm, self.eps, self.act, self.group = block.norm, block.eps, block.act, group
        self.packed = {}
        for name in ("gate", "up", "down"):
            W = getattr(block, name)
            Q = torch.empty((W.shape[0], L.optima_w4_row_bytes(W.shape[1])), dtype=torch.uint8,
                            device=dev)
            scales = torch.empty((W.shape[0], -(-W.shape[1] // group)), dtype=torch.bfloat16,
                                 device=dev)
            L.optima_w4_pack(W, Q, scales, group)
            self.packed[name] = (Q, scales)
        self.codes = torch.empty((max_tokens, d), dtype=torch.int8, device=dev)
        self.code_scales = torch.empty((max_tokens, -(-d // group)), dtype=torch.float32,
                                       device=dev)
        self.hidden = torch.empty((max_tokens, ff), dtype=torch.bfloat16, device=dev)
        space = max(L.optima_w4_workspace_bytes(max_tokens, d, ff, 2),
                    L.optima_w4_workspace_bytes(max_tokens, ff, d, 1))
        self.ws = torch.empty(space, dtype=torch.uint8, device=dev)

    def step(self, X: torch.Tensor, S: torch.Tensor, Y: torch.Tensor) -> None:
        """S <- X + S, Y <- the block's output for it. X, S and Y are [n_tok, d]: X and S
        bfloat16 or float32 of one type, Y bfloat16 or float32."""
        n = X.shape[0]
        if n > self.codes.shape[0]:
            raise ValueError(f"{n} tokens, made for {self.codes.shape[0]}")
        codes, code_scales, H = self.codes[:n], self.code_scales[:n], self.hidden[:n]
        L.optima_rms_norm(X, self.norm, codes, self.eps, R=S, S=S, scales=code_scales,
                          group=self.group)
        L.optima_w4_gated(codes, *self.packed["gate"], *self.packed["up"], H, self.group,
                          act=self.act, x_scales=code_scales, x_group=self.group, ws=self.ws)
        L.optima_w4_linear(H, *self.packed["down"], Y, self.group, ws=self.ws)


def synthetic_block(d: int, ff: int, seed: int = 0, device="cuda:0") -> FeedForward:
    g = torch.Generator(device=device).manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=device)

    return FeedForward(1 + 0.1 * normal(d), normal(ff, d) * d ** -0.5, normal(ff, d) * d ** -0.5,
                       normal(d, ff) * ff ** -0.5)


def main(argv=None) -> None:
    ap = argparse.ArgumentParser(description="Prune, recover and serve a synthetic "
                                             "feed-forward block.")
    ap.add_argument("--d", type=int, default=1024)
    ap.add_argument("--ff", type=int, default=2816)
    ap.add_argument("--tokens", type=int, default=8192)
    ap.add_argument("--sparsity", type=float, default=0.5)
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--group", type=int, default=128, choices=(32, 64, 128))
    ap.add_argument("--vocab", type=int, default=8000,
                    help="tokens of a synthetic output head that scores the blocks; 0: none")
    a = ap.parse_args(argv)
    dev = torch.device("cuda:0")
    g = torch.Generator(device=dev).manual_seed(1)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=dev)

    def timed(call):
        ev = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
        ev[0].record()
        out = call()
        ev[1].record()
        torch.cuda.synchronize()
        return out, ev[0].elapsed_time(ev[1])

    block = synthetic_block(a.d, a.ff)
    # Tokens with a few strong channels, which is what calibration is for.
    spread = torch.exp(normal(a.d))
    X, R = ((normal(a.tokens, a.d) * spread).bfloat16() for _ in range(2))
    Y_dense = output(block, X, R)
    total = float(Y_dense.double().square().sum().item())
    (pruned, masks, rep), ms = timed(lambda: prune_feedforward(
        block, X, R, lambda width: normal(8, width), a.sparsity))
    print(f"prune    {ms:9.2f} ms  output error {rep.err_kept / total:.5f} of the outputs "
          f"(mask only {rep.err_wanda / total:.5f})")
    (better, _), ms = timed(lambda: recover(pruned, masks, Y_dense, X, R, a.steps))
    print(f"recover  {ms:9.2f} ms  output error "
          f"{output_error(better, Y_dense, X, R) / total:.5f} after {a.steps} steps")
    packed, ms = timed(lambda: PackedFeedForward(better, a.group))
    print(f"pack     {ms:9.2f} ms")
    x, r = X[:1].clone(), R[:1].clone()
    y = torch.empty_like(x)
    packed.step(x, r, y)
    want = output(better, X[:1], R[:1])
    print(f"serve    4 bits are {float((y.float() - want).norm() / want.norm()):.4f} off in the "
          "first token")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        packed.step(x, r, y)
    graph.replay()
    _, ms = timed(lambda: [graph.replay() for _ in range(100)])
    print(f"serve    {10 * ms:9.2f} us a token")
    if a.vocab:
        _print_scores(a.vocab, block, {"pruned": pruned, "recovered": better}, X, R)


def _print_scores(vocab: int, dense: FeedForward, others: dict, X: torch.Tensor,
                  R: torch.Tensor) -> None:
    """How probable the dense block's first choices are behind each block, under one head, with it
    in 16 and in 4 bits."""
    from .scoring import PackedHead, score, synthetic_head

    head = synthetic_head(X.shape[1], vocab)
    n = min(2048, X.shape[0])
    X, R = X[:n], R[:n]
    packed = PackedHead(head, max_tokens=n, packed_tokens=True)

    def states(block):
        return (X.float() + R.float()).bfloat16(), output(block, X, R).bfloat16()

    S, Y = states(dense)
    tokens = score(head, Y, torch.full((n,), -1, device=X.device), S, top=1).top_index[:, 0].clone()
    for name, block in {"dense": dense, **others}.items():
        S, Y = states(block)
        s = score(head, Y, tokens, S)
        p = packed.step(Y, S, tokens)
        print(f"score    {name:>9}  log p {float(s.logp.mean()):8.4f}  entropy "
              f"{float(s.entropy.mean()):7.4f}  head in 4 bits {float(p.logp.mean()):8.4f}")


if __name__ == "__main__":
    main()
