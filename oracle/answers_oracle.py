"""64-bit forms of the operators between packed weights and a model's answers: microscaled 4-bit
values, their products, and the log probabilities of tokens with their gradient. Plain torch on
the CPU or, for large sizes, on the inputs' device."""
from __future__ import annotations

import torch

LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _power(e: torch.Tensor) -> torch.Tensor:
    """2^e in float64 for whole e, by its bits: the device's own power is a step off."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def mx4_values(x: torch.Tensor):
    """(values float64 [n, d], codes uint8 [n, d], scale bytes uint8 [n, ceil(d / 32)]) of rows x,
    block by block from the definition."""
    n, d = x.shape
    blocks = -(-d // 32)
    v = torch.zeros(n, blocks * 32, dtype=torch.float64, device=x.device)
    v[:, :d] = x.double()
    v = v.view(n, blocks, 32)
    top = v.abs().amax(2)
    bad = ~torch.isfinite(v).all(2)
    m, e = torch.frexp(torch.where(bad, 1.0, top))
    e = torch.where(m > 0, (e - 3).clamp(min=-127), -127)
    units = (v / _power(e).unsqueeze(2)).abs()
    units = torch.where(bad.unsqueeze(2), 0.0, units)
    code = torch.zeros_like(units, dtype=torch.uint8)
    for k in range(1, 8):  # a value on the border between two codes takes the even one
        border = (LEVELS[k] + LEVELS[k - 1]) / 2
        code[units >= border if k % 2 == 0 else units > border] = k
    size = torch.tensor(LEVELS, dtype=torch.float64, device=x.device)[code.long()]
    negative = torch.signbit(v) & ~bad.unsqueeze(2)
    values = torch.where(negative, -size, size) * _power(e).unsqueeze(2)
    values[bad] = float("nan")
    code = code + 8 * negative.to(torch.uint8)
    scale = torch.where(bad, 255, e + 127).to(torch.uint8)
    return values.view(n, -1)[:, :d], code.view(n, -1)[:, :d], scale


def mx4_layout(code: torch.Tensor, scale: torch.Tensor):
    """(Q, scales) as optima_mx4_pack lays codes and scale bytes out."""
    n, d = code.shape
    Q = torch.zeros(n, -(-d // 256) * 128, dtype=torch.uint8, device=code.device)
    k = torch.arange(d)
    Q[:, k[k % 2 == 0] // 2] = code[:, 0::2]
    Q[:, k[k % 2 == 1] // 2] |= code[:, 1::2] << 4
    S = torch.zeros(n, -(-d // 512) * 16, dtype=torch.uint8, device=code.device)
    j = torch.arange(scale.shape[1])
    c, b = j // 4, j % 4
    S[:, 16 * (c // 4) + 4 * b + c % 4] = scale
    return Q, S


def token_logprobs(x: torch.Tensor, tokens: torch.Tensor, scale: float = 1.0):
    """lse, logp, entropy of logits x, float64."""
    z = x.double() * scale
    n, vocab = z.shape
    m = z.amax(1)
    # From the largest on: beside logits of 1e38 a logarithm of the vocabulary is lost.
    y = z - m.unsqueeze(1)
    rest = torch.logsumexp(y, 1)
    lse = m + rest
    logs = y - rest.unsqueeze(1)
    p = torch.exp(logs)
    entropy = -torch.where(p > 0, p * logs, p * 0).sum(1)
    logp = logs[torch.arange(n, device=z.device), tokens.clamp(0, vocab - 1)]
    none = m == -float("inf")
    entropy[none] = 0.0
    lse[none] = -float("inf")
    logp[none] = -float("inf")
    wrong = ~none & (torch.isnan(z).any(1) | (m == float("inf")))
    for o in (lse, logp, entropy):
        o[wrong] = float("nan")
    logp[tokens < 0] = 0.0
    logp[tokens >= vocab] = float("nan")
    return lse, logp, entropy


def top(x: torch.Tensor, k: int) -> torch.Tensor:
    """Places of the k largest of each row, equal ones by rising place."""
    return torch.sort(x.double(), dim=1, descending=True, stable=True).indices[:, :k]


def token_logprobs_gradient(x, tokens, dlogp, dentropy, dlse, scale: float = 1.0):
    """The gradient of sum(dlogp logp + dentropy entropy + dlse lse) in x, float64, from the
    definition: d logp = onehot - p, d entropy = -p (log p + entropy), d lse = p. 0 where nothing
    is left of a row: its lse is -inf or below -1e30."""
    z = x.double() * scale
    lse = torch.logsumexp(z, 1, keepdim=True)
    logs = z - lse
    p = torch.exp(logs)
    safe = torch.where(p > 0, logs, torch.zeros_like(logs))
    entropy = -(p * safe).sum(1, keepdim=True)
    given = (tokens >= 0) & (tokens < x.shape[1])
    g = torch.where(given, dlogp.double(), 0.0).unsqueeze(1)
    d = -g * p - dentropy.double().unsqueeze(1) * p * (safe + entropy)
    d = d + dlse.double().unsqueeze(1) * p
    d.scatter_add_(1, tokens.clamp(0, x.shape[1] - 1).unsqueeze(1), g)
    d[lse.squeeze(1) < -1e30] = 0.0
    return d * scale
