"""fp64 oracle of the feed-forward operators: RMS norm with the residual's
addition, 8-bit codes, the gated product, their gradients, and 4-bit weights.

NumPy, written from the formulas; used by the tests only.
"""
from __future__ import annotations

import numpy as np


def bf16(v: np.ndarray) -> np.ndarray:
    """float32 values rounded to bf16 (nearest even), as float64. NaN stays NaN."""
    f = np.asarray(v, dtype=np.float32)
    u = f.view(np.uint32).astype(np.uint64)
    r = (((u + 0x7FFF + ((u >> 16) & 1)) >> 16) << 16).astype(np.uint32).view(np.float32)
    return np.where(np.isnan(f), np.float32(np.nan), r).astype(np.float64)


# --------------------------------------------------------------------------- RMS norm


def rms_norm(x, r, w, eps):
    """(s, y) with s = x + r and y = s w / sqrt(mean s^2 + eps)."""
    s = np.asarray(x, np.float64) + (0.0 if r is None else np.asarray(r, np.float64))
    rstd = 1.0 / np.sqrt(np.mean(s * s, axis=1, keepdims=True) + eps)
    return s, s * rstd * np.asarray(w, np.float64)


def rms_norm_backward(s, w, dy, ds, eps):
    """(dx, dw) of sum(dy * y) + sum(ds * s) by x and w."""
    s, w, dy = (np.asarray(v, np.float64) for v in (s, w, dy))
    rstd = 1.0 / np.sqrt(np.mean(s * s, axis=1, keepdims=True) + eps)
    xh, p = s * rstd, dy * w
    dx = rstd * (p - xh * np.mean(p * xh, axis=1, keepdims=True))
    if ds is not None:
        dx = dx + np.asarray(ds, np.float64)
    return dx, np.sum(dy * xh, axis=0)


def groups_of(d: int, group: int) -> np.ndarray:
    """Index of the group of every value of a row (group = 0: one)."""
    return np.arange(d) // (group or d)


def group_max(v: np.ndarray, group: int) -> np.ndarray:
    n, d = v.shape
    g = groups_of(d, group)
    out = np.zeros((n, g[-1] + 1))
    for k in range(d):
        out[:, g[k]] = np.maximum(out[:, g[k]], np.abs(v[:, k]))
    return out


# --------------------------------------------------------------------------- gated


def act(name: str, z):
    return z / (1.0 + np.exp(-z)) if name == "silu" else z


def act_slope(name: str, z):
    sig = 1.0 / (1.0 + np.exp(-z))
    return sig * (1.0 + z * (1.0 - sig)) if name == "silu" else np.ones_like(z)


def gated(x, wg, wu, name):
    """(h, g, u) with g = x wg^T, u = x wu^T, h = act(g) u."""
    x, wg, wu = (np.asarray(v, np.float64) for v in (x, wg, wu))
    g, u = x @ wg.T, x @ wu.T
    return act(name, g) * u, g, u


def gated_backward(x, wg, wu, g, u, dh, name):
    """(dx, dwg, dwu, dg, du) of sum(dh * h) at the given g and u."""
    x, wg, wu, g, u, dh = (np.asarray(v, np.float64) for v in (x, wg, wu, g, u, dh))
    du = dh * act(name, g)
    dg = dh * u * act_slope(name, g)
    return dg @ wg + du @ wu, dg.T @ x, du.T @ x, dg, du


# --------------------------------------------------------------------------- 4 bits


def w4_quantize(w: np.ndarray, group: int):
    """(codes [n, d] int, scales [n, groups]) by the rule scale = bf16(max|w| * (1 / 7)),
    code = clamp(rne(w / scale), -7, 7), in fp32 as the rule names it."""
    w = np.asarray(w, np.float32)
    scales = bf16(group_max(w, group).astype(np.float32) * np.float32(1.0 / 7.0)).astype(np.float32)
    each = scales[:, groups_of(w.shape[1], group)]
    with np.errstate(divide="ignore", invalid="ignore"):
        codes = np.where(each > 0, np.clip(np.rint(w / each), -7, 7), 0)
    return codes.astype(np.int64), scales.astype(np.float64)


def w4_layout(codes: np.ndarray) -> np.ndarray:
    """Codes in their packed layout, one by one."""
    n, d = codes.shape
    rows = -(-d // 128) * 64
    out = np.full((n, rows), 0x88, dtype=np.uint8)
    for k in range(d):
        chunk, i = divmod(k, 128)
        dword, rest = divmod(i, 32)
        block, e = divmod(rest, 8)
        nibble = e // 2 + (4 if e % 2 else 0)
        at = chunk * 64 + block * 16 + dword * 4 + nibble // 2
        v = (codes[:, k] + 8).astype(np.uint8)
        if nibble % 2:
            out[:, at] = (out[:, at] & 0x0F) | (v << 4)
        else:
            out[:, at] = (out[:, at] & 0xF0) | v
    return out


def w4_values(codes: np.ndarray, scales: np.ndarray, group: int) -> np.ndarray:
    return codes * scales[:, groups_of(codes.shape[1], group)]
