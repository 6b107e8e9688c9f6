"""The gated gradient against the fp64 oracle: fp32 inside, rounded once at the end.

Tolerances. U = 2^-24, B = 2^-8 (half a bf16 step). dG and dU come in two bf16 parts: cut to
bf16, and the rest, below 2^-7 of the value, rounded to its own upper eight bits, so that each is
within 2^-16 of its value. Both parts' products are summed in fp32: 2 K U of the sum of
magnitudes over K. The activation's slope may cancel: 16 U of its two parts. Over many entries the
parts' roundings are independent, so that the Frobenius norm is off by less than 2^-16 of itself, by
less than 2^-14 with the fp32 sums, and by the output's rounding: B / sqrt(3) at most, that of
values just above powers of two."""
import numpy as np
import pytest
import torch

from gpu_util import dev, rel_fro
from oracle import feedforward_oracle as F

pytestmark = pytest.mark.gpu

U, B, PARTS = 2.0 ** -24, 2.0 ** -8, 2.0 ** -16
T = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def L():
    import paper_2512_13886_amd as lib
    return lib


def _np(t):
    return t.double().cpu().numpy()


def _inputs(n, d, ff, seed):
    g = torch.Generator(device=dev()).manual_seed(seed)

    def rows(r, c, scale=1.0):
        return (scale * torch.randn(r, c, generator=g, device=dev())).bfloat16()

    return (rows(n, d), rows(ff, d, d ** -0.5), rows(ff, d, d ** -0.5), rows(n, ff), rows(n, ff),
            rows(n, ff)), g


# Small tiles and large ones, split sums, ragged sizes, one token.
@pytest.mark.parametrize("n, d, ff", [(1, 1, 1), (5, 100, 33), (65, 64, 63), (300, 200, 129),
                                      (1999, 1001, 2731)])
@pytest.mark.parametrize("dx, dw", [("f32", "f32"), ("f32", "bf16"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("name", ["silu", "none"])
def test_outputs_are_rounded_once(L, n, d, ff, dx, dw, name):
    (X, Wg, Wu, G, V, dH), g = _inputs(n, d, ff, n + d + ff)
    mask = (torch.rand(ff, d, generator=g, device=dev()) < 0.5).to(torch.uint8)
    dX = torch.empty(n, d, dtype=T[dx], device=dev())
    dWg, dWu = (torch.empty(ff, d, dtype=T[dw], device=dev()) for _ in range(2))
    L.optima_gated_backward(X, Wg, Wu, G, V, dH, dX=dX, dWg=dWg, dWu=dWu,
                            act=1 if name == "silu" else 0, mask_g=mask)
    x, wg, wu, gg, u, dh = (_np(t) for t in (X, Wg, Wu, G, V, dH))
    rx, rg, ru, dg, du = F.gated_backward(x, wg, wu, gg, u, dh, name)
    slope = np.abs(dh * u) * 16 * U * (1 + np.abs(gg))
    act = np.abs(dh * gg) * 16 * U * (1 + np.abs(gg))
    checks = [(dX, rx, np.abs(dg) @ np.abs(wg) + np.abs(du) @ np.abs(wu),
               slope @ np.abs(wg) + act @ np.abs(wu), 4 * ff, dx, 1.0)]
    for got, ref, p, ex, m in ((dWg, rg, dg, slope, _np(mask)), (dWu, ru, du, act, 1.0)):
        checks.append((got, ref * m, np.abs(p).T @ np.abs(x), ex.T @ np.abs(x), 2 * n, dw, m))
    for got, ref, size, extra, k, out, m in checks:
        half = {"f32": U, "bf16": 1.01 * B}[out]
        bound = (1 + half) * ((PARTS + (k + 64) * U) * size + 2 * extra) + half * np.abs(ref) + 1e-36
        assert np.all(np.abs(_np(got) - ref) <= bound * m)
        if np.count_nonzero(ref) > 1000:
            assert rel_fro(_np(got), ref) <= 2.0 ** -14 + (B / 3 ** 0.5 if out == "bf16" else 0.0)


def test_infinities_are_those_of_the_values(L):
    # One infinite value in X, in Wg and in dH. Products with it are infinite or NaN as the
    # value's own would be, in both parts alike; nothing else changes.
    n, d, ff = 70, 64, 48
    (X, Wg, Wu, G, V, dH), _ = _inputs(n, d, ff, 3)
    X[7, 5] = float("inf")
    Wg[11, 9] = float("-inf")
    dH[20, 30] = float("inf")
    dH[21, 11] = 0.0   # 0 times the infinite weight
    dH[22, 11] = 1.0
    V[22, 11] = 1.0
    G[22, 11] = 1.0    # act' = 0.928: a rest; with the identity below: none
    for name in ("silu", "none"):
        dX = torch.empty(n, d, device=dev())
        dWg, dWu = (torch.empty(ff, d, device=dev()) for _ in range(2))
        L.optima_gated_backward(X, Wg, Wu, G, V, dH, dX=dX, dWg=dWg, dWu=dWu,
                                act=1 if name == "silu" else 0)
        x, wg, wu, gg, u, dh = (_np(t) for t in (X, Wg, Wu, G, V, dH))
        with np.errstate(invalid="ignore"):
            rx, rg, ru, _, _ = F.gated_backward(x, wg, wu, gg, u, dh, name)
        for got, ref in ((dX, rx), (dWg, rg), (dWu, ru)):
            got = _np(got)
            for kind in (np.isnan, np.isposinf, np.isneginf):
                assert np.array_equal(kind(got), kind(ref))
        assert np.isneginf(rx[22, 9]) and np.isnan(rx[21, 9])
