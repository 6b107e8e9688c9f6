"""The gated gradient's fp32 outputs against the fp64 oracle.

Tolerances. U = 2^-24. dG and dU come in two bf16 parts: cut to bf16 (the rest is below 2^-7
of the value) and the rest rounded (2^-9 of it), so that each is within 2^-16 of its value.
Both parts' products are summed in fp32: 2 K U of the sum of magnitudes over K. The
activation's slope may cancel: 16 U of its two parts. Over many entries the parts' roundings
are independent, so that the Frobenius norm is off by less than 2^-16 of itself, and by less
than 2^-14 with the fp32 sums."""
import numpy as np
import pytest
import torch

from gpu_util import dev, rel_fro
from oracle import feedforward_oracle as F

pytestmark = pytest.mark.gpu

U, PARTS = 2.0 ** -24, 2.0 ** -16
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


# Small tiles and large ones, split sums, ragged sizes, one token; the other output in bf16
# or in fp32 too, so that one call forms both kinds of operands.
@pytest.mark.parametrize("n, d, ff", [(1, 1, 1), (5, 100, 33), (65, 64, 63), (300, 200, 129),
                                      (1999, 1001, 2731)])
@pytest.mark.parametrize("dx, dw", [("f32", "f32"), ("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("name", ["silu", "none"])
def test_fp32_outputs(L, n, d, ff, dx, dw, name):
    (X, Wg, Wu, G, V, dH), g = _inputs(n, d, ff, n + d + ff)
    mask = (torch.rand(ff, d, generator=g, device=dev()) < 0.5).to(torch.uint8)
    dX = torch.empty(n, d, dtype=T[dx], device=dev())
    dWg, dWu = (torch.empty(ff, d, dtype=T[dw], device=dev()) for _ in range(2))
    L.optima_gated_backward(X, Wg, Wu, G, V, dH, dX=dX, dWg=dWg, dWu=dWu,
                            act=1 if name == "silu" else 0, mask_g=mask)
    x, wg, wu, gg, u, dh = (_np(t) for t in (X, Wg, Wu, G, V, dH))
    rx, rg, ru, dg, du = F.gated_backward(x, wg, wu, gg, u, dh, name)
    rg = rg * _np(mask)
    slope = np.abs(dh * u) * 16 * U * (1 + np.abs(gg))
    act = np.abs(dh * gg) * 16 * U * (1 + np.abs(gg))
    if dx == "f32":
        size = np.abs(dg) @ np.abs(wg) + np.abs(du) @ np.abs(wu)
        assert np.all(np.abs(_np(dX) - rx) <= (PARTS + (4 * ff + 64) * U) * size +
                      2 * (slope @ np.abs(wg) + act @ np.abs(wu)) + U * np.abs(rx) + 1e-36)
        assert rel_fro(_np(dX), rx) <= 2.0 ** -14
    if dw == "f32":
        for got, ref, p, ex, m in ((dWg, rg, dg, slope, _np(mask)), (dWu, ru, du, act, 1.0)):
            bound = (PARTS + (2 * n + 64) * U) * (np.abs(p).T @ np.abs(x)) + \
                2 * ex.T @ np.abs(x) + U * np.abs(ref) + 1e-36
            assert np.all(np.abs(_np(got) - ref) <= bound * m)
            if np.any(ref):
                assert rel_fro(_np(got), ref) <= 2.0 ** -14


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
