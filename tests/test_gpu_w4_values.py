"""16-bit tokens against 4-bit weights: every product is exact and only the weights that are
there enter the sums.

Tolerances. U = 2^-24. A product of a bf16 token and a code is exact in fp32; at most 128 of
them are added in a group, then the groups' and the waves' or ranges' sums, each rounded once:
Y is off by less than (128 + groups + 64) U sum |x w|, in which zero weights have no part."""
import numpy as np
import pytest
import torch

from gpu_util import dev
from oracle import feedforward_oracle as F

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module")
def L():
    import paper_2512_13886_amd as lib
    return lib


def _np(t):
    return t.double().cpu().numpy()


def _packed(L, W, group):
    n, d = W.shape
    Q = torch.empty(n, L.optima_w4_row_bytes(d), dtype=torch.uint8, device=dev())
    sc = torch.empty(n, -(-d // group), dtype=torch.bfloat16, device=dev())
    L.optima_w4_pack(W, Q, sc, group=group)
    codes, scales = F.w4_quantize(W.cpu().numpy(), group)
    return Q, sc, F.w4_values(codes, scales, group)


def _weights(g, n, d):
    W = torch.randn(n, d, generator=g, device=dev())
    return W * (torch.rand(n, d, generator=g, device=dev()) < 0.5)


# One wave's tokens and several, both few-token kernels, one and two 64-token tiles, split sums.
@pytest.mark.parametrize("n", [1, 5, 16, 17, 40, 64, 130])
@pytest.mark.parametrize("d, n_out", [(1, 1), (130, 33), (2100, 40)])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_sums_hold_the_weights_that_are_there(L, n, d, n_out, group):
    g = torch.Generator(device=dev()).manual_seed(n + d + group)
    Q, sc, w = _packed(L, _weights(g, n_out, d), group)
    X = torch.randn(n, d, generator=g, device=dev()).bfloat16()
    Y = torch.empty(n, n_out, device=dev())
    L.optima_w4_linear(X, Q, sc, Y, group=group)
    x = _np(X)
    assert np.all(np.abs(_np(Y) - x @ w.T) <=
                  (128 + sc.shape[1] + 64) * U * (np.abs(x) @ np.abs(w).T) + 1e-37)


@pytest.mark.parametrize("n", [1, 5, 16, 20, 64])
@pytest.mark.parametrize("gated", [False, True])
def test_large_tokens_on_pruned_weights_add_nothing(L, n, gated):
    g = torch.Generator(device=dev()).manual_seed(n)
    d, n_out, group = 1100, 50, 64
    W, W2 = _weights(g, n_out, d), _weights(g, n_out, d)
    W[:, ::7] = 0
    W2[:, ::7] = 0
    (Q, sc, _), (Q2, sc2, _) = _packed(L, W, group), _packed(L, W2, group)
    X = torch.randn(n, d, generator=g, device=dev()).bfloat16()
    outs = []
    for large in (0.0, 3e38):
        X[:, ::7] = large
        Y = torch.empty(n, n_out, device=dev())
        if gated:
            L.optima_w4_gated(X, Q, sc, Q2, sc2, Y, group=group)
        else:
            L.optima_w4_linear(X, Q, sc, Y, group=group)
        outs.append(Y)
    assert torch.equal(*outs)


@pytest.mark.parametrize("n", [2, 16, 20, 70])
def test_infinite_and_very_large_tokens(L, n):
    g = torch.Generator(device=dev()).manual_seed(n)
    d, n_out, group = 300, 40, 32
    W = torch.rand(n_out, d, generator=g, device=dev()) + 0.5
    W *= torch.where(torch.rand(n_out, d, generator=g, device=dev()) < 0.5, 1.0, -1.0)
    W[:, 0] = W[:, 0].sign()
    W[3, 17] = 0.0                          # 0 times infinity
    W[:, 40:] *= 1e-3
    Q, sc, w = _packed(L, W, group)
    X = torch.randn(n, d, generator=g, device=dev()).bfloat16()
    X[0, 17] = float("inf")
    X[1, 50] = float("-inf")
    X[1, 60] = 3e38                         # finite beside the infinity
    X[n - 1, 45] = 3e38                     # the product with 1e-3 is far from infinite
    Y = torch.empty(n, n_out, device=dev())
    L.optima_w4_linear(X, Q, sc, Y, group=group)
    with np.errstate(invalid="ignore"):
        ref = _np(X) @ w.T
    got = _np(Y)
    for kind in (np.isnan, np.isposinf, np.isneginf):
        assert np.array_equal(kind(got), kind(ref))
    assert np.isnan(ref[0, 3]) and np.isinf(ref[0]).sum() == n_out - 1
    if n > 2:
        assert np.isfinite(ref[n - 1]).all()
        assert np.allclose(got[n - 1], ref[n - 1], rtol=1e-5)
