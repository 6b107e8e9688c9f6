"""4-bit weights against the fp64 oracle: codes and scales bit for bit, products within
what fp32 sums may be off by.

Tolerances. U = 2^-24, B = 2^-8 (half a bf16 step). 16-bit activations: an offset of 24
steps is added to and taken off every code, so that the sums of a group hold magnitudes
of up to 24 + 31 steps; with at most 128 + 8 additions a group, and one for each group and
wave, Y is off by less than (160 U) sum |x| 55 s + (groups + 16) U sum |x w|. 8-bit
activations: whole numbers within a group, so only the second part."""
import numpy as np
import pytest
import torch

from gpu_util import dev
from oracle import feedforward_oracle as F

pytestmark = pytest.mark.gpu

U, B = 2.0 ** -24, 2.0 ** -8
T = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def L():
    import paper_2512_13886_amd as lib
    return lib


def _np(t):
    return t.double().cpu().numpy()


def _weights(g, n, d, dt="f32"):
    w = torch.randn(n, d, generator=g, device=dev()) * torch.exp(
        torch.randn(n, 1, generator=g, device=dev()))
    w *= torch.rand(n, d, generator=g, device=dev()) < 0.6
    return w.to(T[dt])


def _pack(L, W, group):
    n, d = W.shape
    Q = torch.full((n, L.optima_w4_row_bytes(d)), 0xAB, dtype=torch.uint8, device=dev())
    sc = torch.full((n, -(-d // group)), float("nan"), device=dev()).bfloat16()
    L.optima_w4_pack(W, Q, sc, group=group)
    return Q, sc


@pytest.mark.parametrize("n, d", [(1, 1), (3, 31), (17, 128), (5, 129), (16, 1000), (33, 4096),
                                  (300, 130)])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_pack(L, n, d, group, dt):
    g = torch.Generator(device=dev()).manual_seed(n + d + group)
    W = _weights(g, n, d, dt)
    W[0] = 0
    Q, sc = _pack(L, W, group)
    codes, scales = F.w4_quantize(W.float().cpu().numpy(), group)
    assert np.array_equal(_np(sc), scales)
    assert np.array_equal(Q.cpu().numpy(), F.w4_layout(codes))
    assert L.optima_w4_row_bytes(d) == Q.shape[1]


def test_pack_nonfinite_and_extremes(L):
    W = torch.zeros(3, 96, device=dev())
    W[0, 3], W[0, 40], W[0, 70] = float("nan"), float("inf"), 1.0
    W[1, :32] = 3.4e38      # the scale is the largest, codes 7
    W[2, :32] = 1e-44       # the scale rounds to zero
    Q, sc = _pack(L, W, 32)
    s = sc.float().cpu().numpy()
    assert np.isnan(s[0, 0]) and np.isinf(s[0, 1]) and np.isfinite(s[0, 2])
    q = Q.cpu().numpy()
    assert np.all(q[0, [b * 16 + k for b in range(4) for k in range(8)]] == 0x88)
    assert np.isfinite(s[1:]).all()
    codes, scales = F.w4_quantize(W[1:].cpu().numpy(), 32)
    assert np.array_equal(s[1:], scales) and np.array_equal(q[1:], F.w4_layout(codes))


def _tokens(g, n, d, x, x_group, pitch):
    """X, its scales and the values it stands for, from rows of `pitch`."""
    if x == "bf16":
        X = torch.randn(n, pitch, generator=g, device=dev()).bfloat16()[:, :d]
        return X, None, _np(X)
    X = torch.randint(-127, 128, (n, pitch), generator=g, device=dev()).to(torch.int8)[:, :d]
    groups = -(-d // x_group) if x_group else 1
    sc = torch.rand(n, groups, generator=g, device=dev()) * 0.02
    return X, sc, _np(X) * _np(sc)[:, F.groups_of(d, x_group)]


def _bound(x, codes, scales, group, exact):
    each = scales[:, F.groups_of(codes.shape[1], group)]
    fine = (scales.shape[1] + 16) * U * (np.abs(x) @ np.abs(codes * each).T)
    return fine if exact else fine + 160 * U * 55 * (np.abs(x) @ each.T)


def _run(L, n, d, n_out, group, x, x_group, y="f32", pad=0, gated=None):
    g = torch.Generator(device=dev()).manual_seed(n + 3 * d + 5 * n_out + group)
    X, xs, xv = _tokens(g, n, d, x, x_group, d + pad)
    Q, sc = _pack(L, _weights(g, n_out, d), group)
    codes, scales = F.w4_quantize(_unpacked(Q, sc, group, d), group)
    buf = torch.full((n + 1, n_out + 3), 77.0, device=dev()).to(T[y])
    Y = buf[:n, :n_out]
    w = F.w4_values(codes, scales, group)
    ref, e = xv @ w.T, _bound(xv, codes, scales, group, x == "i8")
    half = {"f32": 4 * U, "bf16": 1.01 * B}[y]
    if gated is None:
        L.optima_w4_linear(X, Q, sc, Y, group=group, x_scales=xs, x_group=x_group)
    else:
        Q2, sc2 = _pack(L, _weights(g, n_out, d), group)
        c2, s2 = F.w4_quantize(_unpacked(Q2, sc2, group, d), group)
        L.optima_w4_gated(X, Q, sc, Q2, sc2, Y, group=group, act=1 if gated == "silu" else 0,
                          x_scales=xs, x_group=x_group)
        u, eu = xv @ F.w4_values(c2, s2, group).T, _bound(xv, c2, s2, group, x == "i8")
        a = F.act(gated, ref)
        e = 1.1 * e * np.abs(u) + np.abs(a) * eu + 1.1 * e * eu + \
            8 * U * (1 + np.abs(ref)) * np.abs(a * u)
        ref = a * u
    assert np.all(np.abs(_np(Y) - ref) <= e * (1 + 2 * half) + half * np.abs(ref) + 1e-36)
    assert bool((buf[:, n_out:] == 77).all()) and bool((buf[n:] == 77).all())


def _unpacked(Q, sc, group, d):
    """The weights that Q and sc stand for, by the layout, float32."""
    q = Q.cpu().numpy()
    k = np.arange(d)
    i, e = k % 128, k % 8
    nib = e // 2 + 4 * (e % 2)
    at = k // 128 * 64 + i % 32 // 8 * 16 + i // 32 * 4 + nib // 2
    codes = ((q[:, at] >> (4 * (nib % 2)).astype(np.uint8)) & 15).astype(np.int64) - 8
    return (codes * _np(sc)[:, F.groups_of(d, group)]).astype(np.float32)


@pytest.mark.parametrize("n", [1, 3, 16, 17, 33, 64, 65, 130])
@pytest.mark.parametrize("d, n_out", [(1, 1), (127, 16), (128, 17), (300, 40), (2100, 33)])
@pytest.mark.parametrize("group, x, x_group", [(32, "bf16", 0), (128, "bf16", 0), (32, "i8", 32),
                                               (64, "i8", 0), (128, "i8", 128)])
def test_linear(L, n, d, n_out, group, x, x_group):
    _run(L, n, d, n_out, group, x, x_group, y="f32", pad=3)


@pytest.mark.parametrize("n", [1, 20, 70])
@pytest.mark.parametrize("d, n_out", [(100, 20), (1000, 50)])
@pytest.mark.parametrize("group, x, x_group", [(64, "bf16", 0), (64, "i8", 64), (128, "i8", 0)])
@pytest.mark.parametrize("gated", ["silu", "none"])
def test_gated(L, n, d, n_out, group, x, x_group, gated):
    _run(L, n, d, n_out, group, x, x_group, y="bf16", gated=gated)
    _run(L, n, d, n_out, group, x, x_group, y="f32", pad=1, gated=gated)


# Several workgroups of outputs, several 64 tokens and a split sum at once.
@pytest.mark.parametrize("n, d, n_out", [(300, 2100, 300), (129, 4096, 520)])
@pytest.mark.parametrize("group, x, x_group", [(64, "bf16", 0), (64, "i8", 64)])
@pytest.mark.parametrize("gated", [None, "silu"])
def test_many_tokens(L, n, d, n_out, group, x, x_group, gated):
    _run(L, n, d, n_out, group, x, x_group, y="f32", pad=1, gated=gated)


def test_wide(L):
    _run(L, 1, 14336, 512, 128, "i8", 128, y="bf16")
    _run(L, 5, 14336, 512, 64, "bf16", 0, y="f32")
    _run(L, 2, 4096, 4096, 32, "i8", 0, y="bf16", gated="silu")


def test_norm_output_is_taken(L):
    # The 8-bit output of the norm as it comes, through a gated product and back.
    g = torch.Generator(device=dev()).manual_seed(3)
    n, d, ff, group = 4, 300, 90, 64
    X = torch.randn(n, d, generator=g, device=dev()).bfloat16()
    w = torch.rand(d, generator=g, device=dev()) + 0.5
    q = torch.empty(n, d, dtype=torch.int8, device=dev())
    for grp in (0, group):
        sc = torch.empty(n, -(-d // grp) if grp else 1, device=dev())
        L.optima_rms_norm(X, w, q, scales=sc, group=grp)
        Qg, sg = _pack(L, _weights(g, ff, d), group)
        Qu, su = _pack(L, _weights(g, ff, d), group)
        H = torch.empty(n, ff, device=dev())
        L.optima_w4_gated(q, Qg, sg, Qu, su, H, group=group, x_scales=sc, x_group=grp)
        xv = _np(q) * _np(sc)[:, F.groups_of(d, grp)]
        a, b = xv @ _unpacked(Qg, sg, group, d).T, xv @ _unpacked(Qu, su, group, d).T
        ref = F.act("silu", a) * b
        assert np.linalg.norm(_np(H) - ref) <= 1e-5 * np.linalg.norm(ref)


def test_nonfinite(L):
    g = torch.Generator(device=dev()).manual_seed(4)
    X = torch.randn(3, 200, generator=g, device=dev()).bfloat16()
    Q, sc = _pack(L, _weights(g, 40, 200), 64)
    ref, Y = torch.empty(3, 40, device=dev()), torch.empty(3, 40, device=dev())
    L.optima_w4_linear(X, Q, sc, ref, group=64)
    X[1, 199] = float("nan")
    sc[7, 0] = float("nan")
    L.optima_w4_linear(X, Q, sc, Y, group=64)
    keep = [i for i in range(40) if i != 7]
    assert torch.equal(Y[[0, 2]][:, keep], ref[[0, 2]][:, keep])
    assert bool(Y[1].isnan().all()) and bool(Y[:, 7].isnan().all())


def test_graph_and_side_stream(L):
    g = torch.Generator(device=dev()).manual_seed(5)
    X = torch.randn(2, 512, generator=g, device=dev()).bfloat16()
    W = _weights(g, 128, 512)
    Q, sc = _pack(L, W, 128)
    Y = torch.empty(2, 128, device=dev())

    def step(stream=None):
        L.optima_w4_pack(W, Q, sc, stream=stream)
        L.optima_w4_linear(X, Q, sc, Y, stream=stream)

    step()
    ref = Y.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    torch.cuda.synchronize()
    assert torch.equal(ref, Y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        X.copy_(torch.randn(2, 512, generator=g, device=dev()))
        graph.replay()
        torch.cuda.synchronize()
        got = Y.clone()
        step()
        torch.cuda.synchronize()
        assert torch.equal(got, Y)


def test_offsets_past_32_bits(L):
    # Packed weights of more than 2^32 bytes, from 2^33 values.
    n, d, group = (1 << 20) + 3, 8192, 128
    g = torch.Generator(device=dev()).manual_seed(3)
    W = torch.zeros((n, d), dtype=torch.bfloat16, device=dev())
    at = torch.tensor([0, 5, 262143, 262144, 524287, 524288, n - 4, n - 1], device=dev())
    W[at] = torch.randn((len(at), d), generator=g, device=dev()).bfloat16()
    Q, sc = _pack(L, W, group)
    q, s = _pack(L, W[at], group)
    assert torch.equal(Q[at], q) and torch.equal(sc[at], s)
    for tokens in (1, 40):
        X = torch.randn((tokens, d), generator=g, device=dev()).bfloat16()
        Y = torch.empty((tokens, n), dtype=torch.float32, device=dev())
        y = torch.empty((tokens, len(at)), dtype=torch.float32, device=dev())
        L.optima_w4_linear(X, Q, sc, Y, group)
        L.optima_w4_linear(X, q, s, y, group)
        # The same groups' sums, added in another order where the few rows' sums are split.
        assert torch.allclose(Y[:, at], y, rtol=0, atol=float(d * 2.0 ** -24 * y.abs().max() * 8))
        rest = torch.ones(n, dtype=torch.bool, device=dev())
        rest[at] = False
        assert bool((Y[:, rest] == 0).all())


def test_no_tokens(L):
    g = torch.Generator(device=dev()).manual_seed(6)
    Q, sc = _pack(L, _weights(g, 20, 64), 64)
    X = torch.empty(0, 64, dtype=torch.bfloat16, device=dev())
    L.optima_w4_linear(X, Q, sc, torch.empty(0, 20, device=dev()), group=64)
    E = torch.empty(0, 64, device=dev())
    L.optima_w4_pack(E, torch.empty(0, 64, dtype=torch.uint8, device=dev()),
                     torch.empty(0, 1, dtype=torch.bfloat16, device=dev()), group=64)
