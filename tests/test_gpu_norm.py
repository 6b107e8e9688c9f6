"""RMS norm with the residual's addition, its 8-bit output and its gradient, against
the fp64 oracle.

Tolerances. U = 2^-24 is half an fp32 step, B = 2^-8 half a bf16 step. A sum over a row
takes at most 16 additions in a thread, 6 in a wave and 16 over waves; with the products,
the division and the root a forward value is off by less than 64 U relative. The
gradient's terms are each off by less than 64 U of what they are sums of."""
import numpy as np
import pytest
import torch

from gpu_util import dev
from oracle import feedforward_oracle as F

pytestmark = pytest.mark.gpu

U, B = 2.0 ** -24, 2.0 ** -8
EPS = 1e-5
T = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def L():
    import paper_2512_13886_amd as lib
    return lib


def _rows(g, n, d, dt, pitch=None, scale=1.0):
    """[n, d] of a wider buffer (pitch d + 3 or d)."""
    pitch = pitch or d
    wide = scale * torch.randn(max(n, 1), pitch, generator=g, device=dev())
    return wide.to(dt)[:n, :d]


def _out(n, d, dt, pitch):
    """An output in a wider buffer of sentinels, and the buffer."""
    buf = torch.full((n + 1, pitch), 77, device=dev()).to(dt)
    return buf[:n, :d], buf


def _untouched(buf, n, d):
    return bool((buf[:, d:] == 77).all()) and bool((buf[n:] == 77).all())


def _np(t):
    return t.double().cpu().numpy()


# Every width of by_width, its edges, and rows that end inside a chunk of 8.
WIDTHS = [1, 7, 8, 9, 64, 65, 128, 129, 200, 256, 257, 511, 512, 513, 1000, 1024, 1025, 2048, 2049, 4095, 4096, 4100,
          6144, 6145, 8192, 8199, 12288, 12290, 16384]


@pytest.mark.parametrize("d", WIDTHS)
@pytest.mark.parametrize("dt, out, residual", [("bf16", "bf16", True), ("f32", "f32", True),
                                               ("bf16", "f32", False), ("f32", "bf16", False)])
def test_forward(L, d, dt, out, residual):
    n = 5
    g = torch.Generator(device=dev()).manual_seed(d)
    X = _rows(g, n, d, T[dt], d + 3, 2.0)
    R = _rows(g, n, d, T[dt], d + 1) if residual else None
    w = _rows(g, 1, d, T[out])[0].contiguous()
    Y, ybuf = _out(n, d, T[out], d + 5)
    S, sbuf = _out(n, d, T[dt], d + 2) if residual else (None, None)
    L.optima_rms_norm(X, w, Y, eps=EPS, R=R, S=S)
    s, y = F.rms_norm(_np(X), None if R is None else _np(R), _np(w), EPS)
    half = {"f32": U, "bf16": B}
    # x + r is rounded once, relative to s itself
    assert np.all(np.abs(_np(Y) - y) <= (64 * U + half[out]) * np.abs(y) * 1.01 + 1e-37)
    assert _untouched(ybuf, n, d)
    if residual:
        assert np.all(np.abs(_np(S) - s) <= (U + half[dt]) * np.abs(s) * 1.01)
        assert _untouched(sbuf, n, d)


@pytest.mark.parametrize("d", [1, 31, 32, 64, 100, 130, 512, 1000, 1500, 4096, 5001, 7000, 12000,
                               16384])
@pytest.mark.parametrize("group", [0, 32, 64, 128])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_eight_bits(L, d, group, dt):
    n = 6
    g = torch.Generator(device=dev()).manual_seed(d + group)
    X = _rows(g, n, d, T[dt], d + 3)
    X[2] = 0  # a row of zeros
    w = _rows(g, 1, d, torch.float32)[0].contiguous()
    Y, ybuf = _out(n, d, torch.int8, d + 5)
    scales = torch.full((n, -(-d // group) if group else 1), float("nan"), device=dev())
    L.optima_rms_norm(X, w, Y, eps=EPS, scales=scales, group=group)
    _, y = F.rms_norm(_np(X), None, _np(w), EPS)
    top = F.group_max(y, group) / 127
    sc = _np(scales)
    assert np.all(np.abs(sc - top) <= 70 * U * top)
    q = _np(Y)
    assert np.all(np.abs(q) <= 127)
    each = sc[:, F.groups_of(d, group)]
    # half a step, and 64 U of values of up to 127 steps
    assert np.all(np.abs(q * each - y) <= each * (0.5 + 130 * 70 * U))
    assert np.all(q[2] == 0) and np.all(sc[2] == 0)
    assert _untouched(ybuf, n, d)


@pytest.mark.parametrize("d", [5, 33, 96, 200, 777])
def test_many_rows(L, d):
    # Rows that share a wave, and a last workgroup that is not full.
    n = 10007
    g = torch.Generator(device=dev()).manual_seed(1)
    X, w = _rows(g, n, d, torch.bfloat16), torch.ones(d, device=dev())
    Y = torch.empty(n, d, device=dev())
    L.optima_rms_norm(X, w, Y, eps=EPS)
    _, y = F.rms_norm(_np(X), None, np.ones(d), EPS)
    assert np.all(np.abs(_np(Y) - y) <= 65 * U * np.abs(y))


def test_in_place(L):
    g = torch.Generator(device=dev()).manual_seed(2)
    for d in (100, 3000, 9000):
        X, R = _rows(g, 9, d, torch.bfloat16), _rows(g, 9, d, torch.bfloat16)
        w = torch.ones(d, device=dev())
        Y, S = torch.empty_like(X), torch.empty_like(X)
        L.optima_rms_norm(X, w, Y, R=R, S=S)
        X2, R2 = X.clone(), R.clone()
        L.optima_rms_norm(X2, w, X2, R=R2, S=R2)
        assert torch.equal(X2, Y) and torch.equal(R2, S)


def test_nonfinite_stays_in_its_row_and_group(L):
    d = 1000
    g = torch.Generator(device=dev()).manual_seed(4)
    X = _rows(g, 5, d, torch.float32)
    w = torch.ones(d, device=dev())
    ref = torch.empty(5, d, device=dev())
    L.optima_rms_norm(X, w, ref)
    X[1, 17], X[3, 999] = float("nan"), float("inf")
    Y = torch.empty(5, d, device=dev())
    L.optima_rms_norm(X, w, Y)
    assert torch.equal(Y[[0, 2, 4]], ref[[0, 2, 4]])
    assert bool(Y[1].isnan().all())
    # 1 / sqrt(inf) = 0: zeros, and inf * 0 where the infinity was
    assert bool(Y[3, 999].isnan()) and bool((Y[3, :999] == 0).all())
    # A weight that is not finite reaches its own group only.
    X = _rows(g, 5, d, torch.float32)
    w[200] = float("inf")
    q = torch.empty(5, d, dtype=torch.int8, device=dev())
    sc = torch.empty(5, 16, device=dev())
    L.optima_rms_norm(X, w, q, scales=sc, group=64)
    assert bool(sc[:, 3].isinf().all()) and bool((q[:, 192:256] == 0).all())
    assert bool(sc[:, [i for i in range(16) if i != 3]].isfinite().all())
    X[0, 5] = float("nan")
    sc1 = torch.empty(5, 1, device=dev())
    L.optima_rms_norm(X, torch.ones(d, device=dev()), q, scales=sc1)
    assert bool(sc1[0].isnan().all()) and bool((q[0] == 0).all()) and bool(sc1[1:].isfinite().all())


@pytest.mark.parametrize("d", [1, 8, 60, 100, 250, 512, 1000, 2048, 4096, 4100, 8192, 16384])
@pytest.mark.parametrize("dt, n, residual", [("bf16", 1, True), ("f32", 7, False),
                                             ("bf16", 2500, True)])
def test_backward(L, d, dt, n, residual):
    n = min(n, 4_000_000 // d + 1)
    g = torch.Generator(device=dev()).manual_seed(d + n)
    S = _rows(g, n, d, T[dt], d + 3)
    dY = _rows(g, n, d, T[dt], d + 1)
    dS = _rows(g, n, d, T[dt], d + 2) if residual else None
    w = _rows(g, 1, d, T[dt])[0].contiguous()
    dX, buf = _out(n, d, T[dt], d + 5)
    dw = torch.full((d,), float("nan"), device=dev())
    L.optima_rms_norm_backward(S, w, dY, dX, eps=EPS, dS=dS, dweight=dw)
    s, wn, dy = _np(S), _np(w), _np(dY)
    ds = None if dS is None else _np(dS)
    dx, dwn = F.rms_norm_backward(s, wn, dy, ds, EPS)
    rstd = 1 / np.sqrt(np.mean(s * s, axis=1, keepdims=True) + EPS)
    p, xh = np.abs(dy * wn), np.abs(s * rstd)
    size = rstd * (p + xh * np.mean(p * xh, axis=1, keepdims=True))
    if ds is not None:
        size = size + np.abs(ds)
    half = {"f32": U, "bf16": B}[dt]
    assert np.all(np.abs(_np(dX) - dx) <= 64 * U * size + half * 1.01 * np.abs(dx))
    assert _untouched(buf, n, d)
    # rows in a workgroup, its waves, the workgroups' partial sums, and the products
    adds = n / 256 + 4 + 64 + 16 + 64
    assert np.all(np.abs(_np(dw) - dwn) <= adds * U * np.sum(np.abs(dy) * xh, axis=0))
    # the same, added to what is there, and without it
    dw2 = dw.clone()
    dX2 = torch.empty(n, d, dtype=T[dt], device=dev())
    L.optima_rms_norm_backward(S, w, dY, dX2, eps=EPS, dS=dS, dweight=dw2, accumulate=True)
    assert torch.equal(dX2, dX) and torch.equal(dw2, dw + dw)
    dX3 = torch.empty(n, d, dtype=T[dt], device=dev())
    L.optima_rms_norm_backward(S, w, dY, dX3, eps=EPS, dS=dS)
    assert torch.equal(dX3, dX)


def test_backward_against_differences(L):
    # The library's own forward pass, in fp32 on a small row: central differences of
    # 2^-6 have a truncation error of h^2 / 6 times the third derivative (below 1 for
    # these sizes) and a rounding error of 64 U |y| d / h.
    d, h = 9, 2.0 ** -6
    g = torch.Generator(device=dev()).manual_seed(9)
    S, dY = _rows(g, 1, d, torch.float32, scale=2.0), _rows(g, 1, d, torch.float32)
    w = torch.ones(d, device=dev())
    dX, Y = torch.empty_like(S), torch.empty_like(S)
    L.optima_rms_norm_backward(S, w, dY, dX, eps=EPS)
    for i in range(d):
        v = []
        for sign in (1, -1):
            P = S.clone()
            P[0, i] += sign * h
            L.optima_rms_norm(P, w, Y, eps=EPS)
            v.append((Y.double() * dY.double()).sum().item())
        assert abs((v[0] - v[1]) / (2 * h) - dX[0, i].item()) <= h * h / 6 * 10 + 64 * U * 30 / h


def test_backward_in_place_and_no_rows(L):
    g = torch.Generator(device=dev()).manual_seed(3)
    S, dY = _rows(g, 33, 1500, torch.bfloat16), _rows(g, 33, 1500, torch.bfloat16)
    dS, w = _rows(g, 33, 1500, torch.bfloat16), torch.ones(1500, device=dev())
    dX = torch.empty_like(S)
    L.optima_rms_norm_backward(S, w, dY, dX, dS=dS)
    a, b = dY.clone(), dS.clone()
    L.optima_rms_norm_backward(S, w, a, a, dS=dS)
    L.optima_rms_norm_backward(S, w, dY, b, dS=b)
    assert torch.equal(a, dX) and torch.equal(b, dX)
    dw = torch.full((1500,), 3.0, device=dev())
    E = S[:0]
    L.optima_rms_norm_backward(E, w, E, torch.empty_like(E), dweight=dw, accumulate=True)
    assert bool((dw == 3).all())
    L.optima_rms_norm_backward(E, w, E, torch.empty_like(E), dweight=dw)
    assert bool((dw == 0).all())
    L.optima_rms_norm(E, w, torch.empty_like(E))


def test_graph_replays_equal_eager_calls(L):
    g = torch.Generator(device=dev()).manual_seed(8)
    X, R = _rows(g, 64, 4096, torch.bfloat16), _rows(g, 64, 4096, torch.bfloat16)
    w = torch.ones(4096, device=dev())
    Y, S, dX = (torch.empty_like(X) for _ in range(3))
    dw = torch.empty(4096, device=dev())
    ws = torch.empty(L.optima_rms_norm_backward_workspace_bytes(64, 4096), dtype=torch.uint8,
                     device=dev())

    def step():
        L.optima_rms_norm(X, w, Y, R=R, S=S)
        L.optima_rms_norm_backward(S, w, Y, dX, dweight=dw, ws=ws)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(3):
        X.copy_(_rows(g, 64, 4096, torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (Y, S, dX, dw)]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (Y, S, dX, dw))), k


def test_more_threads_than_a_launch_has(L):
    # 256 threads a row: rows past 2^32 / 256 need another launch (and pass 2^31 elements).
    n, d = (1 << 24) + 5, 1025
    X = torch.empty((n, d), dtype=torch.bfloat16, device=dev())
    Y = torch.empty_like(X)
    g = torch.Generator(device=dev()).manual_seed(1)
    w = torch.randn(d, generator=g, device=dev())
    at = [0, 1 << 22, (1 << 22) + 1, (1 << 24) - 1, 1 << 24, n - 1]
    X[at] = torch.randn((len(at), d), generator=g, device=dev()).bfloat16()
    L.optima_rms_norm(X, w, Y)
    want = torch.empty((len(at), d), dtype=torch.bfloat16, device=dev())
    L.optima_rms_norm(X[at], w, want)
    assert torch.equal(Y[at], want)
