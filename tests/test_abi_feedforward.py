"""Refusals of the feed-forward calls: what the C entry points and the binding return or
raise before any launch. No kernel is launched here."""
import ctypes

import pytest
import torch

i64, vp, i32, f32, sz = (ctypes.c_int64, ctypes.c_void_p, ctypes.c_int, ctypes.c_float,
                         ctypes.c_size_t)
F32, BF16, F64, I8 = 0, 1, 2, 3
INVAL, WORKSPACE, UNSUPPORTED = -1, -4, -5
MB = 1 << 20


@pytest.fixture(scope="module")
def lib():
    import paper_2512_13886_amd as L
    return ctypes.CDLL(L.library_path())


def _norm(lib, **kw):
    """optima_rms_norm of 10 tokens of 64 bf16 values, with changes."""
    a = dict(X=1 * MB, ldx=64, R=None, ldr=64, dtype=BF16, n=10, d=64, w=2 * MB, wdt=F32,
             eps=1e-6, S=None, lds=64, Y=3 * MB, ldy=64, ydt=BF16, scales=None, group=0)
    a.update(kw)
    f = lib.optima_rms_norm
    f.argtypes = [vp, i64, vp, i64, i32, i64, i64, vp, i32, f32, vp, i64, vp, i64, i32, vp, i64, vp]
    return f(*a.values(), None)


@pytest.mark.parametrize("change, status", [
    (dict(X=None), INVAL), (dict(w=None), INVAL), (dict(Y=None), INVAL), (dict(n=-1), INVAL),
    (dict(d=0), INVAL), (dict(ldx=63), INVAL), (dict(ldy=63), INVAL), (dict(eps=0.0), INVAL),
    (dict(eps=float("nan")), INVAL), (dict(X=1 * MB + 1), INVAL), (dict(w=2 * MB + 2), INVAL),
    (dict(dtype=I8), UNSUPPORTED), (dict(wdt=F64), UNSUPPORTED), (dict(ydt=F64), UNSUPPORTED),
    (dict(d=16385, ldx=16385, ldy=16385), UNSUPPORTED), (dict(group=32), INVAL),
    (dict(scales=4 * MB), INVAL), (dict(ydt=I8), INVAL), (dict(ydt=I8, scales=4 * MB, group=48), INVAL),
    (dict(Y=1 * MB + 64), INVAL),                 # over X, shifted
    (dict(Y=1 * MB, ldy=80), INVAL),              # over X, another pitch
    (dict(Y=1 * MB, ydt=F32), INVAL),             # over X, another type
    (dict(S=3 * MB), INVAL),                      # S over Y
    (dict(Y=2 * MB), INVAL),                      # over the weight
    (dict(ydt=I8, scales=1 * MB), INVAL),         # scales over X
    (dict(R=4 * MB, ldr=10), INVAL),
])
def test_norm_refusals(lib, change, status):
    assert _norm(lib, **change) == status


def test_norm_without_tokens_reads_nothing(lib):
    assert _norm(lib, n=0, X=None, Y=None) == 0


def _norm_bwd(lib, **kw):
    a = dict(S=1 * MB, lds=64, w=2 * MB, wdt=F32, dY=3 * MB, lddy=64, dS=None, ldds=64, dtype=BF16,
             n=10, d=64, eps=1e-6, dX=4 * MB, lddx=64, dw=5 * MB, acc=0, ws=None, bytes=0)
    a.update(kw)
    f = lib.optima_rms_norm_backward
    f.argtypes = [vp, i64, vp, i32, vp, i64, vp, i64, i32, i64, i64, f32, vp, i64, vp, i32, vp, sz,
                  vp]
    return f(*a.values(), None)


@pytest.mark.parametrize("change, status", [
    (dict(), WORKSPACE), (dict(ws=6 * MB, bytes=4), WORKSPACE), (dict(ws=6 * MB + 2, bytes=MB), WORKSPACE),
    (dict(S=None), INVAL), (dict(dY=None), INVAL), (dict(dX=None), INVAL), (dict(w=None), INVAL),
    (dict(dX=1 * MB), INVAL),                     # over S
    (dict(dX=3 * MB, lddx=70), INVAL),            # over dY, another pitch
    (dict(dw=3 * MB), INVAL), (dict(dw=5 * MB + 2), INVAL), (dict(eps=-1.0), INVAL),
    (dict(dtype=I8), UNSUPPORTED), (dict(d=20000), UNSUPPORTED),
])
def test_norm_backward_refusals(lib, change, status):
    assert _norm_bwd(lib, **change) == status


def _gated(lib, **kw):
    a = dict(X=1 * MB, ldx=128, n=100, d=128, Wg=2 * MB, Wu=3 * MB, ff=32, act=1, H=4 * MB, ldh=32,
             hdt=BF16, G=None, ldg=32, U=None, ldu=32, ws=None, bytes=0)
    a.update(kw)
    f = lib.optima_gated_forward
    f.argtypes = [vp, i64, i64, i64, vp, vp, i64, i32, vp, i64, i32, vp, i64, vp, i64, vp, sz, vp]
    return f(*a.values(), None)


@pytest.mark.parametrize("change, status", [
    (dict(), WORKSPACE), (dict(ws=8 * MB, bytes=100), WORKSPACE), (dict(X=None), INVAL),
    (dict(Wg=None), INVAL), (dict(Wu=None), INVAL), (dict(H=None), INVAL), (dict(n=-1), INVAL),
    (dict(d=0), INVAL), (dict(ff=0), INVAL), (dict(ff=(1 << 20) + 1), INVAL), (dict(act=2), INVAL),
    (dict(hdt=I8), UNSUPPORTED), (dict(ldx=100), INVAL), (dict(ldh=31), INVAL),
    (dict(Wg=2 * MB + 2), INVAL),                 # rows that suit wide loads, but not aligned
    (dict(X=1 * MB + 1), INVAL), (dict(H=1 * MB), INVAL), (dict(H=2 * MB), INVAL),
    (dict(G=4 * MB), INVAL), (dict(G=5 * MB, U=5 * MB), INVAL), (dict(n=(1 << 31) - 1), INVAL),
])
def test_gated_refusals(lib, change, status):
    assert _gated(lib, **change) == status


def _gated_bwd(lib, **kw):
    a = dict(X=1 * MB, ldx=128, n=100, d=128, Wg=2 * MB, Wu=3 * MB, ff=32, act=1, G=4 * MB, ldg=32,
             U=5 * MB, ldu=32, dH=6 * MB, lddh=32, dX=7 * MB, lddx=128, dxdt=BF16, dWg=8 * MB,
             dWu=9 * MB, dwdt=BF16, mg=None, mu=None, acc=0, ws=None, bytes=0)
    a.update(kw)
    f = lib.optima_gated_backward
    f.argtypes = [vp, i64, i64, i64, vp, vp, i64, i32, vp, i64, vp, i64, vp, i64, vp, i64, i32, vp,
                  vp, i32, vp, vp, i32, vp, sz, vp]
    return f(*a.values(), None)


@pytest.mark.parametrize("change, status", [
    (dict(), WORKSPACE), (dict(ws=16 * MB, bytes=1000), WORKSPACE),
    (dict(ws=16 * MB + 8, bytes=64 * MB), WORKSPACE), (dict(X=None), INVAL), (dict(G=None), INVAL),
    (dict(U=None), INVAL), (dict(dH=None), INVAL), (dict(dX=None, dWg=None, dWu=None), INVAL),
    (dict(dWu=None), INVAL), (dict(dWg=None, dWu=None, mg=10 * MB), INVAL), (dict(dxdt=I8), UNSUPPORTED),
    (dict(dwdt=F64), UNSUPPORTED), (dict(act=7), INVAL), (dict(dWg=2 * MB), INVAL),
    (dict(dWu=8 * MB), INVAL), (dict(dX=6 * MB), INVAL), (dict(dWg=10 * MB, mg=10 * MB), INVAL),
    (dict(lddh=16), INVAL),
])
def test_gated_backward_refusals(lib, change, status):
    assert _gated_bwd(lib, **change) == status


def test_gated_workspace_queries():
    import paper_2512_13886_amd as L
    assert L.optima_gated_forward_workspace_bytes(1, 4096, 14336) == 0
    assert L.optima_gated_forward_workspace_bytes(100, 128, 32) >= 100 * 128 * 2
    assert L.optima_gated_forward_workspace_bytes(100, 100, 32) >= (100 + 64) * 128 * 2
    assert L.optima_gated_forward_workspace_bytes(-1, 128, 32) == 0
    assert L.optima_gated_backward_workspace_bytes(100, 0, 32) == 0
    assert L.optima_rms_norm_backward_workspace_bytes(10, 64) >= 64 * 4
    assert L.optima_rms_norm_backward_workspace_bytes(10, L.NORM_MAX_DIM + 1) == 0


@pytest.mark.parametrize("d", [1, 64, 100, 1000])
def test_gated_workspace_never_shrinks_with_more_tokens(d):
    import paper_2512_13886_amd as L
    for q in (L.optima_gated_forward_workspace_bytes, L.optima_gated_backward_workspace_bytes):
        need = [q(n, d, 200) for n in range(300)]
        assert all(a <= b for a, b in zip(need, need[1:]))
    need = [L.optima_rms_norm_backward_workspace_bytes(n, d) for n in range(3000)]
    assert all(a <= b for a, b in zip(need, need[1:]))


def _pack(lib, **kw):
    a = dict(W=1 * MB, dtype=F32, n=10, d=100, group=64, Q=2 * MB, scales=3 * MB)
    a.update(kw)
    f = lib.optima_w4_pack
    f.argtypes = [vp, i32, i64, i64, i64, vp, vp, vp]
    return f(*a.values(), None)


@pytest.mark.parametrize("change, status", [
    (dict(W=None), INVAL), (dict(Q=None), INVAL), (dict(scales=None), INVAL), (dict(n=-1), INVAL),
    (dict(d=0), INVAL), (dict(group=16), INVAL), (dict(group=0), INVAL), (dict(Q=2 * MB + 8), INVAL),
    (dict(dtype=I8), UNSUPPORTED), (dict(Q=1 * MB), INVAL), (dict(scales=2 * MB), INVAL),
    (dict(n=1 << 24, d=1 << 20), INVAL),
])
def test_pack_refusals(lib, change, status):
    assert _pack(lib, **change) == status


def _w4(lib, gated, **kw):
    a = dict(X=1 * MB, ldx=100, xdt=BF16, xs=None, xg=0, n=4, d=100, Q=2 * MB, sc=3 * MB, Q2=4 * MB,
             sc2=5 * MB, group=64, n_out=10, act=1, Y=6 * MB, ldy=10, ydt=BF16, ws=None, bytes=0)
    a.update(kw)
    if gated:
        f = lib.optima_w4_gated
        f.argtypes = [vp, i64, i32, vp, i64, i64, i64, vp, vp, vp, vp, i64, i64, i32, vp, i64, i32,
                      vp, sz, vp]
        return f(*a.values(), None)
    for k in ("Q2", "sc2", "act"):
        del a[k]
    f = lib.optima_w4_linear
    f.argtypes = [vp, i64, i32, vp, i64, i64, i64, vp, vp, i64, i64, vp, i64, i32, vp, sz, vp]
    return f(*a.values(), None)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("change, status", [
    (dict(X=None), INVAL), (dict(Q=None), INVAL), (dict(sc=None), INVAL), (dict(Y=None), INVAL),
    (dict(xdt=F32), UNSUPPORTED), (dict(ydt=I8), UNSUPPORTED), (dict(xdt=I8), INVAL),
    (dict(xs=7 * MB), INVAL), (dict(xg=64), INVAL), (dict(xdt=I8, xs=7 * MB, xg=32), INVAL),
    (dict(group=100), INVAL), (dict(Q=2 * MB + 4), INVAL), (dict(sc=3 * MB + 1), INVAL),
    (dict(ldx=99), INVAL), (dict(ldy=9), INVAL), (dict(n_out=0), INVAL), (dict(Y=1 * MB), INVAL),
    (dict(Y=2 * MB), INVAL), (dict(n=(1 << 21) + 1), INVAL),
])
def test_w4_refusals(lib, gated, change, status):
    assert _w4(lib, gated, **change) == status


def test_w4_gated_refusals(lib):
    assert _w4(lib, True, Q2=None) == INVAL
    assert _w4(lib, True, sc2=None) == INVAL
    assert _w4(lib, True, act=9) == INVAL
    assert _w4(lib, True, Y=4 * MB) == INVAL
    assert _w4(lib, True, Q2=4 * MB + 8) == INVAL


@pytest.mark.parametrize("mats", [1, 2])
def test_w4_workspace(lib, mats):
    import paper_2512_13886_amd as L
    q = L.optima_w4_workspace_bytes
    assert q(16, 4096, 4096, mats) == 0
    need = [q(n, 4096, 4096, mats) for n in range(200)]
    assert need[17] >= 2 * 4096 * 17 * 4 and all(a <= b for a, b in zip(need, need[1:]))
    assert q(17, 4096, 4096, 3) == 0 and q(-1, 4096, 4096, mats) == 0
    big = dict(n=20, d=4096, ldx=4096, n_out=512, ldy=512, X=16 * MB, Y=32 * MB)
    assert _w4(lib, mats == 2, **big) == WORKSPACE
    assert _w4(lib, mats == 2, **big, ws=64 * MB, bytes=1024) == WORKSPACE
    assert _w4(lib, mats == 2, **big, ws=64 * MB + 8, bytes=64 * MB) == WORKSPACE


def test_row_bytes():
    import paper_2512_13886_amd as L
    assert [L.optima_w4_row_bytes(d) for d in (0, 1, 128, 129, 4096)] == [0, 64, 64, 128, 2048]


def test_binding_refuses_host_tensors_and_wrong_shapes():
    # Checks that come before any pointer is read: the tensors here are on the CPU.
    import paper_2512_13886_amd as L
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    w = torch.zeros(32, 64, dtype=torch.bfloat16)
    h = torch.zeros(4, 32, dtype=torch.bfloat16)
    q = torch.zeros(32, 64, dtype=torch.uint8)
    s = torch.zeros(32, 1, dtype=torch.bfloat16)
    for call in (lambda: L.optima_rms_norm(x, torch.zeros(64), x.clone()),
                 lambda: L.optima_rms_norm(x[0], torch.zeros(64), x.clone()),
                 lambda: L.optima_rms_norm_backward(x, torch.zeros(64), x, x.clone()),
                 lambda: L.optima_gated_forward(x, w, w, h),
                 lambda: L.optima_gated_backward(x, w, w, h, h, h, dX=x.clone()),
                 lambda: L.optima_w4_pack(w, q, s),
                 lambda: L.optima_w4_linear(x, q, s, h),
                 lambda: L.optima_w4_gated(x, q, s, q, s, h)):
        with pytest.raises(ValueError):
            call()


def test_rows_takes_any_pitch_and_refuses_what_is_no_rows():
    from paper_2512_13886_amd import _lib

    class Fake:  # a device tensor's metadata
        is_cuda = True
        dtype = torch.bfloat16

        def __init__(self, shape, strides):
            self.shape, self._s = torch.Size(shape), strides

        def stride(self, i):
            return self._s[i]

        def data_ptr(self):
            return 4096

    b = (torch.bfloat16,)
    assert _lib._rows("t", Fake((3, 5), (9, 1)), (3, 5), b) == (4096, 9, _lib.DTYPE_BF16)
    assert _lib._rows("t", Fake((1, 5), (2, 1)), (1, 5), b)[1] == 5   # the pitch of one row
    assert _lib._rows("t", Fake((0, 5), (5, 1)), (0, 5), b)[0] is None
    assert _lib._rows("t", Fake((3, 1), (7, 4)), (3, 1), b)[1] == 7   # one column, any step
    for shape, strides in (((3, 5), (1, 3)), ((3, 5), (0, 1)), ((3, 5), (4, 1)), ((3, 5), (10, 2))):
        with pytest.raises(ValueError):
            _lib._rows("t", Fake(shape, strides), (3, 5), b)
    with pytest.raises(ValueError):
        _lib._rows("t", Fake((3, 4), (9, 1)), (3, 5), b)
    with pytest.raises(ValueError):
        _lib._rows("t", Fake((3, 5), (9, 1)), (3, 5), (torch.float32,))


@pytest.mark.parametrize("d, ff", [(4032, 83), (300, 9000), (1001, 2731), (4096, 14336), (1, 1)])
def test_more_tokens_need_no_less_workspace(d, ff):
    import paper_2512_13886_amd as L
    for query in (L.optima_gated_forward_workspace_bytes,
                  lambda *a: L.optima_w4_workspace_bytes(*a, 1),
                  lambda *a: L.optima_w4_workspace_bytes(*a, 2)):
        need = [query(n, d, ff) for n in [*range(600), 1000, 4096, 4097, 100000]]
        assert all(a <= b for a, b in zip(need, need[1:]))
