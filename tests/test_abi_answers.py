"""Refusals of the packed products and of the log probabilities: what the C entry points and the
binding return or raise before any launch. No kernel is launched here."""
import ctypes

import pytest
import torch

i64, vp, i32, f32, sz = (ctypes.c_int64, ctypes.c_void_p, ctypes.c_int, ctypes.c_float,
                         ctypes.c_size_t)
F32, BF16, F64, I8, MX4 = 0, 1, 2, 3, 4
OK, INVAL, WORKSPACE, UNSUPPORTED = 0, -1, -4, -5
MB = 1 << 20


@pytest.fixture(scope="module")
def lib():
    import paper_2512_13886_amd as L
    return ctypes.CDLL(L.library_path())


def _sizes(lib):
    for name in ("optima_mx4_row_bytes", "optima_mx4_scale_bytes", "optima_mx4_workspace_bytes",
                 "optima_token_logprobs_workspace_bytes"):
        getattr(lib, name).restype = sz
    return lib


def _pack(lib, **kw):
    """optima_mx4_pack of 10 rows of 300 bf16 values, with changes."""
    a = dict(X=1 * MB, ldx=300, dtype=BF16, n=10, d=300, Q=2 * MB, scales=3 * MB)
    a.update(kw)
    f = lib.optima_mx4_pack
    f.argtypes = [vp, i64, i32, i64, i64, vp, vp, vp]
    return f(*a.values(), None)


@pytest.mark.parametrize("change, status", [
    (dict(X=None), INVAL), (dict(Q=None), INVAL), (dict(scales=None), INVAL), (dict(n=-1), INVAL),
    (dict(d=0), INVAL), (dict(d=(1 << 20) + 1, ldx=(1 << 20) + 1), INVAL), (dict(ldx=299), INVAL),
    (dict(dtype=I8), UNSUPPORTED), (dict(dtype=F64), UNSUPPORTED), (dict(Q=2 * MB + 8), INVAL),
    (dict(scales=3 * MB + 2), INVAL), (dict(X=1 * MB + 1), INVAL), (dict(n=1 << 27), INVAL),
    (dict(n=(1 << 26) - 3, d=257, ldx=257, X=1 << 50, Q=1 << 52, scales=1 << 54), INVAL),
    (dict(Q=1 * MB), INVAL), (dict(scales=1 * MB + 64), INVAL), (dict(scales=2 * MB), INVAL),
    (dict(n=0), OK), (dict(n=0, X=None, Q=None, scales=None), OK),
])
def test_pack_refusals(lib, change, status):
    assert _pack(lib, **change) == status


def _unpack(lib, **kw):
    a = dict(Q=2 * MB, scales=3 * MB, n=10, d=300, Y=1 * MB, ldy=300, dtype=BF16)
    a.update(kw)
    f = lib.optima_mx4_unpack
    f.argtypes = [vp, vp, i64, i64, vp, i64, i32, vp]
    return f(*a.values(), None)


@pytest.mark.parametrize("change, status", [
    (dict(Y=None), INVAL), (dict(Q=None), INVAL), (dict(scales=None), INVAL), (dict(n=-1), INVAL),
    (dict(d=0), INVAL), (dict(ldy=299), INVAL), (dict(dtype=MX4), UNSUPPORTED),
    (dict(Q=2 * MB + 8), INVAL), (dict(Y=2 * MB), INVAL), (dict(Y=3 * MB), INVAL), (dict(n=0), OK),
])
def test_unpack_refusals(lib, change, status):
    assert _unpack(lib, **change) == status


def _linear(lib, **kw):
    """optima_mx4_linear of 20 bf16 tokens, 300 -> 500, with changes."""
    a = dict(X=1 * MB, ldx=300, x_dtype=BF16, xs=None, n=20, d=300, Q=2 * MB, scales=3 * MB,
             d_out=500, Y=4 * MB, ldy=500, y_dtype=F32, ws=8 * MB, nbytes=64 * MB)
    a.update(kw)
    f = lib.optima_mx4_linear
    f.argtypes = [vp, i64, i32, vp, i64, i64, vp, vp, i64, vp, i64, i32, vp, sz, vp]
    return f(*a.values(), None)


PACKED = dict(x_dtype=MX4, xs=7 * MB)


@pytest.mark.parametrize("change, status", [
    (dict(X=None), INVAL), (dict(Q=None), INVAL), (dict(scales=None), INVAL), (dict(Y=None), INVAL),
    (dict(n=-1), INVAL), (dict(n=(1 << 21) + 1), INVAL), (dict(d=0), INVAL), (dict(d_out=0), INVAL),
    (dict(d_out=(1 << 24) + 1, ldy=1 << 25), INVAL),
    (dict(n=1 << 12, d_out=1 << 24, ldy=1 << 24, Y=1 << 50, Q=1 << 52, scales=1 << 54, X=1 << 56), INVAL), (dict(ldx=299), INVAL), (dict(ldy=499), INVAL),
    (dict(x_dtype=F32), UNSUPPORTED), (dict(x_dtype=I8), UNSUPPORTED), (dict(y_dtype=MX4), UNSUPPORTED),
    (dict(xs=7 * MB), INVAL), (dict(x_dtype=MX4), INVAL), (dict(PACKED, X=1 * MB + 8), INVAL),
    (dict(PACKED, xs=7 * MB + 2), INVAL), (dict(Q=2 * MB + 8), INVAL), (dict(scales=3 * MB + 1), INVAL),
    (dict(Y=1 * MB), INVAL), (dict(Y=2 * MB), INVAL), (dict(Y=3 * MB), INVAL),
    (dict(PACKED, Y=7 * MB), INVAL), (dict(Y=4 * MB + 2), INVAL),
    (dict(n=0), OK), (dict(PACKED, n=0, X=None, xs=None, Y=None, ws=None), OK),
])
def test_linear_refusals(lib, change, status):
    assert _linear(lib, **change) == status


def test_linear_workspace(lib):
    f = _sizes(lib).optima_mx4_workspace_bytes
    f.argtypes = [i64, i64, i64]
    assert f(8, 4096, 4096) == 0 and f(9, 4096, 1000) > 0
    for d, out in ((4096, 4096), (14336, 4096), (1001, 2731), (64, 64), (4096, 128000)):
        last = 0
        for n in (1, 8, 9, 16, 17, 33, 64, 65, 100, 129, 255, 256, 257, 400, 777, 1025, 2049, 8192, 1 << 21):
            if -(-n // 64) * -(-out // 64) < 1 << 23:
                assert f(n, d, out) >= last
                last = f(n, d, out)
    need = f(20, 4096, 500)
    big = dict(d=4096, ldx=4096, X=64 * MB, Q=65 * MB, scales=70 * MB, Y=72 * MB)
    assert _linear(lib, **big, nbytes=need - 1) == WORKSPACE
    assert _linear(lib, **big, ws=None) == WORKSPACE and _linear(lib, **big, ws=8 * MB + 8) == WORKSPACE
    for bad in ((-1, 64, 64), (1, 0, 64), (1, 64, 0), (1, 1 << 21, 64)):
        assert f(*bad) == 0


def test_row_sizes(lib):
    L = _sizes(lib)
    L.optima_mx4_row_bytes.argtypes = L.optima_mx4_scale_bytes.argtypes = [i64]
    for d in (1, 255, 256, 257, 512, 513, 4096, 14336, 1 << 20):
        assert L.optima_mx4_row_bytes(d) == -(-d // 256) * 128
        assert L.optima_mx4_scale_bytes(d) == -(-d // 512) * 16
    assert L.optima_mx4_row_bytes(0) == 0 and L.optima_mx4_scale_bytes((1 << 20) + 1) == 0


def _logprobs(lib, **kw):
    """optima_token_logprobs of 10 rows of 20000 bf16 logits, with changes."""
    a = dict(X=1 * MB, ldx=20000, dtype=BF16, n=10, vocab=20000, tokens=2 * MB, scale=1.0,
             logp=3 * MB, lse=4 * MB, entropy=5 * MB, k=4, index=6 * MB, top=7 * MB, ws=8 * MB,
             nbytes=MB)
    a.update(kw)
    f = lib.optima_token_logprobs
    f.argtypes = [vp, i64, i32, i64, i64, vp, f32, vp, vp, vp, i64, vp, vp, vp, sz, vp]
    return f(*a.values(), None)


@pytest.mark.parametrize("change, status", [
    (dict(X=None), INVAL), (dict(tokens=None), INVAL), (dict(n=-1), INVAL), (dict(vocab=0), INVAL),
    (dict(vocab=(1 << 20) + 1, ldx=1 << 21), INVAL), (dict(ldx=19999), INVAL),
    (dict(dtype=I8), UNSUPPORTED), (dict(scale=0.0), INVAL), (dict(scale=-1.0), INVAL),
    (dict(scale=float("nan")), INVAL), (dict(scale=float("inf")), INVAL), (dict(k=-1), INVAL),
    (dict(k=33), UNSUPPORTED), (dict(k=0), INVAL), (dict(k=4, index=None, top=None), INVAL),
    (dict(vocab=3, ldx=3), INVAL),
    (dict(logp=None, lse=None, entropy=None, k=0, index=None, top=None), INVAL),
    (dict(tokens=2 * MB + 4), INVAL), (dict(lse=4 * MB + 2), INVAL), (dict(index=6 * MB + 4), INVAL),
    (dict(lse=3 * MB + 36), INVAL), (dict(entropy=1 * MB + 400), INVAL), (dict(logp=2 * MB), INVAL),
    (dict(top=6 * MB + 300), INVAL), (dict(ws=None), WORKSPACE), (dict(ws=8 * MB + 4), WORKSPACE),
    (dict(nbytes=100), WORKSPACE), (dict(n=0, X=None, tokens=None, logp=None, lse=None,
                                         entropy=None, index=None, top=None), OK),
])
def test_logprobs_refusals(lib, change, status):
    assert _logprobs(lib, **change) == status


def test_logprobs_workspace(lib):
    f = _sizes(lib).optima_token_logprobs_workspace_bytes
    f.argtypes = [i64, i64, i64]
    assert f(1, 8000, 8) == 0 and f(1, 20000, 0) > 0
    for vocab in (100, 2049, 5000, 32768, 50001, 128000, 1 << 20):
        for k in (0, 1, 32):
            last = 0
            for n in (1, 2, 31, 32, 33, 63, 64, 65, 66, 127, 128, 200, 682, 683, 1023, 1024, 2047,
                      2048, 2049, 8192, 65536):
                assert f(n, vocab, k) >= last
                last = f(n, vocab, k)
    for bad in ((-1, 10, 0), (1, 0, 0), (1, 10, 11), (1, 100, 33), (1, 100, -1)):
        assert f(*bad) == 0


def _backward(lib, **kw):
    a = dict(X=1 * MB, ldx=5000, dtype=BF16, n=10, vocab=5000, tokens=2 * MB, scale=1.0,
             lse=3 * MB, entropy=4 * MB, dlogp=5 * MB, dentropy=6 * MB, dlse=7 * MB, dX=8 * MB,
             lddx=5000)
    a.update(kw)
    f = lib.optima_token_logprobs_backward
    f.argtypes = [vp, i64, i32, i64, i64, vp, f32, vp, vp, vp, vp, vp, vp, i64, vp]
    return f(*a.values(), None)


@pytest.mark.parametrize("change, status", [
    (dict(X=None), INVAL), (dict(dX=None), INVAL), (dict(lse=None), INVAL), (dict(tokens=None), INVAL),
    (dict(entropy=None), INVAL), (dict(dlogp=None, dentropy=None, dlse=None), INVAL),
    (dict(n=-1), INVAL), (dict(vocab=0), INVAL), (dict(lddx=4999), INVAL), (dict(scale=0.0), INVAL),
    (dict(dtype=MX4), UNSUPPORTED), (dict(dX=1 * MB + 2), INVAL), (dict(dX=1 * MB, lddx=5008), INVAL),
    (dict(dX=3 * MB), INVAL), (dict(dX=2 * MB), INVAL), (dict(dlse=7 * MB + 1), INVAL),
    (dict(n=0, X=None, dX=None, lse=None, tokens=None), OK),
])
def test_backward_refusals(lib, change, status):
    assert _backward(lib, **change) == status


def test_binding_refusals():
    """What the binding refuses by itself, on tensors of the CPU (the first thing it asks)."""
    import paper_2512_13886_amd as L
    x = torch.zeros(2, 300, dtype=torch.bfloat16)
    q, s = torch.zeros(2, 256, dtype=torch.uint8), torch.zeros(2, 16, dtype=torch.uint8)
    y = torch.zeros(2, 2)
    with pytest.raises(ValueError):
        L.optima_mx4_pack(x, q, s)
    with pytest.raises(ValueError):
        L.optima_mx4_pack(x[0], q, s)
    with pytest.raises(ValueError):
        L.optima_mx4_unpack(q, s, x)
    with pytest.raises(ValueError, match="x_scales"):
        L.optima_mx4_linear(q, q, s, y)
    with pytest.raises(ValueError, match="x_scales"):
        L.optima_mx4_linear(x, q, s, y, x_scales=s)
    t, o = torch.zeros(2, dtype=torch.int64), torch.zeros(2)
    with pytest.raises(ValueError):
        L.optima_token_logprobs(x, t, o)
    with pytest.raises(ValueError):
        L.optima_token_logprobs(x[0], t, o)
    with pytest.raises(ValueError):
        L.optima_token_logprobs_backward(x, o, x, tokens=t, dlogp=o)
