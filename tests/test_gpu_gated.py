"""The gated feed-forward product and its gradient against the fp64 oracle.

Tolerances. U = 2^-24, B = 2^-8 (half a bf16 step). A sum of K exact products in fp32 in
any order is off by at most K U of the sum of their magnitudes. The activation adds 8 U
(1 + |g|) relative (the exponential's argument and its two units). In the gradient dG and
dU are rounded to bf16, each by at most B relative; over many of them the roundings are
independent, so that the Frobenius norm of a gradient is off by less than B."""
import numpy as np
import pytest
import torch

from gpu_util import dev, rel_fro
from oracle import feedforward_oracle as F

pytestmark = pytest.mark.gpu

U, B = 2.0 ** -24, 2.0 ** -8
ACT = {"silu": 1, "none": 0}
T = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def L():
    import paper_2512_13886_amd as lib
    return lib


def _np(t):
    return t.double().cpu().numpy()


def _rows(g, n, d, pitch=None, scale=1.0, off=0):
    """bf16 [n, d] of a buffer of rows of `pitch` values, `off` values into it."""
    pitch = pitch or d
    wide = (scale * torch.randn(n * pitch + off, generator=g, device=dev())).bfloat16()
    return wide[off:].view(n, pitch)[:, :d]


def _out(n, d, dt, pitch):
    buf = torch.full((n + 1, pitch), 77, device=dev()).to(dt)
    return buf[:n, :d], buf


def _untouched(buf, n, d):
    return bool((buf[:, d:] == 77).all()) and bool((buf[n:] == 77).all())


def _check_forward(X, Wg, Wu, name, H, G, U_, out):
    x, wg, wu = _np(X), _np(Wg), _np(Wu)
    h, g, u = F.gated(x, wg, wu, name)
    d = x.shape[1]
    eg = d * U * (np.abs(x) @ np.abs(wg).T)
    eu = d * U * (np.abs(x) @ np.abs(wu).T)
    half = {"f32": U, "bf16": B}[out]
    # |act'| <= 1.1, and the products of the two errors
    bound = 1.1 * eg * np.abs(u) + np.abs(F.act(name, g)) * eu + 1.1 * eg * eu + \
        (8 * U * (1 + np.abs(g)) + half * 1.01) * np.abs(h)
    assert np.all(np.abs(_np(H) - h) <= bound * (1 + 2 * half) + 1e-36)
    if G is not None:
        assert np.all(np.abs(_np(G) - g) <= eg * (1 + B) + 1.01 * B * np.abs(g))
        assert np.all(np.abs(_np(U_) - u) <= eu * (1 + B) + 1.01 * B * np.abs(u))


def _forward(L, n, d, ff, name="silu", out="bf16", saved=True, xpitch=None, xoff=0, seed=0):
    g = torch.Generator(device=dev()).manual_seed(seed + n * 7 + d * 3 + ff)
    X = _rows(g, n, d, xpitch, off=xoff)
    Wg, Wu = (_rows(g, ff, d, scale=d ** -0.5 * 2).contiguous() for _ in range(2))
    H, hb = _out(n, ff, T[out], ff + 3)
    G, gb = _out(n, ff, T["bf16"], ff + 1) if saved else (None, None)
    V, ub = _out(n, ff, T["bf16"], ff + 8) if saved else (None, None)
    L.optima_gated_forward(X, Wg, Wu, H, act=ACT[name], G=G, U=V)
    _check_forward(X, Wg, Wu, name, H, G, V, out)
    assert _untouched(hb, n, ff)
    if saved:
        assert _untouched(gb, n, ff) and _untouched(ub, n, ff)


# Few tokens: every number of 16-token blocks and their edges, widths below, at and
# past a 64-value piece and the waves' share, outputs around 16.
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 32, 33, 64])
@pytest.mark.parametrize("d, ff", [(1, 1), (63, 16), (64, 17), (513, 100), (1000, 33)])
def test_few_tokens(L, n, d, ff):
    _forward(L, n, d, ff, xpitch=d + 3, xoff=1)
    _forward(L, n, d, ff, name="none", out="f32", saved=False)


# Tiles: both tile sizes at their edges, one to many stages, widths that are no multiple
# of a stage, unaligned rows of X.
@pytest.mark.parametrize("n, d, ff", [(65, 64, 64), (128, 64, 65), (129, 128, 1), (200, 192, 130),
                                      (300, 1, 100), (257, 65, 129), (500, 100, 333),
                                      (130, 1000, 190)])
def test_small_tiles(L, n, d, ff):
    _forward(L, n, d, ff)
    _forward(L, n, d, ff, name="none", out="f32", xpitch=d + 5, xoff=3)


# Few tiles and long rows: the sum is split, evenly and not, and joined.
@pytest.mark.parametrize("n, d, ff", [(64, 4032, 83), (66, 1025, 1), (130, 2048, 65),
                                      (300, 1000, 33), (1000, 4100, 130)])
@pytest.mark.parametrize("out, saved", [("bf16", True), ("f32", False)])
def test_split_sums(L, n, d, ff, out, saved):
    _forward(L, n, d, ff, out=out, saved=saved)


@pytest.mark.parametrize("n, d, ff", [(2049, 64, 4100), (4096, 128, 2048), (4300, 65, 2300)])
def test_large_tiles(L, n, d, ff):
    _forward(L, n, d, ff, saved=True)
    _forward(L, n, d, ff, out="f32", saved=False)


# Whole rounds of large tiles and small ones for the outputs that are left.
@pytest.mark.parametrize("n, d, ff", [(1500, 1000, 5632), (700, 960, 12529)])
def test_both_tiles(L, n, d, ff):
    _forward(L, n, d, ff, saved=True)
    _forward(L, n, d, ff, out="f32", saved=False)


def test_aligned_pitch_is_read_in_place(L):
    # A row pitch that suits wide loads, and one that does not, give the same bits.
    g = torch.Generator(device=dev()).manual_seed(1)
    X = _rows(g, 300, 128)
    Wg, Wu = _rows(g, 200, 128), _rows(g, 200, 128)
    outs = []
    for pitch in (128, 136, 131):
        P = torch.zeros(300, pitch, dtype=torch.bfloat16, device=dev())[:, :128]
        P.copy_(X)
        H = torch.empty(300, 200, device=dev())
        L.optima_gated_forward(P, Wg, Wu, H)
        outs.append(H)
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


@pytest.mark.parametrize("n", [3, 200])
def test_nonfinite_stays_in_its_rows(L, n):
    g = torch.Generator(device=dev()).manual_seed(2)
    X, Wg, Wu = _rows(g, n, 100), _rows(g, 150, 100), _rows(g, 150, 100)
    ref, H = (torch.empty(n, 150, device=dev()) for _ in range(2))
    L.optima_gated_forward(X, Wg, Wu, ref)
    X[n - 1, 99] = float("nan")
    Wu[149, 0] = float("inf")
    L.optima_gated_forward(X, Wg, Wu, H)
    assert torch.equal(H[:n - 1, :149], ref[:n - 1, :149])
    assert bool(H[n - 1].isnan().all()) and not bool(H[:, 149].isfinite().any())


@pytest.mark.parametrize("n, xpitch", [(2, 257), (20, 257), (40, 259), (64, 258)])
def test_odd_rows_leave_their_neighbours_alone(L, n, xpitch):
    # Rows at odd elements may be read from the element before: it belongs to another row.
    g = torch.Generator(device=dev()).manual_seed(n)
    d, ff = 257, 40
    wide = torch.full((n, xpitch), float("nan"), dtype=torch.bfloat16, device=dev())
    X = wide[:, :d]
    X.copy_(_rows(g, n, d))
    Wg, Wu = _rows(g, ff, d), _rows(g, ff, d)
    ref, H = (torch.empty(n, ff, device=dev()) for _ in range(2))
    L.optima_gated_forward(X, Wg, Wu, ref)
    _check_forward(X, Wg, Wu, "silu", ref, None, None, "f32")
    X[0, d - 1] = float("nan")
    Wg[3, d - 1] = float("inf")
    Wu[8, d - 1] = float("nan")
    L.optima_gated_forward(X, Wg, Wu, H)
    rest = [i for i in range(ff) if i not in (3, 8)]
    assert torch.equal(H[1:, rest], ref[1:, rest])
    assert bool(H[0].isnan().all()) and bool(H[:, 8].isnan().all())
    assert not bool(H[:, 3].isfinite().any())


def _backward(L, n, d, ff, name="silu", dx="bf16", dw="bf16", masked=False, pad=0, seed=0):
    gen = torch.Generator(device=dev()).manual_seed(seed + n * 7 + d * 3 + ff)
    X = _rows(gen, n, d, d + pad, off=pad)
    Wg, Wu = (_rows(gen, ff, d, scale=d ** -0.5).contiguous() for _ in range(2))
    G, V = _rows(gen, n, ff, ff + pad), _rows(gen, n, ff, ff + pad)
    dH = _rows(gen, n, ff, ff + 2 * pad)
    mg = mu = None
    if masked:
        mg, mu = ((torch.rand(ff, d, generator=gen, device=dev()) < 0.5).to(torch.uint8)
                  for _ in range(2))
    dX, buf = _out(n, d, T[dx], d + 3)
    dWg, dWu = (torch.full((ff, d), float("nan"), dtype=T[dw], device=dev()) for _ in range(2))
    L.optima_gated_backward(X, Wg, Wu, G, V, dH, dX=dX, dWg=dWg, dWu=dWu, act=ACT[name], mask_g=mg,
                            mask_u=mu)
    x, wg, wu, g, u, dh = (_np(t) for t in (X, Wg, Wu, G, V, dH))
    rx, rg, ru, dg, du = F.gated_backward(x, wg, wu, g, u, dh, name)
    # dG and dU: the rounding, and fp32 in what is rounded
    step = 1.01 * B
    size = np.abs(dg) @ np.abs(wg) + np.abs(du) @ np.abs(wu)
    # act' may cancel: 16 U of its two parts
    slope = np.abs(dh * u) * 16 * U * (1 + np.abs(g))
    extra = slope @ np.abs(wg)
    half = {"f32": U, "bf16": step}
    assert np.all(np.abs(_np(dX) - rx) <=
                  (step + (2 * ff + 64) * U) * size + 2 * extra + half[dx] * np.abs(rx) + 1e-36)
    assert rel_fro(_np(dX), rx) <= B
    assert _untouched(buf, n, d)
    for got, ref, p, m, ex in ((dWg, rg, dg, mg, slope), (dWu, ru, du, mu, 0 * slope)):
        size = np.abs(p).T @ np.abs(x)
        if m is not None:
            off = _np(m) == 0
            assert not np.any(got.float().cpu().numpy().view(np.uint32)[off])  # +0 exactly
            ref, size = ref * ~off, size * ~off
        assert np.all(np.abs(_np(got) - ref) <= (step + (n + 64) * U) * size +
                      2 * ex.T @ np.abs(x) + half[dw] * np.abs(ref) + 1e-36)
        if np.any(ref):
            assert rel_fro(_np(got), ref) <= B


@pytest.mark.parametrize("n, d, ff", [(1, 1, 1), (1, 64, 64), (5, 100, 33), (64, 65, 130),
                                      (65, 64, 63), (300, 200, 129), (257, 300, 64)])
@pytest.mark.parametrize("masked", [False, True])
def test_backward(L, n, d, ff, masked):
    _backward(L, n, d, ff, masked=masked, pad=3)
    _backward(L, n, d, ff, name="none", dx="f32", dw="f32", masked=masked)


@pytest.mark.parametrize("n", [3, 200, 2000])
def test_backward_nonfinite_under_masks(L, n):
    # NaN and infinity where the masks are 0 leave no trace in the weights' gradients.
    gen = torch.Generator(device=dev()).manual_seed(n)
    X, Wg, Wu = (_rows(gen, r, 100) for r in (n, 150, 150))
    G, V, dH = (_rows(gen, n, 150) for _ in range(3))
    masks = [(torch.rand(150, 100, generator=gen, device=dev()) < 0.5).to(torch.uint8)
             for _ in range(2)]
    for m in masks:
        m[10] = 0  # a row with nothing left
        m[:, 5] = 0
    outs = []
    for bad in (False, True):
        x, dh = X.clone(), dH.clone()
        if bad:
            x[n - 1, 5] = float("inf")
            dh[0, 10] = float("nan")
        dX = torch.empty(n, 100, device=dev())
        dWg, dWu = (torch.full((150, 100), float("nan"), device=dev()) for _ in range(2))
        L.optima_gated_backward(x, Wg, Wu, G, V, dh, dX=dX, dWg=dWg, dWu=dWu, mask_g=masks[0],
                                mask_u=masks[1])
        outs.append((dX, dWg, dWu))
    for ref, got in zip(outs[0][1:], outs[1][1:]):
        assert torch.equal(ref, got) and not bool(got[10].any()) and not bool(got[:, 5].any())
    assert bool(outs[1][0][0].isnan().all()) and torch.equal(outs[0][0][1:], outs[1][0][1:])


# Products that take the large tile, one of the two or both, and long sums over few
# outputs.
@pytest.mark.parametrize("n, d, ff", [(2300, 2100, 300), (4096, 64, 2048), (600, 128, 5000)])
def test_backward_large(L, n, d, ff):
    _backward(L, n, d, ff, masked=True)


def test_backward_parts_and_accumulation(L):
    gen = torch.Generator(device=dev()).manual_seed(5)
    n, d, ff = 190, 100, 70
    X, Wg, Wu = _rows(gen, n, d), _rows(gen, ff, d), _rows(gen, ff, d)
    G, V, dH = (_rows(gen, n, ff) for _ in range(3))
    mask = (torch.rand(ff, d, generator=gen, device=dev()) < 0.5).to(torch.uint8)
    for dt in (torch.float32, torch.bfloat16):
        dX, dWg, dWu = (torch.empty(s, dtype=dt, device=dev()) for s in ((n, d), (ff, d), (ff, d)))
        L.optima_gated_backward(X, Wg, Wu, G, V, dH, dX=dX, dWg=dWg, dWu=dWu, mask_g=mask)
        only = torch.empty_like(dX)
        L.optima_gated_backward(X, Wg, Wu, G, V, dH, dX=only)
        assert torch.equal(only, dX)
        a, b = torch.empty_like(dWg), torch.empty_like(dWu)
        L.optima_gated_backward(X, Wg, Wu, G, V, dH, dWg=a, dWu=b, mask_g=mask)
        assert torch.equal(a, dWg) and torch.equal(b, dWu)
        a.fill_(1.0)
        b.fill_(-2.0)
        L.optima_gated_backward(X, Wg, Wu, G, V, dH, dWg=a, dWu=b, mask_g=mask, accumulate=True)
        if dt == torch.float32:  # one fp32 addition
            assert torch.equal(a, 1.0 + dWg) and torch.equal(b, -2.0 + dWu)
        assert bool((a[mask == 0] == 1).all())


def test_backward_against_differences(L):
    # The library's forward pass with fp32 outputs. Differences of 2^-5 in weights that
    # are whole multiples of 2^-8 keep every operand exact in bf16; H is quadratic in
    # Wu o Wg for the identity activation, so that central differences of one entry are
    # exact up to the sums' fp32 errors.
    gen = torch.Generator(device=dev()).manual_seed(6)
    n, d, ff, h = 4, 6, 5, 2.0 ** -5

    def grid(*shape):
        return (torch.randint(-32, 33, shape, generator=gen, device=dev()).float() / 32).bfloat16()

    X, Wg, Wu, dH = grid(n, d), grid(ff, d), grid(ff, d), grid(n, ff)
    H = torch.empty(n, ff, device=dev())

    def loss(x, wg, wu):
        L.optima_gated_forward(x, wg, wu, H, act=0)
        return (H.double() * dH.double()).sum().item()

    G, V = (X.float() @ Wg.float().t()).bfloat16(), (X.float() @ Wu.float().t()).bfloat16()
    dX = torch.empty(n, d, device=dev())
    dWg, dWu = torch.empty(ff, d, device=dev()), torch.empty(ff, d, device=dev())
    L.optima_gated_backward(X, Wg, Wu, G, V, dH, dX=dX, dWg=dWg, dWu=dWu, act=0)
    # G, U, dG and dU are rounded to bf16: 2 B of the sums of magnitudes, which are below
    # 6 * 5 * 6 here.
    for k, (t, grad) in enumerate(((X, dX), (Wg, dWg), (Wu, dWu))):
        scale = grad.abs().max().item() + 1
        for i in np.ndindex(*t.shape):
            v = []
            for sign in (1, -1):
                ops = [X, Wg, Wu]
                ops[k] = t.clone()
                ops[k][i] += sign * h
                v.append(loss(*ops))
            assert abs((v[0] - v[1]) / (2 * h) - grad[i].item()) <= 2 * 1.01 * B * 6 * scale


@pytest.mark.parametrize("n", [3, 200])
def test_side_stream_graph_and_repeats(L, n):
    gen = torch.Generator(device=dev()).manual_seed(7)
    d, ff = 200, 300
    X, Wg, Wu, dH = _rows(gen, n, d), _rows(gen, ff, d), _rows(gen, ff, d), _rows(gen, n, ff)
    H, G, V = (torch.empty(n, ff, dtype=torch.bfloat16, device=dev()) for _ in range(3))
    dX = torch.empty(n, d, dtype=torch.bfloat16, device=dev())
    dWg, dWu = torch.empty(ff, d, device=dev()), torch.empty(ff, d, device=dev())
    ws = torch.empty(max(L.optima_gated_forward_workspace_bytes(n, d, ff),
                         L.optima_gated_backward_workspace_bytes(n, d, ff)), dtype=torch.uint8,
                     device=dev())

    def step(stream=None):
        L.optima_gated_forward(X, Wg, Wu, H, G=G, U=V, ws=ws, stream=stream)
        L.optima_gated_backward(X, Wg, Wu, G, V, dH, dX=dX, dWg=dWg, dWu=dWu, ws=ws, stream=stream)

    def outs():
        torch.cuda.synchronize()
        return [t.clone() for t in (H, G, V, dX, dWg, dWu)]

    step()
    ref = outs()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    assert all(torch.equal(a, b) for a, b in zip(ref, outs()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(3):
        X.copy_(_rows(gen, n, d))
        graph.replay()
        got = outs()
        step()
        assert all(torch.equal(a, b) for a, b in zip(got, outs())), k


def test_offsets_past_32_bits(L):
    # n d_ff past 2^31 values; the tokens are independent, so that a few of them alone
    # give the same h and dX up to the order of the sums (and dG, dU rounded alike).
    n, d, ff = 40001, 64, 60000
    g = torch.Generator(device=dev()).manual_seed(5)

    def rows(*shape, scale=1.0):
        return torch.randn(shape, generator=g, device=dev(), dtype=torch.bfloat16).mul_(scale)

    X, Wg, Wu = rows(n, d), rows(ff, d, scale=d ** -0.5), rows(ff, d, scale=d ** -0.5)
    H, G, V, dH = (torch.empty((n, ff), dtype=torch.bfloat16, device=dev()) for _ in range(4))
    L.optima_gated_forward(X, Wg, Wu, H, G=G, U=V)
    dH.normal_(generator=g)
    dX = torch.empty((n, d), dtype=torch.float32, device=dev())
    dWg, dWu = (torch.empty((ff, d), dtype=torch.float32, device=dev()) for _ in range(2))
    L.optima_gated_backward(X, Wg, Wu, G, V, dH, dX, dWg, dWu)
    at = torch.tensor([0, 1, 20000, 35791, 35792, 39999, 40000], device=dev())
    few = torch.empty((len(at), ff), dtype=torch.bfloat16, device=dev())
    L.optima_gated_forward(X[at], Wg, Wu, few)
    assert rel_fro(_np(H[at]), _np(few)) <= B
    few_dx = torch.empty((len(at), d), dtype=torch.float32, device=dev())
    L.optima_gated_backward(X[at], Wg, Wu, G[at], V[at], dH[at], dX=few_dx)
    # Sums of 2 ff products in another order, in fp32.
    _, _, _, dg, du = F.gated_backward(_np(X[at]), _np(Wg), _np(Wu), _np(G[at]), _np(V[at]),
                                       _np(dH[at]), "silu")
    bound = 2 * 2 * ff * U * (np.abs(dg) @ np.abs(_np(Wg)) + np.abs(du) @ np.abs(_np(Wu)))
    assert np.all(np.abs(_np(dX[at]) - _np(few_dx)) <= 1.01 * bound)
    # dW of the first and last outputs, against the oracle's on the same G and U.
    cols = slice(ff - 8, ff)
    _, wg, wu, _, _ = F.gated_backward(_np(X), _np(Wg[cols]), _np(Wu[cols]), _np(G[:, cols]),
                                       _np(V[:, cols]), _np(dH[:, cols]), "silu")
    assert rel_fro(_np(dWg[cols]), wg) <= B and rel_fro(_np(dWu[cols]), wu) <= B


def test_no_tokens(L):
    e = torch.empty(0, 64, dtype=torch.bfloat16, device=dev())
    f = torch.empty(0, 32, dtype=torch.bfloat16, device=dev())
    W = torch.ones(32, 64, device=dev()).bfloat16()
    L.optima_gated_forward(e, W, W, f)
    a, b = (torch.full((32, 64), 5.0, device=dev()) for _ in range(2))
    L.optima_gated_backward(e, W, W, f, f, f, dX=torch.empty_like(e), dWg=a, dWu=b, accumulate=True)
    assert bool((a == 5).all()) and bool((b == 5).all())
    L.optima_gated_backward(e, W, W, f, f, f, dWg=a, dWu=b)
    assert bool((a == 0).all()) and bool((b == 0).all())
