"""Microscaled 4-bit packing and its products against the oracle."""
import pytest
import torch

from oracle import answers_oracle as O
from test_mx4_plans_host import SLABS, TILES

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def L():
    import paper_2512_13886_amd as L
    return L


def dev():
    return torch.device("cuda:0")


def _room(L, n, d, fill=0xAA):
    return (torch.full((n, L.optima_mx4_row_bytes(d)), fill, dtype=torch.uint8, device=dev()),
            torch.full((n, L.optima_mx4_scale_bytes(d)), fill, dtype=torch.uint8, device=dev()))


def _pack(L, x):
    Q, s = _room(L, *x.shape)
    L.optima_mx4_pack(x, Q, s)
    return Q, s


def _rows(n, d, dtype, seed, pad=0, shift=0):
    """Rows with blocks of very different size, out of a wider buffer, on the device."""
    g = torch.Generator().manual_seed(seed)
    wide = torch.randn(n, d + pad, generator=g)
    wide *= torch.exp2(torch.randint(-12, 12, (n, -(-(d + pad) // 32)), generator=g).float()
                       ).repeat_interleave(32, 1)[:, :d + pad]
    flat = torch.zeros(n * (d + pad) + shift, dtype=dtype)
    flat[shift:] = wide.reshape(-1).to(dtype)
    return flat.to(dev())[shift:].view(n, d + pad)[:, :d]


DIMS = (1, 7, 8, 31, 32, 33, 100, 255, 256, 257, 512, 513, 1001, 4096)


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("d", DIMS)
def test_pack_is_exact(L, d, dtype):
    for n, pad, shift in ((1, 0, 0), (3, 5, 1), (17, 0, 3)):
        x = _rows(n, d, dtype, d + n, pad, shift)
        values, code, scale = O.mx4_values(x.cpu())
        Q, s = _pack(L, x)
        wq, ws = O.mx4_layout(code, scale)
        # A rounded zero keeps its sign in the code; the padding is written too.
        assert torch.equal(Q.cpu(), wq) and torch.equal(s.cpu(), ws)
        for out in (torch.float32, torch.bfloat16):
            wide = torch.full((n, d + 3), 7.0, dtype=out, device=dev())
            L.optima_mx4_unpack(Q, s, wide[:, :d])
            assert torch.equal(wide[:, :d].double().cpu(), values)
            assert (wide[:, d:] == 7.0).all()


def test_pack_borders_and_special_values(L):
    grid = torch.arange(-64, 65, dtype=torch.float32) / 8  # all borders between codes
    rows = [torch.nn.functional.pad(grid * 2.0 ** e, (0, 160 - 129)) for e in (-126, -20, 0, 60, 124)]
    rows.append(torch.zeros(160))
    rows.append(torch.full((160,), 2.0 ** -149))
    rows.append(torch.linspace(0, 1, 160) * 2.0 ** -126)  # subnormal and first normal numbers
    rows.append(torch.full((160,), torch.finfo(torch.float32).max))
    odd = torch.linspace(-3, 3, 160)
    for k, v in ((40, float("nan")), (75, float("inf")), (159, -float("inf"))):
        odd[k] = v
    rows.append(odd)
    x = torch.stack(rows)
    values, code, scale = O.mx4_values(x)
    Q, s = _pack(L, x.to(dev()))
    wq, ws = O.mx4_layout(code, scale)
    assert torch.equal(Q.cpu(), wq) and torch.equal(s.cpu(), ws)
    Y = torch.empty(len(rows), 160, device=dev())
    L.optima_mx4_unpack(Q, s, Y)
    assert torch.equal(torch.isnan(Y.cpu()), torch.isnan(values))
    assert torch.equal(Y.cpu().double().nan_to_num(9.0), values.nan_to_num(9.0))


def test_unpack_of_every_code_and_scale(L):
    Q = torch.arange(256, device=dev()).to(torch.uint8).view(1, 256)[:, :128].repeat(256, 1)
    Q = torch.cat([Q[:128], Q[:128] + 128]).contiguous()
    s = torch.arange(256, device=dev()).to(torch.uint8).view(256, 1).repeat(1, 16).contiguous()
    Y = torch.empty(256, 256, device=dev())
    L.optima_mx4_unpack(Q, s, Y)
    c = torch.stack([Q & 15, Q >> 4], 2).view(256, 256).cpu().long()
    size = torch.tensor(O.LEVELS + tuple(-v for v in O.LEVELS), dtype=torch.float64)[c]
    want = size * torch.ldexp(torch.ones(256, 1, dtype=torch.float64), torch.arange(256).view(256, 1) - 127)
    want[255] = float("nan")
    want = want.float()  # exact, or past the range: infinity
    assert torch.equal(torch.isnan(Y.cpu()), torch.isnan(want))
    assert torch.equal(Y.cpu().nan_to_num(9.0), want.nan_to_num(9.0))


def _weights(L, n, d, seed):
    g = torch.Generator(device=dev()).manual_seed(seed)
    w = 0.02 * torch.randn(n, d, generator=g, device=dev())
    w *= torch.rand(n, d, generator=g, device=dev()) < 0.5
    Q, s = _pack(L, w)
    return Q, s, O.mx4_values(w)[0]


def _tokens(n, d, seed, pad=0):
    g = torch.Generator(device=dev()).manual_seed(seed)
    x = torch.randn(n, d + pad, generator=g, device=dev())
    x[:, : 3] *= 20
    return x.bfloat16()[:, :d]


def _bound(x, w, y, dtype):
    """Every product is exact and joins the fp32 sum with one rounding at most, of a value that is
    no larger than the sum of the absolute values; one more to the output's type."""
    d = x.shape[1]
    size = torch.mm(x.abs(), w.abs().t().contiguous())
    return size * (d * 2.0 ** -24) * (1 + 2.0 ** -8) + y.abs() * torch.finfo(dtype).eps / 2


def _check(L, X, Q, s, w, out, packed, pad=0):
    n, d = X.shape
    ff = Q.shape[0]
    x = X.double()
    args = dict(X=X)
    if packed:
        xq, xs = _pack(L, X)
        x = O.mx4_values(X)[0]
        args = dict(X=xq, x_scales=xs)
    wide = torch.full((n + 1, ff + pad), 5.0, dtype=out, device=dev())
    L.optima_mx4_linear(Q=Q, scales=s, Y=wide[:n, :ff], **args)
    want = torch.mm(x, w.t().contiguous())
    off = (wide[:n, :ff].double() - want).abs()
    assert (off <= _bound(x, w, want, out)).all(), float((off - _bound(x, w, want, out)).max())
    assert (wide[n] == 5.0).all() and (wide[:, ff:] == 5.0).all()
    return wide[:n, :ff]


@pytest.mark.parametrize("packed", (False, True))
@pytest.mark.parametrize("d, ff", ((1, 1), (33, 15), (100, 16), (257, 17), (512, 100), (1001, 273),
                                   (4097, 64)))
def test_linear(L, d, ff, packed):
    Q, s, w = _weights(L, ff, d, d + ff)
    for n in (1, 2, 4, 5, 13, 16, 17, 31, 33, 64, 65, 130):
        X = _tokens(n, d, n, pad=n % 3)
        _check(L, X, Q, s, w, torch.float32, packed, pad=n % 4)
        _check(L, X, Q, s, w, torch.bfloat16, packed, pad=(n + 1) % 4)


@pytest.mark.parametrize("packed", (False, True))
@pytest.mark.parametrize("n, d, ff", ((1, 14336, 4096), (16, 4096, 14336), (10, 4096, 14336),
                                      (6, 1500, 9000), (12, 4096, 8200), (9, 14336, 9001), (64, 4096, 1000),
                                      (100, 14336, 768), (300, 1000, 2731), (777, 4097, 5001)))
def test_linear_of_full_sizes(L, n, d, ff, packed):
    Q, s, w = _weights(L, ff, d, 3)
    _check(L, _tokens(n, d, 4), Q, s, w, torch.bfloat16, packed)
    _check(L, _tokens(n, d, 5), Q, s, w, torch.float32, packed)


@pytest.mark.parametrize("n, d, ff", ((256, 768, 256), (1000, 4096, 300), (513, 257, 1001),
                                      (2049, 1000, 512), (4096, 512, 4096)))
def test_linear_of_many_packed_tokens(L, n, d, ff):
    Q, s, w = _weights(L, ff, d, 3)
    _check(L, _tokens(n, d, 4), Q, s, w, torch.bfloat16, True, pad=3)
    _check(L, _tokens(n, d, 5), Q, s, w, torch.float32, True)


@pytest.mark.parametrize("n, d, ff", sorted(TILES))
def test_every_tile(L, n, d, ff):
    Q, s, w = _weights(L, ff, d, 5)
    _check(L, _tokens(n, d, 6), Q, s, w, torch.float32, True, pad=1)
    _check(L, _tokens(n, d, 7), Q, s, w, torch.bfloat16, True)


@pytest.mark.parametrize("n, d, ff", sorted(SLABS))
def test_every_slab(L, n, d, ff):
    Q, s, w = _weights(L, ff, d, 5)
    _check(L, _tokens(n, d, 6), Q, s, w, torch.float32, False, pad=1)
    _check(L, _tokens(n, d, 7), Q, s, w, torch.bfloat16, False)


@pytest.mark.parametrize("packed", (False, True))
@pytest.mark.parametrize("n", (1, 9, 20, 50, 200, 600))
def test_whole_numbers_are_exact(L, n, packed):
    """Whole numbers whose sums stay below 2^24: every order of the sum gives the same."""
    g = torch.Generator(device=dev()).manual_seed(n)
    levels = torch.tensor([0.0, 1, 2, 3, 4, 6, -1, -2, -3, -4, -6], device=dev())
    # A 6 in every block: scale 1.
    X = levels[torch.randint(0, 11, (n, 2000), generator=g, device=dev())].bfloat16()
    w = levels[torch.randint(0, 11, (300, 2000), generator=g, device=dev())]
    X[:, ::32], w[:, ::32] = 6, 6
    Q, s = _pack(L, w)
    Y = torch.empty(n, 300, device=dev())
    args = dict(zip(("X", "x_scales"), _pack(L, X))) if packed else dict(X=X)
    L.optima_mx4_linear(Q=Q, scales=s, Y=Y, **args)
    assert torch.equal(Y.double(), torch.mm(X.double(), w.double().t().contiguous()))


@pytest.mark.parametrize("packed", (False, True))
@pytest.mark.parametrize("n", (5, 40, 300))
def test_special_tokens_stay_in_their_rows(L, n, packed):
    Q, s, w = _weights(L, 200, 600, 1)
    X = _tokens(n, 600, 2).clone()
    clean = _check(L, X, Q, s, w, torch.float32, packed).clone()
    X[1, 599], X[3, 0] = float("nan"), float("inf")
    args = dict(X=X)
    if packed:
        xq, xs = _pack(L, X)
        args = dict(X=xq, x_scales=xs)
    Y = torch.empty(n, 200, device=dev())
    L.optima_mx4_linear(Q=Q, scales=s, Y=Y, **args)
    assert torch.isnan(Y[1]).all()
    assert not torch.isfinite(Y[3]).any()
    keep = [r for r in range(n) if r not in (1, 3)]
    assert torch.equal(Y[keep], clean[keep])


@pytest.mark.parametrize("n", (2, 40, 300))
def test_special_weights_stay_in_their_columns(L, n):
    w = 0.02 * torch.randn(100, 600, generator=torch.Generator().manual_seed(1)).to(dev())
    Q, s = _pack(L, w)
    X = _tokens(n, 600, 2)
    clean = _check(L, X, Q, s, O.mx4_values(w)[0], torch.float32, False).clone()
    w[7, 100] = float("inf")
    Q, s = _pack(L, w)
    xq, xs = _pack(L, X)
    Y = torch.empty(n, 100, device=dev())
    L.optima_mx4_linear(X, Q, s, Y)
    keep = [c for c in range(100) if c != 7]
    assert torch.isnan(Y[:, 7]).all() and torch.equal(Y[:, keep], clean[:, keep])
    L.optima_mx4_linear(xq, Q, s, Y, x_scales=xs)
    assert torch.isnan(Y[:, 7]).all() and torch.isfinite(Y[:, keep]).all()


def test_pruned_weights_add_nothing(L):
    """Zero rows of W give exact zeros, for every form."""
    w = torch.zeros(50, 700, device=dev())
    Q, s = _pack(L, w)
    for n in (1, 30, 300):
        X = _tokens(n, 700, n)
        for args in (dict(X=X), dict(zip(("X", "x_scales"), _pack(L, X)))):
            Y = torch.full((n, 50), 3.0, device=dev())
            L.optima_mx4_linear(Q=Q, scales=s, Y=Y, **args)
            assert (Y == 0).all()


@pytest.mark.parametrize("packed", (False, True))
@pytest.mark.parametrize("n", (1, 20, 100, 600))
def test_graph_and_streams(L, n, packed):
    """Two graphs of their own workspaces, replayed between eager calls on a third stream."""
    d, ff = 1500, 700
    Q, s, w = _weights(L, ff, d, 1)
    sets = []
    for k in range(2):
        X, Y = _tokens(n, d, 10 + k).clone(), torch.empty(n, ff, device=dev())
        room = _room(L, n, d)
        ws = torch.empty(max(16, L.optima_mx4_workspace_bytes(n, d, ff)), dtype=torch.uint8, device=dev())
        sets.append((X, Y, room, ws))

    def step(X, Y, room, ws, stream=None):
        if packed:
            L.optima_mx4_pack(X, *room, stream=stream)
            L.optima_mx4_linear(room[0], Q, s, Y, x_scales=room[1], ws=ws, stream=stream)
        else:
            L.optima_mx4_linear(X, Q, s, Y, ws=ws, stream=stream)

    graphs = []
    for one in sets:
        step(*one)
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            step(*one)
        graphs.append(graph)
    side = torch.cuda.Stream()
    for trial in range(3):
        wants = []
        for k, (X, Y, room, ws) in enumerate(sets):
            X.copy_(_tokens(n, d, 20 + 2 * trial + k))
            own = torch.empty_like(Y)
            step(X, own, _room(L, n, d), torch.empty_like(ws))
            Y.zero_()
            wants.append(own)
        torch.cuda.synchronize()
        for graph in graphs:
            graph.replay()
        eager = torch.empty_like(sets[0][1])
        side.wait_stream(torch.cuda.current_stream())
        other = (sets[0][0], eager, _room(L, n, d), torch.empty_like(sets[0][3]))
        torch.cuda.synchronize()
        step(*other, stream=side)
        torch.cuda.synchronize()
        for (X, Y, room, ws), want in zip(sets, wants):
            assert torch.equal(Y, want)
        assert torch.equal(eager, wants[0])


def test_no_tokens(L):
    Q, s, _ = _weights(L, 20, 100, 1)
    X = torch.empty(0, 100, dtype=torch.bfloat16, device=dev())
    L.optima_mx4_linear(X, Q, s, torch.empty(0, 20, device=dev()))
    room = _room(L, 0, 100)
    L.optima_mx4_pack(X, *room)
    L.optima_mx4_linear(room[0], Q, s, torch.empty(0, 20, device=dev()), x_scales=room[1])
    L.optima_mx4_unpack(*room, torch.empty(0, 100, device=dev()))


def test_offsets_past_32_bits(L):
    """Codes of 4.3 GB and outputs of 4.3 GB: the last rows against products of those alone."""
    d, ff = 8192, (1 << 20) + 100
    Q = torch.randint(0, 256, (ff, L.optima_mx4_row_bytes(d)), dtype=torch.uint8, device=dev())
    s = torch.randint(118, 124, (ff, L.optima_mx4_scale_bytes(d)), dtype=torch.uint8, device=dev())
    assert Q.numel() > 1 << 32
    for n in (2, 40):
        X = _tokens(n, d, n)
        for args in (dict(X=X), dict(zip(("X", "x_scales"), _pack(L, X)))):
            Y, last = torch.empty(n, ff, device=dev()), torch.empty(n, 100, device=dev())
            L.optima_mx4_linear(Q=Q, scales=s, Y=Y, **args)
            L.optima_mx4_linear(Q=Q[-100:].clone(), scales=s[-100:].clone(), Y=last, **args)
            x = X.double() if "x_scales" not in args else O.mx4_values(X)[0]
            wide = torch.empty(100, d, device=dev())
            L.optima_mx4_unpack(Q[-100:].clone(), s[-100:].clone(), wide)
            want = torch.mm(x, wide.double().t().contiguous())
            bound = _bound(x, wide.double(), want, torch.float32)
            assert ((Y[:, -100:].double() - want).abs() <= bound).all()
            assert ((last.double() - want).abs() <= bound).all()
    wide = torch.empty(ff, d, dtype=torch.bfloat16, device=dev())
    L.optima_mx4_unpack(Q, s, wide)
    tail = torch.empty(100, d, dtype=torch.bfloat16, device=dev())
    L.optima_mx4_unpack(Q[-100:].clone(), s[-100:].clone(), tail)
    assert torch.equal(wide[-100:], tail)
    Q2, s2 = _room(L, ff, d)
    L.optima_mx4_pack(wide, Q2, s2)
    back = torch.empty(100, d, dtype=torch.bfloat16, device=dev())
    L.optima_mx4_unpack(Q2[-100:].clone(), s2[-100:].clone(), back)
    assert torch.equal(back, O.mx4_values(tail)[0].bfloat16())


@pytest.mark.parametrize("n", (1, 13, 40, 200, 1000))
def test_results_repeat(L, n):
    Q, s, _ = _weights(L, 1000, 3000, 1)
    X = _tokens(n, 3000, 2)
    room = _pack(L, X)
    first = [torch.empty(n, 1000, device=dev()) for _ in range(2)]
    L.optima_mx4_linear(X, Q, s, first[0])
    L.optima_mx4_linear(room[0], Q, s, first[1], x_scales=room[1])
    for _ in range(3):
        Y = torch.empty(n, 1000, device=dev())
        L.optima_mx4_linear(X, Q, s, Y)
        assert torch.equal(Y, first[0])
        L.optima_mx4_linear(room[0], Q, s, Y, x_scales=room[1])
        assert torch.equal(Y, first[1])


def test_refusals(L):
    Q, s = _room(L, 20, 600)
    X = _tokens(4, 600, 1)
    Y = torch.empty(4, 20, device=dev())
    for bad in (dict(X=X[:, ::2]), dict(X=X.float()), dict(Q=Q[:, :256]), dict(scales=s[:10]),
                dict(Y=Y[:3]), dict(Y=Y.half()), dict(Y=Y.t()), dict(x_scales=s[:4]),
                dict(X=Q[:4]), dict(X=X[:, :500])):
        with pytest.raises(ValueError):
            L.optima_mx4_linear(**dict(dict(X=X, Q=Q, scales=s, Y=Y), **bad))
    with pytest.raises(ValueError):
        L.optima_mx4_pack(X, Q, s)
    with pytest.raises(L.OptimaError):  # Y over X
        L.optima_mx4_linear(X, Q, s, X[:, :20])
    X = _tokens(40, 3000, 1)
    Q, s = _room(L, 20, 3000)
    with pytest.raises(L.OptimaError):
        L.optima_mx4_linear(X, Q, s, torch.empty(40, 20, device=dev()),
                            ws=torch.empty(16, dtype=torch.uint8, device=dev()))
