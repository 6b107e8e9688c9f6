"""The gradient of log probabilities where |lse| is large: masks by a common negative constant, and
logits far from 0. There one fp32 lse holds little or nothing of ln sum exp(z - max z), and the
gradient has to come from the row itself."""
import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24  # half a step of fp32, relative
SIZES = (3, 100, 129, 1000, 2048, 2049, 8193, 50001)  # 16, 64 and 256 lanes, one and several parts


@pytest.fixture(scope="module")
def L():
    import paper_2512_13886_amd as L
    return L


def dev():
    return torch.device("cuda:0")


def _exact(x, tokens, g, scale):
    """(the gradient, how far it may be off but for its last rounding) in 64 bits, from y = z - max z, of
    which nothing grows with z. log p = y - ln S has the roundings of the difference, its scale, the
    final difference, and of ln S: S is a sum of at most vocab / 64 terms in order and 64 more joined, each
    with exponents off by 4 |y| and 16 rescalings of 2 |y| + 2 at most; the power has 2 |log p| + 2
    more. H is the forward call's, with such errors of S and of sum p |y| and sum p y^2. Where |lse| is no
    more than 256 log p is z - lse: one rounding of z, and of lse one of scale max z, its sum, and itself."""
    x = x.double()
    y = (x - x.amax(1, keepdim=True)) * scale
    S = torch.exp(y).sum(1, keepdim=True)
    lnS = torch.log(S)
    logs = y - lnS
    p = torch.exp(logs)
    some = p > 0
    ya, la = (torch.where(some, t, torch.zeros_like(t)) for t in (y, logs))
    h = -(p * la).sum(1, keepdim=True)
    a, gh, gl = (t.double().unsqueeze(1) for t in g)
    given = (tokens >= 0).unsqueeze(1)
    a = torch.where(given, a, torch.zeros_like(a))
    want = p * (gl - a - gh * (la + h))
    want.scatter_add_(1, tokens.clamp(min=0).unsqueeze(1), a)
    D, E = ((p * t).sum(1, keepdim=True) for t in (ya.abs(), ya * ya))
    steps = x.shape[1] / 64 + 64 + 48
    s = 6 * D + steps + 4
    b_h = U * (s * (1 + D) + 6 * E + (steps + 6) * D + 4 * (lnS + D))
    e_log = U * (3 * ya.abs() + 2 * la.abs() + s + 4 * lnS)
    m = x.amax(1, keepdim=True) * scale
    near = (m + lnS).abs() <= 257
    e_log = e_log + near * U * (torch.where(some, x * scale, 0.0).abs() + 2 * m.abs() + 2 * (m + lnS).abs())
    e_p = p * (e_log + U * (4 * la.abs() + 4))
    inner = gl.abs() + a.abs() + gh.abs() * (la.abs() + h)
    off = e_p * inner + p * (gh.abs() * (e_log + b_h) + 6 * U * inner) + 2 * U * (p * inner + a.abs())
    return want * scale, off * scale * 1.01


def _backward(L, x, tokens, g, scale, dx=None):
    n = x.shape[0]
    lse, entropy = torch.empty(n, device=dev()), torch.empty(n, device=dev())
    L.optima_token_logprobs(x, None, None, lse=lse, entropy=entropy, scale=scale)
    dx = torch.empty(n, x.shape[1], dtype=x.dtype, device=dev()) if dx is None else dx
    L.optima_token_logprobs_backward(x, lse, dx, tokens=tokens, dlogp=g[0], entropy=entropy,
                                     dentropy=g[1], dlse=g[2], scale=scale)
    return dx


def _rows(vocab, dtype, seed, at):
    """Rows of logits around each of `at`, and between them rows around 0."""
    g = torch.Generator(device=dev()).manual_seed(seed)
    x = 2.5 * torch.randn(2 * len(at), vocab + 3, generator=g, device=dev())
    x[::2] += torch.tensor(at, device=dev()).unsqueeze(1)
    tokens = torch.randint(0, vocab, (2 * len(at),), generator=g, device=dev())
    tokens[::5] = -1
    return x.to(dtype)[:, :vocab], tokens, [torch.randn(2 * len(at), generator=g, device=dev())
                                            for _ in range(3)]


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("vocab", SIZES)
def test_logits_far_from_zero(L, vocab, dtype):
    for scale in (1.0, 0.5):
        x, tokens, g = _rows(vocab, dtype, vocab, (-1e9, -1e6, -1e5, -3000.0, 3000.0, 1e5, 1e6, 1e9))
        want, off = _exact(x, tokens, g, scale)
        off += want.abs() * torch.finfo(dtype).eps / 2 + 2.0 ** -126
        got = _backward(L, x, tokens, g, scale).double()
        assert torch.isfinite(got).all()
        assert ((got - want).abs() <= off).all(), ((got - want).abs() - off).amax(1)
        # The rows between are what they are alone.
        alone = _backward(L, x[1::2].contiguous(), tokens[1::2].contiguous(),
                          [t[1::2].contiguous() for t in g], scale)
        assert torch.equal(alone.double(), got[1::2])
        room = x.clone()
        assert torch.equal(_backward(L, room, tokens, g, scale, room).double(), got)


@pytest.mark.parametrize("vocab", SIZES)
def test_rows_of_one_value(L, vocab):
    """Rows masked by one constant: p = 1 / vocab everywhere, and no gradient of the entropy."""
    at = torch.tensor([-1e29, -1e9, -1e5, -300.0, 300.0, 1e5, 1e9, 1e38], device=dev())
    x = at.unsqueeze(1).repeat(1, vocab)
    n = len(at)
    one, tokens = torch.ones(n, device=dev()), torch.zeros(n, dtype=torch.int64, device=dev())
    steps = U * (vocab / 64 + 64 + 48 + 20 + 8 * torch.log(torch.tensor(float(vocab))).item())
    dx = _backward(L, x, tokens, [0 * one, 0 * one, one], 1.0).double()
    assert (dx.sum(1) - 1).abs().max() <= steps
    assert (dx * vocab - 1).abs().max() <= steps
    dx = _backward(L, x, tokens, [one, 0 * one, 0 * one], 1.0).double()
    want = torch.full_like(dx, -1 / vocab)
    want[:, 0] += 1
    assert (dx - want).abs().max() <= steps
    dx = _backward(L, x, tokens, [0 * one, one, 0 * one], 1.0).double()
    assert (dx * vocab).abs().max() <= 2 * steps


def test_masks_beside_values(L):
    """-1e9 added to half of a row's logits, all of them, or to whole rows of a batch."""
    vocab = 9000
    x, tokens, g = _rows(vocab, torch.float32, 1, (0.0, -1e9))
    x = x.clone()
    x[1, ::2] -= 1e9
    x[3, 1:] -= 1e9
    tokens[:] = torch.tensor([0, 1, 2, 0])
    want, off = _exact(x, tokens, g, 1.25)
    off += want.abs() * U + 2.0 ** -126
    got = _backward(L, x, tokens, g, 1.25).double()
    assert ((got - want).abs() <= off).all()


def test_lse_of_more_than_the_row(L):
    """A row that is a part of a wider one, with the wider one's lse: p = exp(z - lse), also where lse
    is large."""
    x = torch.randn(3, 6000, generator=torch.Generator().manual_seed(1)).to(dev())
    x += torch.tensor([[0.0], [4096.0], [-4096.0]], device=dev())
    lse, one = torch.empty(3, device=dev()), torch.ones(3, device=dev())
    L.optima_token_logprobs(x, None, None, lse=lse)
    for half in (x[:, :2500].contiguous(), x[:, 2500:].contiguous()):
        dx = torch.empty_like(half)
        L.optima_token_logprobs_backward(half, lse, dx, dlse=one)
        want = torch.exp(half.double() - lse.double().unsqueeze(1))
        assert ((dx.double() - want).abs() <= want * U * 200).all()
    # Nothing of the part is left: its share is 0.
    half = torch.full((3, 2500), -float("inf"), device=dev())
    L.optima_token_logprobs_backward(half, lse, half, dlse=one)
    assert (half == 0).all()


def test_far_rows_in_graphs(L):
    for vocab in (900, 30000):
        x, tokens, g = _rows(vocab, torch.bfloat16, 2, (-1e9, 1e4, 0.0))
        x = x.contiguous()
        lse, entropy = torch.empty(6, device=dev()), torch.empty(6, device=dev())
        dx = torch.empty_like(x)

        def step(out):
            L.optima_token_logprobs(x, tokens, None, lse=lse, entropy=entropy)
            L.optima_token_logprobs_backward(x, lse, out, tokens=tokens, dlogp=g[0], entropy=entropy,
                                             dentropy=g[1], dlse=g[2])
        step(dx)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(dx)
        for trial in range(3):
            x.copy_(_rows(vocab, torch.bfloat16, 5 + trial, (0.0, -1e9, 500.0))[0])
            dx.zero_()
            graph.replay()
            torch.cuda.synchronize()
            own = torch.empty_like(dx)
            step(own)
            assert torch.equal(own, dx)
