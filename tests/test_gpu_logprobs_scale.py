"""The least and the largest scales of the log probabilities (one over a temperature): a first choice
taken for certain, and a distribution that is all but uniform."""
import pytest
import torch

pytestmark = pytest.mark.gpu
SCALES = (1e-30, 1e10, 1e38, 2.3e38, 2.5e38, 3.4e38)


@pytest.fixture(scope="module")
def L():
    import paper_2512_13886_amd as L
    return L


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("vocab", (100, 1500, 5000, 50001))
@pytest.mark.parametrize("scale", SCALES)
def test_scale(L, vocab, dtype, scale):
    """The largest logits are 0 and alike, `ties` of them: lse = H = ln ties and log p = -ln ties. A sum of
    ones is exact, its logarithm off by two steps at most, and a step here is below 2^-20."""
    dev = torch.device("cuda:0")
    x = -1 - torch.rand(6, vocab, generator=torch.Generator().manual_seed(vocab)).to(dev)
    for r in range(6):
        x[r, :: vocab // (r + 1)] = 0
    x[5, 1], x[4, 2:40] = -float("inf"), -float("inf")
    x = x.to(dtype)
    ties = (x == 0).sum(1).double() if scale > 1 else (x > -float("inf")).sum(1).double()
    tokens = torch.zeros(6, dtype=torch.int64, device=dev)
    out = [torch.empty(6, device=dev) for _ in range(3)]
    top = torch.empty(6, 1, device=dev)
    index = torch.empty(6, 1, dtype=torch.int64, device=dev)
    for k in (0, 1):
        L.optima_token_logprobs(x, tokens, out[0], lse=out[1], entropy=out[2], scale=scale,
                                **(dict(top_logp=top, top_index=index) if k else {}))
        for got, want in ((out[0], -ties.log()), (out[1], ties.log()), (out[2], ties.log())):
            assert ((got.double() - want).abs() <= 2.0 ** -18).all(), (got, want)
    assert torch.equal(top[:, 0], out[0]) and (index == 0).all()
    # p is 1 over ties at these and 0 elsewhere; times scale.
    dx, one = torch.empty(6, vocab, device=dev, dtype=dtype), torch.ones(6, device=dev)
    L.optima_token_logprobs_backward(x, out[1], dx, dlse=one, scale=scale)
    on = (x == 0) if scale > 1 else (x > -float("inf"))
    want = torch.where(on, scale / ties.unsqueeze(1), 0.0)
    off = want * (2.0 ** -16 + 1.001 * torch.finfo(dtype).eps / 2)
    # The largest bf16 value is (2 - 2^-7) 2^127 = 3.3895e38; from half a step above it, 3.3962e38, the nearest
    # is infinity: that is what 3.4e38 is rounded to.
    over = want >= (2 - 2.0 ** -8) * 2.0 ** 127 if dtype == torch.bfloat16 else want < 0
    assert ((dx.double() - want).abs() <= off)[~over].all() and (dx[over] == float("inf")).all()
