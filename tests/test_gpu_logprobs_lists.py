"""The longest lists of alternatives: many rows of up to 8192 values, a wave each, whose lists fill most
of a CU's LDS; and rows just above, by workgroups."""
import pytest
import torch

from oracle import answers_oracle as O
from test_gpu_logprobs import L, _bounds, _call, _logits, _near, dev  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("n, vocab, k", ((4096, 8192, 32), (4097, 8191, 20), (4099, 2049, 32), (4097, 8193, 32),
                                         (4095, 8192, 32), (5000, 4000, 20)))
def test_long_lists(L, n, vocab, k, dtype):  # noqa: F811
    x, tokens = _logits(n, vocab, dtype, vocab + n, pad=1, shift=1)
    x = x.clone()
    g = torch.Generator(device=dev()).manual_seed(1)
    x[1::8] = torch.randint(0, 3, (len(x[1::8]), vocab), generator=g, device=dev()).to(dtype)  # ties
    x[2::8] = 0
    x[3::8] = -float("inf")
    x[4::8] = -float("inf")
    x[4::8, -5:] = 1
    x[5::8] = torch.arange(vocab, device=dev()).to(dtype) / 64
    x[6::8] = -(torch.arange(vocab, device=dev()) % 512).to(dtype) / 8  # the largest in one lane's values
    lse, logp, entropy, index, top = _call(L, x, tokens, k)
    assert torch.equal(index, O.top(x, k))
    rows = torch.cat([torch.arange(40), torch.arange(n - 40, n)]).to(dev())
    x, tokens = x[rows], tokens[rows]
    want = O.token_logprobs(x, tokens)
    b = [t.nan_to_num(0.0, 0.0, 0.0) for t in _bounds(x, tokens, 1.0)]
    for got, ref, off in zip((lse, logp, entropy), want, b):
        _near(got[rows], ref, off)
    z = x.double().gather(1, index[rows])
    alone = (want[0] == -float("inf")).unsqueeze(1)
    ref = torch.where(alone, -float("inf"), z - want[0].unsqueeze(1))
    _near(top[rows], ref, b[3].unsqueeze(1) + 8 * 2.0 ** -24 * z.abs().nan_to_num(0.0, 0.0, 0.0))


def test_long_lists_repeat(L):  # noqa: F811
    x, tokens = _logits(4096, 8192, torch.bfloat16, 5)
    first = [t.clone() for t in _call(L, x, tokens, 32)]
    for _ in range(3):
        for a, b in zip(first, _call(L, x, tokens, 32)):
            assert torch.equal(a, b)
