"""Packed products whose scales have no more alignment than is asked for: 4 bytes."""
import pytest
import torch

from oracle import answers_oracle as O
from test_gpu_mx4 import L, _bound, _pack, _tokens, _weights, dev  # noqa: F401

pytestmark = pytest.mark.gpu


def _moved(s, by):
    """A copy that begins `by` bytes after a multiple of 16."""
    room = torch.zeros(s.numel() + 32, dtype=torch.uint8, device=dev())
    at = -room.data_ptr() % 16 + by
    out = room[at:at + s.numel()].view(s.shape)
    out.copy_(s)
    assert out.data_ptr() % 16 == by and out.is_contiguous()
    return out


@pytest.mark.parametrize("n, d, ff", ((1, 600, 300), (16, 1000, 9000), (17, 512, 100), (64, 4096, 1000),
                                      (130, 1001, 700), (777, 513, 257), (2049, 600, 129)))
def test_scales_at_any_dword(L, n, d, ff):  # noqa: F811
    Q, s, w = _weights(L, ff, d, 3)
    X = _tokens(n, d, 4)
    xq, xs = _pack(L, X)
    x = O.mx4_values(X)[0]
    want = torch.mm(x, w.t().contiguous())
    for bx, bw in ((4, 0), (0, 8), (12, 4)):
        for out in (torch.float32, torch.bfloat16):
            wide = torch.full((n + 1, ff + 3), 5.0, dtype=out, device=dev())
            L.optima_mx4_linear(xq, Q, _moved(s, bw), wide[:n, :ff], x_scales=_moved(xs, bx))
            assert ((wide[:n, :ff].double() - want).abs() <= _bound(x, w, want, out)).all()
            assert (wide[n] == 5.0).all() and (wide[:, ff:] == 5.0).all()
    # 16-bit tokens, packing and back take such scales too.
    Y = torch.empty(n, ff, device=dev())
    L.optima_mx4_linear(X, Q, _moved(s, 4), Y)
    want = torch.mm(X.double(), w.t().contiguous())
    assert ((Y.double() - want).abs() <= _bound(X.double(), w, want, torch.float32)).all()
    to = _moved(torch.zeros_like(xs), 4)
    L.optima_mx4_pack(X, xq, to)
    assert torch.equal(to, xs)
    back = torch.empty(n, d, device=dev())
    L.optima_mx4_unpack(xq, to, back)
    assert torch.equal(back.double(), x)


def test_tokens_past_one_launch(L):  # noqa: F811
    """More groups of 16 tokens than a launch has in one direction, with outputs past a pitch."""
    n, d, ff = 65535 * 16 + 33, 32, 1
    Q, s, w = _weights(L, ff, d, 3)
    X = _tokens(n, d, 4)
    xq, xs = _pack(L, X)
    Y = torch.full((n, 2), 5.0, device=dev())
    L.optima_mx4_linear(xq, Q, _moved(s, 4), Y[:, :1], x_scales=xs)
    x = O.mx4_values(X)[0]
    want = torch.mm(x, w.t().contiguous())
    assert ((Y[:, :1].double() - want).abs() <= _bound(x, w, want, torch.float32)).all()
    assert (Y[:, 1] == 5.0).all()
