"""Few 16-bit tokens: every form of the kernel that splits a row's sum over waves, in one and in two blocks
of outputs, of widths that are multiples of 8 and of others."""
import pytest
import torch

from test_gpu_mx4 import L, _bound, _check, _tokens, _weights, dev  # noqa: F401
from test_mx4_few_host import FEW

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n, d, ff", sorted(FEW))
def test_every_few_token_form(L, n, d, ff):  # noqa: F811
    Q, s, w = _weights(L, ff, d, 5)
    _check(L, _tokens(n, d, 6), Q, s, w, torch.float32, False, pad=1)
    _check(L, _tokens(n, d, 7, pad=3), Q, s, w, torch.bfloat16, False)


@pytest.mark.parametrize("n, d, ff", ((3, 1001, 66000), (8, 1001, 13000), (16, 1001, 9000)))
def test_rows_at_odd_elements(L, n, d, ff):  # noqa: F811
    """A NaN before and behind every row of tokens: nothing past a row's ends is used."""
    Q, s, w = _weights(L, ff, d, 5)
    flat = torch.full((n * (d + 2) + 1,), float("nan"), dtype=torch.bfloat16, device=dev())
    X = flat[1:].view(n, d + 2)[:, :d]
    X.copy_(_tokens(n, d, 6))
    Y = torch.empty(n, ff, device=dev())
    L.optima_mx4_linear(X, Q, s, Y)
    want = torch.mm(X.double(), w.t().contiguous())
    assert ((Y.double() - want).abs() <= _bound(X.double(), w, want, torch.float32)).all()
