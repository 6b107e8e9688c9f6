"""Sizes for every plan of the gated product and its gradient that layers of real widths take:
the 256 x 256 tiles of the gradient, with and without split sums, and the few-token kernel with
all its waves, several rounds of the main loop, and rows at odd elements. tests/test_plans_host.py
holds these sizes to their plans. Tolerances as in test_gpu_gated.py."""
import pytest

from test_gpu_gated import L, _backward, _forward  # noqa: F401  (L: the fixture)

pytestmark = pytest.mark.gpu

# n, d, ff -> tile side, ranges of dX's and dW's sums.
GRADIENTS = {(1999, 1001, 2731): (256, 3, 1), (1024, 1024, 4096): (256, 8, 1),
             (8192, 768, 3000): (256, 1, 1), (8000, 1000, 700): (256, 1, 4),
             (190, 100, 70): (128, 1, 1), (300, 200, 129): (128, 4, 4), (600, 128, 5000): (128, 16, 1)}
# All taken by the few-token kernel: sixteen waves (d >= 2048, up to 8 tokens, or up to 16 and
# few outputs), both widths of its operands, one to four blocks of tokens.
FEW = [(1, 2048, 700), (8, 2048, 700), (1, 4096, 300), (8, 4096, 700), (1, 4097, 400), (8, 4097, 400),
       (1, 9000, 40), (16, 1024, 8192), (13, 1001, 4100), (9, 2500, 5000), (16, 4097, 4100),
       (20, 2000, 500), (17, 3001, 300), (32, 1100, 4100), (40, 1500, 200), (64, 1101, 600)]


@pytest.mark.parametrize("n, d, ff", list(GRADIENTS))
def test_gradient(L, n, d, ff):  # noqa: F811
    _backward(L, n, d, ff, masked=True)


@pytest.mark.parametrize("n, d, ff", [(1024, 1024, 4096), (8000, 1000, 700)])
def test_gradient_fp32(L, n, d, ff):  # noqa: F811
    _backward(L, n, d, ff, name="none", dx="f32", dw="f32", pad=3)


@pytest.mark.parametrize("n, d, ff", FEW)
def test_few_tokens(L, n, d, ff):  # noqa: F811
    _forward(L, n, d, ff)
    _forward(L, n, d, ff, name="none", out="f32", xpitch=d + 3, xoff=1)
