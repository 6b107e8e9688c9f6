"""4-bit products of up to 16 tokens over more batches of chunks than a workgroup has waves, at
every number of tokens a wave loads at once and of waves its LDS leaves. Tolerances as in
test_gpu_w4.py."""
import pytest

from test_gpu_w4 import L, _run  # noqa: F401  (L: the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [1, 4, 5, 8, 9, 10, 12, 15, 16])
@pytest.mark.parametrize("d", [4500, 9001])
@pytest.mark.parametrize("x, x_group", [("bf16", 0), ("i8", 64)])
@pytest.mark.parametrize("gated", [None, "silu"])
def test_few_tokens(L, n, d, x, x_group, gated):  # noqa: F811
    _run(L, n, d, 50, 64, x, x_group, y="f32", pad=1, gated=gated)
