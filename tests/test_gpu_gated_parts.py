"""An output of the gated gradient has the same bits whether or not the others are asked for:
the order of its sums goes by the sizes alone. Sizes at which sums are split, differently for the
best of one output and of all, and one whose sums are not."""
import pytest
import torch

from gpu_util import dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n, d, ff", [(600, 128, 5000), (256, 1024, 2816), (1024, 1024, 4096),
                                      (190, 100, 70), (3, 300, 2000)])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_outputs_alone_and_together(n, d, ff, dt):
    import paper_2512_13886_amd as L
    g = torch.Generator(device=dev()).manual_seed(n + d + ff)

    def rows(r, c):
        return torch.randn(r, c, generator=g, device=dev()).bfloat16()

    X, Wg, Wu, G, V, dH = (rows(*s) for s in ((n, d), (ff, d), (ff, d), (n, ff), (n, ff), (n, ff)))
    dX, dWg, dWu, x, wg, wu = (torch.empty(s, dtype=dt, device=dev())
                               for s in 2 * ((n, d), (ff, d), (ff, d)))
    L.optima_gated_backward(X, Wg, Wu, G, V, dH, dX=dX, dWg=dWg, dWu=dWu)
    L.optima_gated_backward(X, Wg, Wu, G, V, dH, dX=x)
    L.optima_gated_backward(X, Wg, Wu, G, V, dH, dWg=wg, dWu=wu)
    assert torch.equal(x, dX) and torch.equal(wg, dWg) and torch.equal(wu, dWu)
