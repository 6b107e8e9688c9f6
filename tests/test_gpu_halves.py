"""The feed-forward calls on columns of one buffer: the same bits as on matrices of their own."""
import pytest
import torch

from gpu_util import dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n, d, ff", [(3, 100, 33), (7, 64, 64), (200, 65, 129)])
def test_columns_of_one_buffer(n, d, ff):
    import paper_2512_13886_amd as L
    g = torch.Generator(device=dev()).manual_seed(n)

    def rows(r, c):
        return torch.randn(r, c, generator=g, device=dev()).bfloat16()

    X, R, Wg, Wu, dH = rows(n, d), rows(n, d), rows(ff, d), rows(ff, d), rows(n, ff)
    w = torch.rand(d, generator=g, device=dev()) + 0.5

    def run(wide):
        def matrices(*widths):
            if wide:
                buf = torch.full((n, sum(widths)), 7.0, dtype=torch.bfloat16, device=dev())
                return torch.split(buf, widths, 1)
            return [torch.full((n, c), 7.0, dtype=torch.bfloat16, device=dev()) for c in widths]
        S, A = matrices(d, d)
        L.optima_rms_norm(X, w, A, R=R, S=S)
        G, U, H = matrices(ff, ff, ff)
        L.optima_gated_forward(A, Wg, Wu, H, G=G, U=U)
        dX, x = matrices(d, d)
        x.copy_(A)
        L.optima_gated_backward(x, Wg, Wu, G, U, dH, dX=dX)
        return [t.clone() for t in (S, A, G, U, H, dX, x)]

    assert all(torch.equal(a, b) for a, b in zip(run(False), run(True)))
