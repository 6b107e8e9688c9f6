"""The feed-forward half with widths that are no multiple of anything, against the fp64 oracle;
tolerances as in test_gpu_feedforward.py."""
import numpy as np
import pytest
import torch

from gpu_util import rel_fro
from oracle import feedforward_oracle as F
from test_gpu_feedforward import B, MATRICES, _np, _oracle, _start, _tokens, _weights

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d, ff", [(101, 335), (130, 322), (64, 333)])
def test_prune_recover_and_serve(d, ff):
    from paper_2512_13886_amd import feedforward as M
    block = M.synthetic_block(d, ff, seed=d)
    X, R = _tokens(701, d, ff)
    Y = M.output(block, X, R)
    x, r = _np(X), _np(R)
    y_dense = _oracle(_weights(block), x, r, block.eps)[-1]
    assert Y.shape == (701, d) and rel_fro(_np(Y), y_dense) <= 3 * B
    out, masks, rep = M.prune_feedforward(block, X, R, _start)
    for m in MATRICES:
        kept, W = masks[m].bool(), getattr(out, m)
        assert bool((W[~kept] == 0).all()) and bool((kept.sum(1) >= W.shape[1] // 2).all())
    assert rep.err_kept < rep.err_wanda
    s, a, g, u, h, y = _oracle(_weights(out), x, r, out.eps)
    ratio = np.linalg.norm(y - y_dense) / np.linalg.norm(y_dense)
    err = float(np.sum((y - y_dense) ** 2))
    assert abs(rep.err_kept - err) <= 2 * (2 * 3 * B / ratio) * err

    loss, got = M.gradients(out, masks, Y, X, R)
    assert loss == pytest.approx(rep.err_kept / (2 * 701), rel=1e-5)
    weights = _weights(out)
    da, dwg, dwu, _, _ = F.gated_backward(a, weights[1], weights[2], g, u,
                                          (y - y_dense) / 701 @ weights[3], "silu")
    _, dw = F.rms_norm_backward(s, weights[0], da, None, out.eps)
    for k, v in {"norm": dw, "gate": dwg * _np(masks["gate"]), "up": dwu * _np(masks["up"])}.items():
        assert rel_fro(_np(got[k]), v) <= (8 + 2 * 3 / ratio) * B, k

    better, losses = M.recover(out, masks, Y, X, R, steps=5)
    assert losses[-1] < losses[0] and M.output_error(better, Y, X, R) < rep.err_kept
    packed = M.PackedFeedForward(better, 32, max_tokens=3)
    S, served = R[:3].clone(), torch.empty_like(X[:3])
    packed.step(X[:3], S, served)
    values = [_np(better.norm)]
    for m in MATRICES:
        codes, scales = F.w4_quantize(getattr(better, m).cpu().numpy(), 32)
        values.append(F.w4_values(codes, scales, 32))
    _, a, _, _, _, y = _oracle(values, x[:3], r[:3], better.eps)
    half = F.group_max(a, 32)[:, F.groups_of(d, 32)] / 254
    assert rel_fro(_np(served), y) <= 2 * 1.1 * np.linalg.norm(half) / np.linalg.norm(a) + 4 * B
