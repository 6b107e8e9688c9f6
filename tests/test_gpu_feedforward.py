"""The feed-forward half of a block, pruned, recovered and served, against the fp64 oracle.

Tolerances, B = 2^-8 (half a bf16 step, relative). A matrix that is rounded to bf16
changes by at most B of its Frobenius norm, and products with random matrices pass that
on. On the way to y three are rounded (a, h, and g and u as the gradient sees them), and y -
y_dense has the rounding of both y relative to a difference that is `ratio` times as
large. The gradient rounds dy, dh, dg and du, and da. The served block's 8-bit codes are
off by half a step, max / 254, in each value of a group."""
import numpy as np
import pytest
import torch

from gpu_util import dev, log, rel_fro
from oracle import feedforward_oracle as F

pytestmark = pytest.mark.gpu

B = 2.0 ** -8
MATRICES = ("gate", "up", "down")


@pytest.fixture(scope="module")
def ff():
    from paper_2512_13886_amd import feedforward
    return feedforward


def _np(t):
    return t.double().cpu().numpy()


def _tokens(n, d, seed):
    g = torch.Generator(device=dev()).manual_seed(seed)
    spread = torch.exp(torch.randn(d, generator=g, device=dev()))
    return tuple((torch.randn((n, d), generator=g, device=dev()) * spread).bfloat16()
                 for _ in range(2))


def _weights(block):
    """The norm's weight in fp64 and the matrices as the products take them."""
    return [_np(block.norm)] + [_np(getattr(block, m).bfloat16()) for m in MATRICES]


def _oracle(weights, x, r, eps):
    w, wg, wu, wd = weights
    s, a = F.rms_norm(x, r, w, eps)
    h, g, u = F.gated(a, wg, wu, "silu")
    return s, a, g, u, h, h @ wd.T


def _start(width):
    g = torch.Generator(device=dev()).manual_seed(width)
    return torch.randn((8, width), generator=g, device=dev())


@pytest.fixture(scope="module")
def pruned(ff):
    block = ff.synthetic_block(128, 320, seed=3)
    X, R = _tokens(1024, 128, 4)
    Y = ff.output(block, X, R)
    return block, X, R, Y, *ff.prune_feedforward(block, X, R, _start)


def test_output(ff, pruned):
    block, X, R, Y = pruned[:4]
    y = _oracle(_weights(block), _np(X), _np(R), block.eps)[-1]
    assert rel_fro(_np(Y), y) <= 3 * B


def test_prune(ff, pruned):
    block, X, R, Y, out, masks, rep = pruned
    for m in MATRICES:
        mask, W = masks[m].bool(), getattr(out, m)
        assert bool((mask.sum(1) == W.shape[1] // 2).all())
        assert bool((W[~mask] == 0).all())
    assert rep.err_kept < rep.err_wanda
    assert not any(rep.skipped.values()) and all(v > 0 for v in rep.iterations.values())
    x, r = _np(X), _np(R)
    y_dense = _oracle(_weights(block), x, r, block.eps)[-1]
    y = _oracle(_weights(out), x, r, out.eps)[-1]
    err = float(np.sum((y - y_dense) ** 2))
    ratio = np.sqrt(err / np.sum(y_dense ** 2))
    log(f"  error of the outputs {ratio:.3f}, mask only "
        f"{np.sqrt(rep.err_wanda / np.sum(y_dense ** 2)):.3f}")
    assert abs(rep.err_kept - err) <= 2 * (2 * 3 * B / ratio) * err


def test_gradients(ff, pruned):
    block, X, R, Y, out, masks, rep = pruned
    n = X.shape[0]
    loss, got = ff.gradients(out, masks, Y, X, R)
    assert loss == pytest.approx(rep.err_kept / (2 * n), rel=1e-5)
    x, r, weights = _np(X), _np(R), _weights(out)
    y_dense = _oracle(_weights(block), x, r, block.eps)[-1]

    def oracle_loss(weights):
        return np.sum((_oracle(weights, x, r, out.eps)[-1] - y_dense) ** 2) / (2 * n)

    s, a, g, u, h, y = _oracle(weights, x, r, out.eps)
    dy = (y - y_dense) / n
    da, dwg, dwu, _, _ = F.gated_backward(a, weights[1], weights[2], g, u, dy @ weights[3], "silu")
    _, dw = F.rms_norm_backward(s, weights[0], da, None, out.eps)
    want = {"norm": dw, "gate": dwg * _np(masks["gate"]), "up": dwu * _np(masks["up"])}
    ratio = np.linalg.norm(y - y_dense) / np.linalg.norm(y_dense)
    for k, v in want.items():
        assert rel_fro(_np(got[k]), v) <= (8 + 2 * 3 / ratio) * B, k
    for k in ("gate", "up"):
        assert bool((got[k][masks[k] == 0] == 0).all())
    # Along the gradient the oracle's own loss changes by its square.
    for i, k in enumerate(("norm", "gate", "up")):
        step = 1e-4 * np.linalg.norm(weights[i]) / np.linalg.norm(want[k])
        both = []
        for sign in (1, -1):
            moved = list(weights)
            moved[i] = weights[i] + sign * step * want[k]
            both.append(oracle_loss(moved))
        assert (both[0] - both[1]) / (2 * step) == pytest.approx(np.sum(want[k] ** 2), rel=1e-4)


def test_recover(ff, pruned):
    block, X, R, Y, out, masks, rep = pruned
    before = {m: getattr(out, m).clone() for m in ("norm", *MATRICES)}
    better, losses = ff.recover(out, masks, Y, X, R, steps=10)
    assert len(losses) == 10 and losses[-1] < losses[0]
    assert ff.output_error(better, Y, X, R) < rep.err_kept
    for m in ("norm", *MATRICES):
        assert torch.equal(getattr(out, m), before[m])
    for m in MATRICES:
        assert bool((getattr(better, m)[masks[m] == 0] == 0).all())
    again, _ = ff.recover(out, masks, Y, X, R, steps=10)
    assert all(torch.equal(getattr(better, m), getattr(again, m)) for m in ("norm", *MATRICES))


@pytest.mark.parametrize("n, group", [(1, 128), (1, 32), (5, 64), (40, 128)])
def test_serve(ff, pruned, n, group):
    out = pruned[4]
    X, R = _tokens(n, 128, 9)
    packed = ff.PackedFeedForward(out, group, max_tokens=n)
    S, Y = R.clone(), torch.empty_like(X)
    packed.step(X, S, Y)
    values = [_np(out.norm)]
    for m in MATRICES:
        codes, scales = F.w4_quantize(getattr(out, m).cpu().numpy(), group)
        values.append(F.w4_values(codes, scales, group))
    s, a, g, u, h, y = _oracle(values, _np(X), _np(R), out.eps)
    assert np.all(np.abs(_np(S) - s) <= B * np.abs(s) * 1.01)
    half = F.group_max(a, group)[:, F.groups_of(128, group)] / 254
    codes_off = np.linalg.norm(half) / np.linalg.norm(a)
    # g and u both carry the codes' roundings, with slopes of up to 1.1; h and y their own.
    assert rel_fro(_np(Y), y) <= 2 * 1.1 * codes_off + 4 * B


def test_serve_in_a_graph(ff, pruned):
    out = pruned[4]
    X, R = _tokens(1, 128, 11)
    packed = ff.PackedFeedForward(out)
    x, s, y = X.clone(), R.clone(), torch.empty_like(X)
    packed.step(x, s, y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        packed.step(x, s, y)
    for seed in range(4):
        X, R = _tokens(1, 128, 20 + seed)
        s2, y2 = R.clone(), torch.empty_like(X)
        packed.step(X, s2, y2)
        x.copy_(X)
        s.copy_(R)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(s, s2) and torch.equal(y, y2)


def test_serve_refuses_more_tokens(ff, pruned):
    packed = ff.PackedFeedForward(pruned[4], max_tokens=2)
    X, R = _tokens(3, 128, 1)
    with pytest.raises(ValueError):
        packed.step(X, R, torch.empty_like(X))
