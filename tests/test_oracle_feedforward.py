"""The feed-forward oracle: hand-worked values, gradients against differences,
and the 4-bit layout against its description."""
import numpy as np
import pytest
import torch

from oracle import feedforward_oracle as F


def test_bf16_matches_torch():
    rng = np.random.default_rng(1)
    v = (rng.standard_normal(4096) * np.exp(rng.uniform(-40, 40, 4096))).astype(np.float32)
    want = torch.from_numpy(v).bfloat16().double().numpy()
    assert np.array_equal(F.bf16(v), want)
    assert np.isnan(F.bf16(np.array([np.nan], np.float32))[0])


def test_norm_by_hand():
    # rows (3, 4) + (0, 0): mean square 12.5
    s, y = F.rms_norm(np.array([[3.0, 4.0]]), None, np.array([1.0, 2.0]), 0.0)
    assert np.allclose(y, [[3 / np.sqrt(12.5), 8 / np.sqrt(12.5)]])
    s, y = F.rms_norm(np.array([[1.0, 2.0]]), np.array([[2.0, 2.0]]), np.ones(2), 0.0)
    assert np.array_equal(s, [[3.0, 4.0]])


@pytest.mark.parametrize("d", [1, 2, 7])
def test_norm_gradient_against_differences(d):
    rng = np.random.default_rng(d)
    s, w = rng.standard_normal((3, d)), rng.standard_normal(d)
    dy, ds = rng.standard_normal((3, d)), rng.standard_normal((3, d))
    eps, h = 1e-3, 1e-5
    dx, dw = F.rms_norm_backward(s, w, dy, ds, eps)

    def loss(s, w):
        return np.sum(dy * F.rms_norm(s, None, w, eps)[1]) + np.sum(ds * s)

    for i in np.ndindex(*s.shape):
        e = np.zeros_like(s)
        e[i] = h
        assert abs((loss(s + e, w) - loss(s - e, w)) / (2 * h) - dx[i]) <= 1e-7 * (1 + abs(dx[i]))
    for i in range(d):
        e = np.zeros(d)
        e[i] = h
        assert abs((loss(s, w + e) - loss(s, w - e)) / (2 * h) - dw[i]) <= 1e-7 * (1 + abs(dw[i]))


@pytest.mark.parametrize("name", ["silu", "none"])
def test_gated_gradient_against_differences(name):
    rng = np.random.default_rng(3)
    x, wg, wu = rng.standard_normal((4, 3)), rng.standard_normal((5, 3)), rng.standard_normal((5, 3))
    dh = rng.standard_normal((4, 5))
    _, g, u = F.gated(x, wg, wu, name)
    dx, dwg, dwu, _, _ = F.gated_backward(x, wg, wu, g, u, dh, name)
    h = 1e-5
    for k, (v, grad) in enumerate(((x, dx), (wg, dwg), (wu, dwu))):
        for i in np.ndindex(*v.shape):
            e = np.zeros_like(v)
            e[i] = h
            up = [x, wg, wu]
            dn = [x, wg, wu]
            up[k], dn[k] = v + e, v - e
            diff = (np.sum(dh * F.gated(*up, name)[0]) - np.sum(dh * F.gated(*dn, name)[0])) / (2 * h)
            assert abs(diff - grad[i]) <= 1e-7 * (1 + abs(grad[i]))


def test_w4_rule_and_layout():
    w = np.zeros((1, 130), np.float32)
    w[0, 0], w[0, 1], w[0, 33], w[0, 129] = 7.0, -3.4, 2.0, -1.0
    codes, scales = F.w4_quantize(w, 32)
    assert scales.shape == (1, 5)
    assert scales[0, 0] == 1.0 and scales[0, 2] == 0.0
    assert codes[0, 0] == 7 and codes[0, 1] == -3 and codes[0, 33] == 7 and codes[0, 129] == -7
    q = F.w4_layout(codes)
    assert q.shape == (1, 128)
    # code 0: chunk 0, block 0, dword 0, nibble 0; code 1: nibble 4 of the same dword
    assert q[0, 0] == 0x80 | 15 and q[0, 2] == 0x80 | 5
    # code 33: dword 1 of block 0, nibble 4; code 129: chunk 1, nibble 4
    assert q[0, 6] == 0x80 | 15 and q[0, 64 + 2] == 0x80 | 1
    assert np.count_nonzero(q != 0x88) == 4


def test_w4_zeros_stay_zero():
    rng = np.random.default_rng(5)
    w = (rng.standard_normal((8, 200)) * (rng.random((8, 200)) < 0.5)).astype(np.float32)
    for group in (32, 64, 128):
        codes, scales = F.w4_quantize(w, group)
        v = F.w4_values(codes, scales, group)
        assert np.all(v[w == 0] == 0)
        # half a step, and what the scale's rounding to 8 bits cuts off at the top
        step = scales[:, F.groups_of(200, group)]
        assert np.all(np.abs(v - w) <= 0.5 * step * (1 + 2.0 ** -5))
