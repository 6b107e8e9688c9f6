"""The oracle of the packed products and the log probabilities against values worked out by hand
and against differences."""
import torch

from oracle import answers_oracle as O


def test_codes_of_a_block():
    # max 5.0: e = 2, scale 1. Ties go to the even code: 0.25 -> 0, 0.75 -> 1, 1.25 -> 1,
    # 1.75 -> 2, 2.5 -> 2, 3.5 -> 4, 5 -> 4.
    x = torch.tensor([[0.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.3, -0.25, 4.9]])
    v, c, s = O.mx4_values(x)
    assert v.tolist() == [[0.0, 0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, -0.5, 0.0, 4.0]]
    assert c.tolist() == [[0, 0, 2, 2, 4, 4, 6, 6, 9, 8, 6]] and s.tolist() == [[127]]


def test_scales():
    x = torch.zeros(1, 32 * 6)
    x[0, 32] = 7.9          # the largest of its binade is cut to 6
    x[0, 64] = 2.0 ** -149  # scales stop at 2^-127
    x[0, 96] = 3e38
    x[0, 128] = float("inf")
    x[0, 160] = float("nan")
    v, _, s = O.mx4_values(x)
    assert s.tolist() == [[0, 127, 0, 252, 255, 255]]
    assert v[0, 32] == 6.0 and v[0, 64] == 0.0 and v[0, 96] == 6.0 * 2.0 ** 125
    assert torch.isnan(v[0, 128:]).all() and not torch.isnan(v[0, :128]).any()


def test_layout_places():
    n, d = 2, 700
    code = torch.arange(n * d).view(n, d) % 16
    scale = torch.arange(n * 22).view(n, 22)
    Q, S = O.mx4_layout(code.to(torch.uint8), scale.to(torch.uint8))
    assert Q.shape == (2, 384) and S.shape == (2, 32)
    assert int(Q[1, 100]) == int(code[1, 200]) + 16 * int(code[1, 201])
    # Block 21 of the row: 128 values number 5, block 1 of them.
    assert int(S[1, 16 + 4 * 1 + 1]) == 22 + 21


def test_gradient_against_differences():
    g = torch.Generator().manual_seed(0)
    x = torch.randn(4, 9, generator=g, dtype=torch.float64)
    x[1, 3] = x[1, 5] = -float("inf")
    tokens = torch.tensor([2, 0, -1, 8])
    dlogp, dh, dl = (torch.randn(4, generator=g, dtype=torch.float64) for _ in range(3))

    def f(x):
        lse, logp, entropy = O.token_logprobs(x, tokens, 0.7)
        return (dlogp * logp + dh * entropy + dl * lse).sum()

    want = O.token_logprobs_gradient(x, tokens, dlogp, dh, dl, 0.7)
    for r in range(4):
        for c in range(9):
            if x[r, c] == -float("inf"):
                assert want[r, c] == 0
                continue
            up, down = x.clone(), x.clone()
            up[r, c] += 1e-5
            down[r, c] -= 1e-5
            # Second order differences: 1e-10 of third derivatives of order 1, and 1e-16 / 1e-5.
            assert abs((f(up) - f(down)) / 2e-5 - want[r, c]) < 1e-8


def test_rows_with_nothing_left():
    inf, nan = float("inf"), float("nan")
    x = torch.tensor([[-inf, -inf], [1.0, nan], [inf, 0.0], [0.0, -inf]])
    lse, logp, entropy = O.token_logprobs(x, torch.tensor([0, 0, 1, 0]))
    assert lse[0] == -inf and logp[0] == -inf and entropy[0] == 0
    assert all(torch.isnan(o[i]) for o in (lse, logp, entropy) for i in (1, 2))
    assert lse[3] == 0 and logp[3] == 0 and entropy[3] == 0
    assert O.top(torch.tensor([[1.0, 3.0, 1.0, 3.0]]), 3).tolist() == [[1, 3, 0]]
