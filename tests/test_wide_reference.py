"""The plain forms that the floating-point operators are compared with, against what they have to be: differences, closed forms."""
import numpy as np
import pytest

import wide_reference as R


@pytest.mark.parametrize("kind", ["none", "relu", "silu"])
def test_gradients_are_those_of_the_forward_pass(kind):
    rng = np.random.default_rng(1)
    n, hw, c, groups, eps = 2, 5, 6, 3, 1e-3
    x = rng.normal(size=(n, hw, c)) + 0.3
    gamma, beta, dy = rng.normal(1, 0.3, c), rng.normal(0, 0.3, c), rng.normal(size=(n, hw, c))

    def loss(x, gamma, beta):
        return (R.gn_fwd(x, groups, eps, gamma, beta, kind)[0] * dy).sum()

    mean, rstd = R.gn_stats(x, groups, eps)
    dx, dgamma, dbeta = R.gn_bwd(dy, x, mean, rstd, gamma, beta, kind)[:3]
    h = 1e-6
    for v, grad in ((x, dx), (gamma, dgamma), (beta, dbeta)):
        for at in list(np.ndindex(v.shape))[:24]:
            keep = v[at]
            v[at] = keep + h
            up = loss(x, gamma, beta)
            v[at] = keep - h
            down = loss(x, gamma, beta)
            v[at] = keep
            assert abs((up - down) / (2 * h) - grad[at]) < 1e-6 * (1 + abs(grad[at]))


def test_block_form():
    x = np.zeros((6, 40))
    x[0, :3] = [127.0, -127.0, 126.5]          # exactly 127 steps of 1; a tie goes to the even code
    x[1, :3] = [127.0001, 64.0, 1.0]           # the step doubles
    x[2, 33] = 1e-45                           # the smallest step there is
    x[3, 0] = np.inf
    x[4, 39] = np.nan
    x[5, 0], x[5, 1] = 1.9999 * 2.0 ** 127, 2.0 ** 121
    codes, exps, back = R.block_form(x)
    assert list(codes[0, :3]) == [127, -127, 126] and exps[0, 0] == 127
    assert list(codes[1, :3]) == [64, 32, 0] and exps[1, 0] == 128
    assert exps[2, 1] == 1 and not codes[2].any() and exps[2, 0] == 1
    assert exps[3, 0] == 255 and np.isnan(back[3, :32]).all() and not back[3, 32:].any()
    assert exps[4, 1] == 255 and np.isnan(back[4, 32:]).all() and not back[4, :32].any()
    assert exps[5, 0] == 249 and codes[5, 0] == 63 and codes[5, 1] == 0     # 2^121 is half a step of 2^122: to the even code
    y = np.random.default_rng(0).normal(size=(50, 70)) * np.exp(np.random.default_rng(1).normal(0, 4, (50, 1)))
    _, exps, back = R.block_form(y)
    step = np.repeat(2.0 ** (exps.astype(float) - 127), 32, 1)[:, :70]
    assert (np.abs(back - y) <= step / 2).all() and (np.abs(back) <= 127 * step).all()
