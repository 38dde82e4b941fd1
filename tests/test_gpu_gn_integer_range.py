"""Group norm on integer sums over the whole range of their exponents and of their errors' exponents."""
import numpy as np
import pytest
import torch

from paper_2105_13890_b200 import eoq

import gpu_util as G
import wide_reference as R

pytestmark = pytest.mark.gpu

SHAPES = [(2, 64, 64, 8), (3, 35, 48, 3), (1, 7000, 40, 1), (2, 9, 4100, 4)]


def call(acc, e, e_exp, gamma, beta, groups, x_exp, eps, kept, act):
    n, hw, c = acc.shape
    d = eoq.gn_desc(n, hw, c, groups, eoq.EOQ_I32, act, eps, x_exp=x_exp)
    ws = G.empty(eoq.eoq_gn_workspace_size(d), torch.uint8)
    accd, ed, ee, g, b = (G.dev(v) for v in (acc, e, np.array([e_exp], np.int32), gamma, beta))
    y, dx = G.zeros((n, hw, c), torch.int8), G.zeros((n, hw, c), torch.float32)
    stats, dg, db = G.zeros((n, groups, 2), torch.float32), G.zeros(c, torch.float32), G.zeros(c, torch.float32)
    codes = G.zeros((n, hw, c), torch.int8) if kept == "codes" else None
    exps = G.zeros((n * hw, -(-c // 32)), torch.uint8) if kept == "codes" else None
    eoq.eoq_gn_fwd(G.handle(), d, accd, g, b, y, stats, codes, exps, ws)
    eoq.eoq_gn_bwd(G.handle(), d, ed, ee, None if codes is not None else accd, codes, exps, g, b, stats, dx, dg, db, ws)
    torch.cuda.synchronize()
    assert G.status_clear() == 0
    return [G.host(t).astype(np.float64) for t in (y, stats, dx, dg, db)]


def make(n, hw, c, seed):
    rng = np.random.default_rng(seed)
    acc = rng.integers(-40000, 60000, (n, hw, c)).astype(np.int32)
    e = np.clip(np.rint(rng.normal(0, 32, (n, hw, c))), -127, 127).astype(np.int8)
    return acc, e, rng.normal(0.5, 0.1, c).astype(np.float32), rng.normal(0, 0.1, c).astype(np.float32)


@pytest.mark.parametrize("kept", ["input", "codes"])
@pytest.mark.parametrize("x_exp,eps", [(60, 1e-5), (45, 0.0), (-60, 0.0), (-60, 1e-34)])
@pytest.mark.parametrize("n,hw,c,groups", SHAPES)
def test_every_exponent_of_the_sums(n, hw, c, groups, x_exp, eps, kept):
    """At 60 the squares of the values lie far beyond fp32, mean, rstd and all that is returned within it."""
    acc, e, gamma, beta = make(n, hw, c, 3 + c)
    y, stats, dx, dg, db = call(acc, e, -12, gamma, beta, groups, x_exp, eps, kept, eoq.EOQ_ACT_SILU)
    xw, g, b, eps = acc.astype(np.float64) * 2.0 ** x_exp, gamma.astype(np.float64), beta.astype(np.float64), float(np.float32(eps))
    want, mean, rstd, bound = R.gn_fwd(xw, groups, eps, g, b, "silu")
    top = np.abs(xw).reshape(n, hw, groups, -1).max((1, 3))
    R.within(stats[..., 0], mean, 64 * R.EPS32 * top)
    R.within(stats[..., 1], rstd, rstd * 64 * R.EPS32 * (1 + top * rstd))
    assert (np.abs(y - np.clip(want * 128, -127, 127)) <= 0.5 + 128 * bound).all()
    if kept == "codes":
        xw = R.block_form(xw.reshape(-1, c))[2].reshape(xw.shape)
    r = R.gn_bwd(e.astype(np.float64) * 2.0 ** -12, xw, stats[..., 0], stats[..., 1], g, b, "silu")
    for got, at in ((dx, 0), (dg, 1), (db, 2)):
        R.within(got, r[at], r[at + 3])


@pytest.mark.parametrize("kept", ["input", "codes"])
@pytest.mark.parametrize("e_exp", [120, -120])
@pytest.mark.parametrize("n,hw,c,groups", SHAPES)
def test_every_exponent_of_the_errors(n, hw, c, groups, e_exp, kept):
    """Errors of one sign in one channel and of the other in the next: at 120 the sums of either are no fp32 numbers, dx is one."""
    acc, e, gamma, beta = make(n, hw, c, 7 + c)
    acc, e = acc * 8, (np.abs(e) + 64).clip(max=127).astype(np.int8)
    e[..., 1::2] = -e[..., 1::2]
    _, stats, dx, dg, db = call(acc, e, e_exp, gamma, beta, groups, -14, 1e-5, kept, eoq.EOQ_ACT_NONE)
    xw = acc.astype(np.float64) * 2.0 ** -14
    if kept == "codes":
        xw = R.block_form(xw.reshape(-1, c))[2].reshape(xw.shape)
    r = R.gn_bwd(e.astype(np.float64) * 2.0 ** e_exp, xw, stats[..., 0], stats[..., 1], gamma.astype(np.float64), beta.astype(np.float64), "none")
    assert np.abs(r[0]).max() < 2.0 ** 128
    R.within(dx, r[0], r[3])
    for got, at in ((dg, 1), (db, 2)):
        # what is certain to be beyond the largest number, and what is not near it
        beyond, inside = np.abs(r[at]) - r[at + 3] > 2.0 ** 128, np.abs(r[at]) + r[at + 3] < 2.0 ** 128 * (1 - 2.0 ** -20)
        assert (got[beyond] == np.copysign(np.inf, r[at][beyond])).all()
        R.within(got[inside], r[at][inside], r[at + 3][inside])
    assert e_exp < 0 or np.isinf(db).any()
