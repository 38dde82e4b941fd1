"""Group norm with an activation, channels last (eoq_gn_fwd, eoq_gn_bwd), against its plain form in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2105_13890_b200 import eoq

import gpu_util as G
import wide_reference as R

pytestmark = pytest.mark.gpu

TYPES = {"fp32": (torch.float32, eoq.EOQ_F32), "fp16": (torch.float16, eoq.EOQ_F16), "bf16": (torch.bfloat16, eoq.EOQ_BF16)}
ACTS = {"none": eoq.EOQ_ACT_NONE, "relu": eoq.EOQ_ACT_RELU, "silu": eoq.EOQ_ACT_SILU}
# n, pixels, channels, groups, and channels of the wider tensors that x, y, dy and dx are parts of
SHAPES = [
    (1, 1, 8, 1, 0), (1, 1, 8, 8, 0), (2, 1, 64, 32, 0), (3, 2, 16, 4, 0), (1, 49, 512, 32, 0), (2, 196, 256, 32, 0), (3, 45, 120, 8, 0),
    (3, 45, 120, 8, 24), (2, 61, 30, 5, 0), (2, 61, 35, 5, 3), (1, 7, 13, 1, 0), (5, 300, 8, 2, 0), (2, 333, 96, 16, 0), (1, 2100, 16, 4, 0),
    (1, 50, 2048, 1, 0), (2, 9, 4100, 4, 0), (1, 5, 1001, 7, 0), (40, 3, 64, 16, 0), (600, 4, 32, 8, 8), (1, 12000, 64, 32, 0), (2, 5, 24, 2, 8),
    (1, 900, 320, 10, 0), (2, 700, 72, 24, 0),
]


def make(n, hw, c, extra, name, seed, mean=0.5, spread=1.0):
    rng = np.random.default_rng(seed)
    td = TYPES[name][0]
    x = torch.from_numpy(rng.normal(mean, spread, (n, hw, c + extra)) * rng.uniform(0.5, 1.5, c + extra)).to(td).to("cuda:0")
    dy = torch.from_numpy(rng.normal(0, 0.1, (n, hw, c + extra))).to(td).to("cuda:0")
    gamma, beta = rng.normal(1, 0.3, c).astype(np.float32), rng.normal(0, 0.3, c).astype(np.float32)
    return x, dy, gamma, beta


def call(x, dy, gamma, beta, c, groups, name, kind, kept, eps=1e-5, want=True):
    """Forward and backward on the GPU; tensors [n, hw, c + extra], of which the first c channels count."""
    n, hw, width = x.shape
    td, ed = TYPES[name]
    d = eoq.gn_desc(n, hw, c, groups, ed, ACTS[kind], eps, x_stride=width, y_stride=width, dy_stride=width, dx_stride=width)
    ws = torch.full((eoq.eoq_gn_workspace_size(d) + 256,), 0xFF, dtype=torch.uint8, device="cuda:0")   # (NaN everywhere)
    y, dx = torch.full_like(x, 33.0), torch.full_like(x, 33.0)
    stats, dgamma, dbeta = G.zeros((n, groups, 2), torch.float32), G.zeros(c, torch.float32), G.zeros(c, torch.float32)
    blocks = -(-c // 32)
    codes = torch.full((n * hw * c + 16,), 77, dtype=torch.int8, device="cuda:0") if kept == "codes" else None
    exps = torch.full((n * hw * blocks + 16,), 78, dtype=torch.uint8, device="cuda:0") if kept == "codes" else None
    g, b = (None if v is None else G.dev(v) for v in (gamma, beta))
    need = eoq.eoq_gn_workspace_size(d)
    eoq.eoq_gn_fwd(G.handle(), d, x, g, b, y, stats, codes, exps, ws[:need])
    ws[:need].fill_(0xFF)
    eoq.eoq_gn_bwd(G.handle(), d, dy, None, None if kept == "codes" else x, codes, exps, g, b, stats, dx, dgamma if want else None,
                   dbeta if want else None, ws[:need])
    torch.cuda.synchronize()
    assert (ws[need:] == 0xFF).all() and (y[..., c:] == 33).all() and (dx[..., c:] == 33).all()
    if codes is not None:
        assert (codes[n * hw * c:] == 77).all() and (exps[n * hw * blocks:] == 78).all()
        codes, exps = codes[:n * hw * c].view(n, hw, c), exps[:n * hw * blocks].view(n * hw, blocks)
    return {"y": y[..., :c], "stats": stats, "codes": codes, "exps": exps, "dx": dx[..., :c], "dgamma": dgamma, "dbeta": dbeta}


def wide(t):
    return t.double().cpu().numpy()


def check(x, dy, gamma, beta, c, groups, name, kind, kept, eps=1e-5):
    got = call(x, dy, gamma, beta, c, groups, name, kind, kept, eps)
    xw, dyw = wide(x[..., :c]), wide(dy[..., :c])
    one, zero = np.ones(c), np.zeros(c)
    g, b = (one if gamma is None else gamma.astype(np.float64)), (zero if beta is None else beta.astype(np.float64))
    y, mean, rstd, bound = R.gn_fwd(xw, groups, eps, g, b, kind)
    R.within(wide(got["y"]), y, bound, name)
    n, hw = x.shape[:2]
    top = np.abs(xw).reshape(n, hw, groups, -1).max((1, 3))
    stats = wide(got["stats"])
    # (see gn_fwd: the mean to 64 roundings of the largest value, rstd by half the relative error of the variance)
    R.within(stats[..., 0], mean, 64 * R.EPS32 * top)
    R.within(stats[..., 1], rstd, rstd * 64 * R.EPS32 * (1 + top * rstd))
    if kept == "codes":
        codes, exps, back = R.block_form(xw.reshape(-1, c))
        assert np.array_equal(G.host(got["codes"]).reshape(-1, c), codes) and np.array_equal(G.host(got["exps"]), exps)
        xw = back.reshape(xw.shape)
    dx, dgamma, dbeta, bdx, bdgamma, bdbeta = R.gn_bwd(dyw, xw, stats[..., 0], stats[..., 1], g, b, kind)
    got_dx = wide(got["dx"])
    if kind == "relu":
        # where z is within its error of zero the gate may go either way: those elements, and what the sums move with them, are left out
        u = (xw - R._wide(stats[..., 0], c)) * R._wide(stats[..., 1], c)
        z = g * u + b
        doubt = np.abs(z) < 16 * R.EPS32 * (np.abs(g) * (np.abs(xw) + np.abs(R._wide(stats[..., 0], c))) * R._wide(stats[..., 1], c) + np.abs(b))
        assert doubt.sum() <= 2 + 1e-4 * doubt.size
        loose = (np.abs(g * dyw) * doubt).reshape(n, hw, groups, -1).mean((1, 3))
        r = R._wide(stats[..., 1], c)
        bdx = bdx + r * (R._wide(loose, c) * (1 + np.abs(u) * np.abs(u).max()) + np.abs(g * dyw) * doubt)
        bdbeta = bdbeta + (np.abs(dyw) * doubt).sum((0, 1))
        bdgamma = bdgamma + (np.abs(dyw * u) * doubt).sum((0, 1))
    R.within(got_dx, dx, bdx, name)
    R.within(wide(got["dgamma"]), dgamma, bdgamma)
    R.within(wide(got["dbeta"]), dbeta, bdbeta)
    return got


@pytest.mark.parametrize("name", sorted(TYPES))
@pytest.mark.parametrize("n,hw,c,groups,extra", SHAPES)
def test_shapes_and_types(n, hw, c, groups, extra, name):
    x, dy, gamma, beta = make(n, hw, c, extra, name, n * 31 + hw * 7 + c)
    for kept in ("input", "codes"):
        check(x, dy, gamma, beta, c, groups, name, "silu", kept)


@pytest.mark.parametrize("name", sorted(TYPES))
@pytest.mark.parametrize("n,hw,c,groups,extra", [(1, 40000, 64, 1, 0), (1, 25000, 96, 1, 1), (2, 3000, 301, 1, 0), (1, 30, 4096, 2, 0), (2, 1500, 22, 2, 0),
                                                 (2, 1500, 22, 1, 4), (8, 20, 64, 8, 0), (5, 64, 24, 3, 0), (9, 700, 32, 4, 0), (1, 9, 32, 2, 0),
                                                 (1, 6000, 256, 1, 0), (3, 4000, 24, 8, 0), (2, 12544, 64, 16, 0)])
def test_groups_of_every_size(n, hw, c, groups, extra, name):
    """Groups that stay on one SM, on a cluster's, on none; pairs of channels; samples that share a cluster and that do not."""
    x, dy, gamma, beta = make(n, hw, c, extra, name, n * 37 + hw * 7 + c)
    for kept in ("input", "codes"):
        check(x, dy, gamma, beta, c, groups, name, "silu", kept)


@pytest.mark.parametrize("kind", ["none", "relu"])
@pytest.mark.parametrize("n,hw,c,groups,extra", [(2, 50, 64, 8, 0), (3, 45, 120, 8, 24), (2, 61, 35, 5, 3), (1, 12000, 64, 32, 0)])
def test_activations_and_missing_parameters(n, hw, c, groups, extra, kind):
    x, dy, gamma, beta = make(n, hw, c, extra, "bf16", 5 + c)
    check(x, dy, gamma, beta, c, groups, "bf16", kind, "codes")
    check(x, dy, None, beta, c, groups, "bf16", kind, "input")
    check(x, dy, gamma, None, c, groups, "bf16", kind, "input")
    got, bare = (call(x, dy, gamma, beta, c, groups, "bf16", kind, "input", want=w) for w in (True, False))
    assert torch.equal(got["dx"], bare["dx"])


@pytest.mark.parametrize("hw,c,groups", [(400, 64, 8), (3000, 24, 3), (30, 33, 3)])
def test_means_far_from_zero_cost_no_digits(hw, c, groups):
    """The spread is a thousandth of the mean, and a border of zeros-like values comes first: raw squares would lose every digit."""
    x, dy, gamma, beta = make(2, hw, c, 0, "fp32", 9, mean=1000.0, spread=1.0)
    x = 1000.0 + (x - x.mean((0, 1), keepdim=True)) * 1.0
    check(x, dy, gamma, beta, c, groups, "fp32", "silu", "input")
    x[:, :5] = 0.0
    check(x, dy, gamma, beta, c, groups, "fp32", "none", "input")


def test_a_constant_group_and_eps():
    x, dy, gamma, beta = make(2, 30, 32, 0, "fp32", 11)
    x[0, :, :8] = 3.25
    got = check(x, dy, gamma, beta, 32, 4, "fp32", "none", "input", eps=1e-3)
    assert np.array_equal(wide(got["y"])[0, :, :8], np.broadcast_to(beta[:8].astype(np.float64), (30, 8)))


def test_nan_and_infinity_stay_in_their_group():
    n, hw, c, groups = 3, 70, 64, 8
    x, dy, gamma, beta = make(n, hw, c, 0, "fp16", 13)
    clean = call(x, dy, gamma, beta, c, groups, "fp16", "silu", "input")
    x[0, 11, 5], x[2, 69, 60] = float("nan"), float("inf")
    got = call(x, dy, gamma, beta, c, groups, "fp16", "silu", "input")
    hit = np.zeros((n, hw, c), bool)
    hit[0, :, 0:8] = hit[2, :, 56:64] = True
    for k in ("y", "dx"):
        v, w = wide(got[k]), wide(clean[k])
        assert np.isnan(v[hit]).all() and np.array_equal(v[~hit], w[~hit])
    assert np.isnan(wide(got["dgamma"])[:8]).all() and np.isfinite(wide(got["dgamma"])[8:56]).all()
    # ReLU lets a NaN through as well
    assert np.isnan(wide(call(x, dy, gamma, beta, c, groups, "fp16", "relu", "input")["y"])[hit]).all()
    G.status_clear()
    call(x, dy, gamma, beta, c, groups, "fp16", "silu", "codes")
    assert G.status_clear() == eoq.EOQ_DEV_NONFINITE


@pytest.mark.parametrize("name", sorted(TYPES))
def test_large_and_tiny_values(name):
    """Gates far out on both sides, and values whose squares leave the type."""
    x, dy, gamma, beta = make(2, 64, 48, 0, name, 17)
    check(x, dy, gamma * 40, beta * 10, 48, 6, name, "silu", "codes")
    big = {"fp32": 1e15, "fp16": 5000.0, "bf16": 1e15}[name]
    check((x * big).to(x.dtype), dy, gamma, beta, 48, 6, name, "silu", "codes")


@pytest.mark.parametrize("kept", ["input", "codes"])
def test_the_same_bits_every_time_on_any_stream_and_replayed(kept):
    n, hw, c, groups = 4, 500, 96, 8
    x, dy, gamma, beta = make(n, hw, c, 0, "bf16", 19)
    d = eoq.gn_desc(n, hw, c, groups, eoq.EOQ_BF16, eoq.EOQ_ACT_SILU)
    g, b = G.dev(gamma), G.dev(beta)
    need = eoq.eoq_gn_workspace_size(d)

    def buffers():
        return {"y": torch.empty_like(x), "dx": torch.empty_like(x), "stats": G.zeros((n, groups, 2), torch.float32), "dg": G.zeros(c, torch.float32),
                "db": G.zeros(c, torch.float32), "ws": G.empty(need, torch.uint8), "codes": G.zeros((n, hw, c), torch.int8) if kept == "codes" else None,
                "exps": G.zeros((n * hw, 3), torch.uint8) if kept == "codes" else None}

    def step(o):
        eoq.eoq_gn_fwd(G.handle(), d, x, g, b, o["y"], o["stats"], o["codes"], o["exps"], o["ws"])
        eoq.eoq_gn_bwd(G.handle(), d, dy, None, None if kept == "codes" else x, o["codes"], o["exps"], g, b, o["stats"], o["dx"], o["dg"], o["db"], o["ws"])

    first, second, third = buffers(), buffers(), buffers()
    step(first)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(second)
    step(first)            # two calls on one handle at once, a workspace each
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(third)
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    for k in ("y", "dx", "stats", "dg", "db"):
        assert torch.equal(first[k], second[k]) and torch.equal(first[k], third[k]), k
    x.copy_(x.flip(1))
    graph.replay()
    torch.cuda.synchronize()
    R.within(wide(third["dg"]), wide(first["dg"]), 1e9)     # (runs on)
    assert not torch.equal(third["y"], first["y"])


@pytest.mark.parametrize("name", ["bf16", "fp32"])
def test_pairs_of_channels_with_the_eight_bit_form(name):
    """Rows that only pairs of elements are aligned in, and channels in whole blocks: the 8-bit form is written beside the output."""
    x, dy, gamma, beta = make(2, 50, 64, 2, name, 41)
    check(x, dy, gamma, beta, 64, 8, name, "silu", "codes")


@pytest.mark.parametrize("n", [3, 160])
@pytest.mark.parametrize("c,groups,name,kept", [(96, 16, "bf16", "codes"), (120, 8, "fp16", "input"), (40, 2, "fp16", "codes"), (24, 2, "fp32", "input")])
def test_groups_that_cut_vectors(n, c, groups, name, kept):
    """Groups that are no whole vectors, in few blocks and in many: the width of the vectors goes by both."""
    x, dy, gamma, beta = make(n, 65, c, 0, name, 47)
    check(x, dy, gamma, beta, c, groups, name, "silu", kept)


def test_addresses_beyond_32_bits():
    """Pixels 2^30 elements apart: the last ones lie beyond 2^32 elements."""
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB of free device memory")
    hw, c, groups, stride = 6, 64, 8, 1 << 30
    rng = np.random.default_rng(43)
    big = torch.empty(5 * stride + c, dtype=torch.bfloat16, device="cuda:0")
    x = torch.as_strided(big, (hw, c), (stride, 1))
    x.copy_(torch.from_numpy(rng.normal(size=(hw, c))))
    dy = torch.from_numpy(rng.normal(size=(hw, c))).bfloat16().to("cuda:0")
    d = eoq.gn_desc(1, hw, c, groups, eoq.EOQ_BF16, eoq.EOQ_ACT_SILU, x_stride=stride)
    flat = eoq.gn_desc(1, hw, c, groups, eoq.EOQ_BF16, eoq.EOQ_ACT_SILU)
    got = []
    for desc, src in ((d, x), (flat, x.contiguous())):
        o = {k: torch.empty(hw, c, dtype=torch.bfloat16, device="cuda:0") for k in ("y", "dx")}
        o["stats"], o["dg"], o["db"] = G.zeros((1, groups, 2), torch.float32), G.zeros(c, torch.float32), G.zeros(c, torch.float32)
        ws = G.empty(eoq.eoq_gn_workspace_size(desc), torch.uint8)
        eoq.eoq_gn_fwd(G.handle(), desc, src, None, None, o["y"], o["stats"], None, None, ws)
        eoq.eoq_gn_bwd(G.handle(), desc, dy, None, src, None, None, None, None, o["stats"], o["dx"], o["dg"], o["db"], ws)
        got.append(o)
    torch.cuda.synchronize()
    for k in got[0]:
        assert torch.equal(got[0][k], got[1][k]), k


def test_directional_derivative():
    """<gradient, direction> against differences of the GPU's own forward pass.  Central differences are off by h^2 / 6 of the third
    derivative and by the forward pass's rounding over h: with h = 2^-6, u of order one and 2,000 terms summed in 64 bits, well under 1%."""
    n, hw, c, groups = 2, 40, 24, 3
    x, dy, gamma, beta = make(n, hw, c, 0, "fp32", 23)
    got = call(x, dy, gamma, beta, c, groups, "fp32", "silu", "input")
    way = torch.from_numpy(np.random.default_rng(1).normal(size=x.shape)).float().to("cuda:0") * dy.sign() * 0.1
    h = 2.0 ** -6
    up, down = (wide(call(x + s * h * way, dy, gamma, beta, c, groups, "fp32", "silu", "input")["y"]) for s in (1, -1))
    num = ((up - down) * wide(dy)).sum() / (2 * h)
    ana = (wide(got["dx"]) * wide(way)).sum()
    assert abs(num - ana) < 0.01 * (np.abs(wide(got["dx"]) * wide(way)).sum())


@pytest.mark.parametrize("kept", ["input", "codes"])
@pytest.mark.parametrize("n,hw,c,groups", [(2, 64, 64, 8), (3, 35, 48, 3), (1, 20, 30, 5)])
def test_integer_sums(n, hw, c, groups, kept):
    """int32 sums in, Q_a2 codes out; int8 errors with an exponent in device memory in, fp32 out."""
    rng = np.random.default_rng(29 + c)
    acc = rng.integers(-40000, 60000, (n, hw, c)).astype(np.int32)
    e = np.clip(np.rint(rng.normal(0, 32, (n, hw, c))), -127, 127).astype(np.int8)
    gamma, beta = rng.normal(0.5, 0.1, c).astype(np.float32), rng.normal(0, 0.1, c).astype(np.float32)
    d = eoq.gn_desc(n, hw, c, groups, eoq.EOQ_I32, eoq.EOQ_ACT_SILU, x_exp=-14)
    ws = G.empty(eoq.eoq_gn_workspace_size(d), torch.uint8)
    accd, ed, ee = G.dev(acc), G.dev(e), G.dev(np.array([-12], np.int32))
    y, dx = G.zeros((n, hw, c), torch.int8), G.zeros((n, hw, c), torch.float32)
    stats, dg, db = G.zeros((n, groups, 2), torch.float32), G.zeros(c, torch.float32), G.zeros(c, torch.float32)
    codes = G.zeros((n, hw, c), torch.int8) if kept == "codes" else None
    exps = G.zeros((n * hw, -(-c // 32)), torch.uint8) if kept == "codes" else None
    g, b = G.dev(gamma), G.dev(beta)
    eoq.eoq_gn_fwd(G.handle(), d, accd, g, b, y, stats, codes, exps, ws)
    eoq.eoq_gn_bwd(G.handle(), d, ed, ee, None if codes is not None else accd, codes, exps, g, b, stats, dx, dg, db, ws)
    torch.cuda.synchronize()
    xw = acc.astype(np.float64) * 2.0 ** -14
    want, mean, rstd, bound = R.gn_fwd(xw, groups, 1e-5, gamma.astype(np.float64), beta.astype(np.float64), "silu")
    q = np.clip(want * 128, -127, 127)
    assert (np.abs(G.host(y) - q) <= 0.5 + 128 * bound).all()
    sw = wide(stats)
    if kept == "codes":
        wc, we, back = R.block_form(xw.reshape(-1, c))
        assert np.array_equal(G.host(codes).reshape(-1, c), wc) and np.array_equal(G.host(exps), we)
        xw = back.reshape(xw.shape)
    r = R.gn_bwd(e.astype(np.float64) * 2.0 ** -12, xw, sw[..., 0], sw[..., 1], gamma.astype(np.float64), beta.astype(np.float64), "silu")
    R.within(wide(dx), r[0], r[3])
    R.within(wide(dg), r[1], r[4])
    R.within(wide(db), r[2], r[5])
    assert G.status_clear() == 0
    eoq.eoq_gn_bwd(G.handle(), d, ed, G.dev(np.array([121], np.int32)), accd, None, None, g, b, stats, dx, dg, db, ws)
    assert G.status_clear() == eoq.EOQ_DEV_RANGE


def test_behind_a_convolution_and_back():
    """As a network uses it: convolution, group norm on its exact sums with their 8-bit form kept, the codes into the next convolution; back
    through Q_e of the normalisation's error into both passes of the convolution in front."""
    n, h, w, ci, co, groups = 2, 10, 9, 32, 64, 8
    rng = np.random.default_rng(31)
    x0 = G.dev(rng.integers(-100, 100, (n, h, w, ci)).astype(np.int8))
    wt = G.dev(rng.integers(-30, 30, (co, 3, 3, ci)).astype(np.int8))
    gd = eoq.conv_desc(n, h, w, ci, co, 3, 3, 1, 1)
    hd = G.handle()
    x5, acc = G.zeros((n, h, w, co), torch.int8), G.zeros((n, h, w, co), torch.int32)
    eoq.eoq_conv_fwd(hd, gd, x0, None, 0, wt, 128, 0, None, True, x5, None, None, acc, G.workspace(gd, eoq.EOQ_PASS_FWD))
    d = eoq.gn_desc(n, h * w, co, groups, eoq.EOQ_I32, eoq.EOQ_ACT_RELU, x_exp=-14)
    ws = G.empty(eoq.eoq_gn_workspace_size(d), torch.uint8)
    gamma, beta = G.dev(np.full(co, 0.4, np.float32)), G.dev(np.full(co, 0.05, np.float32))
    y, stats = G.zeros((n, h, w, co), torch.int8), G.zeros((n, groups, 2), torch.float32)
    codes, exps = G.zeros((n, h, w, co), torch.int8), G.zeros((n * h * w, co // 32), torch.uint8)
    eoq.eoq_gn_fwd(hd, d, acc, gamma, beta, y, stats, codes, exps, ws)
    kept = acc.clone()
    acc.zero_()                                                    # the sums need not stay
    e, ee = G.dev(np.clip(np.rint(rng.normal(0, 32, (n, h, w, co))), -127, 127).astype(np.int8)), G.dev(np.array([-12], np.int32))
    da, dg, db = G.zeros((n, h, w, co), torch.float32), G.zeros(co, torch.float32), G.zeros(co, torch.float32)
    eoq.eoq_gn_bwd(hd, d, e, ee, None, codes, exps, gamma, beta, stats, da, dg, db, ws)
    e3, e3x = G.zeros((n, h, w, co), torch.int8), G.zeros(1, torch.int32)
    eoq.eoq_quantize(hd, eoq.EOQ_SQ, da, True, None, da.numel(), e3, e3x)
    g, gx = G.zeros((co, 3, 3, ci), torch.int8), G.zeros(1, torch.int32)
    eoq.eoq_conv_wgrad(hd, gd, e3, e3x, x0, 0, g, gx, None, G.workspace(gd, eoq.EOQ_PASS_WGRAD))
    torch.cuda.synchronize()
    assert G.status_clear() == 0
    # the same in 64 bits, with the values the 8-bit form stands for
    xw = wide(kept).reshape(n, h * w, co) * 2.0 ** -14
    mean, rstd = R.gn_stats(xw, groups, 1e-5)
    back = R.block_form(xw.reshape(-1, co))[2].reshape(xw.shape)
    ga, be = np.full(co, np.float64(np.float32(0.4))), np.full(co, np.float64(np.float32(0.05)))
    dx = R.gn_bwd(wide(e).reshape(n, h * w, co) * 2.0 ** -12, back, mean, rstd, ga, be, "relu")[0]
    scale = np.abs(dx).max()
    gated = np.abs(ga * (back - R._wide(mean, co)) * R._wide(rstd, co) + be) > 1e-5
    assert (np.abs(wide(da).reshape(dx.shape) - dx)[gated] < 1e-4 * scale).all()
    # weight gradient: that of the error rounded to 127 steps, in the direction of the exact one
    p = np.lib.stride_tricks.sliding_window_view(np.pad(wide(x0), ((0, 0), (1, 1), (1, 1), (0, 0))), (3, 3), (1, 2))
    gw = np.einsum("nhwo,nhwcyx->oyxc", dx.reshape(n, h, w, co), p)
    got = wide(g)
    cos = (gw * got).sum() / np.sqrt((gw ** 2).sum() * (got ** 2).sum())
    assert cos > 0.99 and got.any()
