"""Weight gradients from errors and the 8-bit form of the input (eoq_ckpt_wgrad) against sums in 64 bits."""
import itertools

import numpy as np
import pytest
import torch

from paper_2105_13890_b200 import eoq

import gpu_util as G
import wide_reference as R

pytestmark = pytest.mark.gpu

TYPES = {"fp32": (torch.float32, eoq.EOQ_F32, 3), "fp16": (torch.float16, eoq.EOQ_F16, 2), "bf16": (torch.bfloat16, eoq.EOQ_BF16, 1)}


def make(rows, c_out, c_in, name, seed, extra=0):
    rng = np.random.default_rng(seed)
    dy = torch.from_numpy(rng.normal(0, 0.1, (rows, c_out + extra))).to(TYPES[name][0]).to("cuda:0")
    codes, exps, back = R.block_form(rng.normal(size=(rows, c_in)) * np.exp(rng.normal(0, 1.5, (rows, 1))))
    return dy, codes, exps, back


def call(dy, codes, exps, name, c_out):
    rows, c_in = codes.shape
    need = eoq.eoq_ckpt_wgrad_workspace_size(rows, c_out, c_in, TYPES[name][1])
    ws = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device="cuda:0")
    raw = torch.full((c_out * c_in + 64,), 33.0, device="cuda:0")
    eoq.eoq_ckpt_wgrad(G.handle(), dy, TYPES[name][1], rows, c_out, dy.shape[1], G.dev(codes), G.dev(exps), c_in, raw, ws[:need] if need else None)
    torch.cuda.synchronize()
    assert (raw[c_out * c_in:] == 33).all() and (ws[need:] == 0xFF).all()
    assert G.status_clear() == 0
    return raw[:c_out * c_in].view(c_out, c_in)


def check(dy, codes, exps, back, name, c_out):
    """Products are exact; each step of 16 rows (of each part of dy) is one addition of fp32, and so is joining a split (at most 148): off by at
    most a whole step of the sum of magnitudes, and the 16 products of a step are added among one another with as much."""
    got = call(dy, codes, exps, name, c_out).double().cpu().numpy()
    d = dy[:, :c_out].double().cpu().numpy()
    rows = codes.shape[0]
    room = (2 * TYPES[name][2] * (-(-rows // 16)) + 148) * 2.0 ** -23 * (np.abs(d).T @ np.abs(back))
    R.within(got, d.T @ back, room)
    return got


@pytest.mark.parametrize("name", sorted(TYPES))
@pytest.mark.parametrize("rows,c_out,c_in,extra", [(1, 8, 16, 0), (1, 1, 1, 0), (5, 3, 7, 0), (64, 128, 64, 0), (63, 128, 128, 0), (200, 256, 256, 0),
                                                   (65, 136, 272, 0), (300, 40, 48, 24), (1000, 100, 50, 1), (129, 17, 300, 0), (2000, 64, 64, 8),
                                                   (4096, 16, 16, 0), (777, 130, 520, 2), (130, 1032, 33, 0), (20000, 24, 96, 0)])
def test_shapes_and_types(rows, c_out, c_in, extra, name):
    check(*make(rows, c_out, c_in, name, rows + c_in, extra), name, c_out)


@pytest.mark.parametrize("name", sorted(TYPES))
@pytest.mark.parametrize("rows,c_out,c_in", [(1, 136, 144), (64, 256, 256), (1000, 264, 528), (5000, 512, 272), (2500, 1024, 256), (9000, 136, 1040)])
def test_tiles_of_two_blocks(rows, c_out, c_in, name):
    """More than 128 columns on both sides: in bf16, blocks work in pairs; ends inside either block's half; sums that move on."""
    check(*make(rows, c_out, c_in, name, rows + c_in), name, c_out)


@pytest.mark.parametrize("rows,c_out,c_in", [(3000, 3, 7), (9000, 33, 31), (700, 1, 5)])
def test_splits_of_odd_matrices(rows, c_out, c_in):
    """Several splits of a matrix whose elements are no multiple of four."""
    assert c_out * c_in % 4 and eoq.eoq_ckpt_wgrad_workspace_size(rows, c_out, c_in, eoq.EOQ_F16) > 0
    check(*make(rows, c_out, c_in, "fp16", rows), "fp16", c_out)


def test_every_operand_has_its_place():
    """One row at a time against the outer product: exact, so that a swapped row, column or part shows."""
    for name, c_out in itertools.product(sorted(TYPES), (128, 256)):
        for row in (0, 1, 7, 8, 15, 16, 63, 64, 100):
            dy, codes, exps, back = make(101, c_out, 256, name, 7)
            keep = torch.zeros_like(dy)
            keep[row] = dy[row]
            got = call(keep, codes, exps, name, c_out).double().cpu().numpy()
            want = np.outer(keep[row].double().cpu().numpy(), back[row])
            # three parts are added in two roundings; with one or two parts the last of them rounds
            R.within(got, want, {"bf16": 0, "fp16": 2.0 ** -23, "fp32": 2.0 ** -22}[name] * np.abs(want))


@pytest.mark.parametrize("name", sorted(TYPES))
def test_nan_infinity_and_marked_blocks(name):
    rows, c_out, c_in = 150, 64, 96
    dy, codes, exps, back = make(rows, c_out, c_in, name, 3)
    dy[10, 3], dy[20, 5] = float("nan"), float("inf")
    codes[20, codes[20] == 0] = 1                     # (0 * infinity is a NaN of its own)
    back = np.repeat(2.0 ** (exps.astype(float) - 127), 32, 1)[:, :c_in] * codes
    clean = call(torch.where(torch.isfinite(dy), dy, torch.zeros_like(dy)), codes, exps, name, c_out).cpu().numpy()
    exps[70, 2], codes[70, 64:] = 255, 0
    got = call(dy, codes, exps, name, c_out).cpu().numpy()
    assert np.isnan(got[:, 64:]).all() and np.isnan(got[3]).all()
    assert np.array_equal(got[5, :64], np.copysign(np.inf, back[20, :64]).astype(np.float32))
    others = [o for o in range(c_out) if o not in (3, 5)]
    assert np.array_equal(got[others, :64], clean[others, :64])


def test_range_of_the_steps():
    """Blocks from the smallest step to the largest values; dy at the ends of its range."""
    rows, c_out, c_in = 64, 64, 64
    rng = np.random.default_rng(5)
    codes = rng.integers(-127, 128, (rows, c_in)).astype(np.int8)
    exps = np.zeros((rows, 2), np.uint8)
    exps[:, 0], exps[:, 1] = 1, 120
    back = np.repeat(2.0 ** (exps.astype(float) - 127), 32, 1) * codes
    for name, big in (("bf16", 2.0 ** 100), ("fp32", 2.0 ** 100), ("fp16", 60000.0)):
        dy = torch.from_numpy(rng.normal(size=(rows, c_out)) * big / 8).to(TYPES[name][0]).to("cuda:0")
        check(dy, codes, np.full_like(exps, 120) if name == "fp16" else exps, codes * 2.0 ** -7 if name == "fp16" else back, name, c_out)
    tiny = torch.from_numpy(rng.integers(-3, 4, (rows, c_out)) * 2.0 ** -24).half().to("cuda:0")      # the smallest fp16 numbers
    check(tiny, codes, np.full_like(exps, 127), codes.astype(np.float64), "fp16", c_out)


@pytest.mark.parametrize("name", ["bf16", "fp16"])
def test_addresses_beyond_32_bits(name):
    """Rows of errors 2^30 elements apart."""
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB of free device memory")
    rows, c_out, c_in, stride = 6, 136, 144, 1 << 30
    dy, codes, exps, back = make(rows, c_out, c_in, name, 43)
    big = torch.empty(5 * stride + c_out, dtype=dy.dtype, device="cuda:0")
    far = torch.as_strided(big, (rows, c_out), (stride, 1))
    far.copy_(dy)
    out = G.zeros((c_out, c_in), torch.float32)
    ws = G.empty(max(eoq.eoq_ckpt_wgrad_workspace_size(rows, c_out, c_in, TYPES[name][1]), 256), torch.uint8)
    eoq.eoq_ckpt_wgrad(G.handle(), far, TYPES[name][1], rows, c_out, stride, G.dev(codes), G.dev(exps), c_in, out, ws)
    torch.cuda.synchronize()
    assert torch.equal(out, call(dy, codes, exps, name, c_out))


def test_two_calls_at_once():
    """Two streams, one handle, a workspace each: nothing of one call reaches the other."""
    a, b = make(5000, 256, 272, "bf16", 51), make(4000, 130, 65, "fp16", 52)
    want = [call(dy, codes, exps, name, dy.shape[1]) for (dy, codes, exps, _), name in ((a, "bf16"), (b, "fp16"))]
    jobs = []
    for (dy, codes, exps, _), name in ((a, "bf16"), (b, "fp16")):
        c_out, c_in = dy.shape[1], codes.shape[1]
        jobs.append((dy, name, c_out, G.dev(codes), G.dev(exps), c_in, G.zeros((c_out, c_in), torch.float32),
                     G.empty(eoq.eoq_ckpt_wgrad_workspace_size(dy.shape[0], c_out, c_in, TYPES[name][1]), torch.uint8), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(20):
        for dy, name, c_out, codes, exps, c_in, out, ws, stream in jobs:
            with torch.cuda.stream(stream):
                eoq.eoq_ckpt_wgrad(G.handle(), dy, TYPES[name][1], dy.shape[0], c_out, c_out, codes, exps, c_in, out, ws)
    torch.cuda.synchronize()
    for job, w in zip(jobs, want):
        assert torch.equal(job[6], w)


def test_the_same_bits_every_time_and_replayed():
    rows, c_out, c_in = 3000, 192, 160
    dy, codes, exps, _ = make(rows, c_out, c_in, "bf16", 11)
    first = call(dy, codes, exps, "bf16", c_out)
    cd, ed, ws = G.dev(codes), G.dev(exps), G.empty(eoq.eoq_ckpt_wgrad_workspace_size(rows, c_out, c_in, eoq.EOQ_BF16), torch.uint8)
    out = G.zeros((c_out, c_in), torch.float32)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        eoq.eoq_ckpt_wgrad(G.handle(), dy, eoq.EOQ_BF16, rows, c_out, c_out, cd, ed, c_in, out, ws)
    for _ in range(3):
        ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, first)
    dy.mul_(2)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, 2 * first)


def test_a_layer_behind_a_normalisation():
    """As a step uses them: normalise, put the output away, gradient of the 1x1 convolution behind it from what was put away."""
    n, hw, c, c_out = 2, 49, 96, 64
    g = torch.Generator(device="cuda:0").manual_seed(3)
    x = torch.randn(n, hw, c, device="cuda:0", generator=g).bfloat16()
    d = eoq.gn_desc(n, hw, c, 8, eoq.EOQ_BF16, eoq.EOQ_ACT_SILU)
    y = torch.empty_like(x)
    hd = G.handle()
    eoq.eoq_gn_fwd(hd, d, x, None, None, y, None, None, None, G.empty(eoq.eoq_gn_workspace_size(d), torch.uint8))
    codes, exps = G.zeros((n * hw, c), torch.int8), G.zeros((n * hw, 3), torch.uint8)
    eoq.eoq_ckpt_save(hd, y, eoq.EOQ_BF16, 0, n * hw, c, c, codes, exps)
    torch.cuda.synchronize()
    kept = R.block_form(y.double().cpu().numpy().reshape(-1, c))
    y.zero_()
    dy = (0.1 * torch.randn(n * hw, c_out, device="cuda:0", generator=g)).bfloat16()
    dw = G.zeros((c_out, c), torch.float32)
    ws = G.empty(max(eoq.eoq_ckpt_wgrad_workspace_size(n * hw, c_out, c, eoq.EOQ_BF16), 256), torch.uint8)
    eoq.eoq_ckpt_wgrad(hd, dy, eoq.EOQ_BF16, n * hw, c_out, c_out, codes, exps, c, dw, ws)
    torch.cuda.synchronize()
    assert np.array_equal(G.host(codes), kept[0]) and np.array_equal(G.host(exps), kept[1])
    d64 = dy.double().cpu().numpy()
    R.within(dw.double().cpu().numpy(), d64.T @ kept[2], 200 * 2.0 ** -23 * (np.abs(d64).T @ np.abs(kept[2])))
