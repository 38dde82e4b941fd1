"""Tensors put away in 8 bits and read back (eoq_ckpt_save, eoq_ckpt_load) against the definition, bit for bit."""
import numpy as np
import pytest
import torch

from paper_2105_13890_b200 import eoq

import gpu_util as G
import wide_reference as R

pytestmark = pytest.mark.gpu

TYPES = {"fp32": (torch.float32, eoq.EOQ_F32), "fp16": (torch.float16, eoq.EOQ_F16), "bf16": (torch.bfloat16, eoq.EOQ_BF16)}


def save(x, dtype, cols=None, stride=None, src_exp=0, offset=0):
    """x: device tensor [rows, stride]; the first `cols` columns are put away."""
    rows = x.shape[0]
    cols = cols or x.shape[1]
    raw = torch.full((rows * cols + 64,), 77, dtype=torch.int8, device="cuda:0")
    exps = torch.full((rows * -(-cols // 32) + 64,), 78, dtype=torch.uint8, device="cuda:0")
    codes = raw[offset:]
    eoq.eoq_ckpt_save(G.handle(), x, dtype, src_exp, rows, cols, stride or x.shape[1], codes, exps)
    torch.cuda.synchronize()
    assert (raw[:offset] == 77).all() and (raw[offset + rows * cols:] == 77).all() and (exps[rows * -(-cols // 32):] == 78).all()
    return codes[:rows * cols].view(rows, cols), exps[:rows * -(-cols // 32)].view(rows, -1)


def check(x, name, cols=None, offset=0):
    """x: float64 numpy [rows, stride] of values that the type holds"""
    td, ed = TYPES[name]
    xd = torch.from_numpy(x).to(td).to("cuda:0")
    cols = cols or x.shape[1]
    codes, exps = save(xd, ed, cols, offset=offset)
    want_codes, want_exps, back = R.block_form(xd[:, :cols].double().cpu().numpy())
    assert np.array_equal(G.host(exps), want_exps) and np.array_equal(G.host(codes), want_codes)
    for out, (to, eo) in TYPES.items():
        dst = torch.full(x.shape, 55.0, dtype=to, device="cuda:0")
        eoq.eoq_ckpt_load(G.handle(), codes, exps, x.shape[0], cols, dst, eo, x.shape[1])
        got = dst.double().cpu().numpy()
        assert (got[:, cols:] == 55).all()
        want = torch.from_numpy(np.clip(back, -65504, 65504) if out == "fp16" else back).to(to).double().numpy()
        assert np.array_equal(got[:, :cols], want, equal_nan=True), out
    return exps


@pytest.mark.parametrize("name", sorted(TYPES))
@pytest.mark.parametrize("rows,cols,stride,offset", [(1, 1, 1, 0), (1, 32, 32, 0), (3, 8, 8, 0), (7, 40, 40, 0), (5, 33, 37, 0), (257, 64, 64, 0), (300, 64, 64, 1),
                                                     (65, 1000, 1000, 0), (33, 1000, 1008, 0), (9, 4104, 4104, 0), (4, 2500, 2500, 3), (2100, 96, 96, 0),
                                                     (70000, 16, 16, 0)])
def test_matches_the_definition(rows, cols, stride, offset, name):
    rng = np.random.default_rng(rows * 7919 + cols)
    x = rng.normal(size=(rows, stride)) * np.exp(rng.normal(0, 2, (rows, 1)))
    check(x, name, cols, offset)
    assert G.status_clear() == 0


@pytest.mark.parametrize("name", sorted(TYPES))
@pytest.mark.parametrize("cols", [64, 45])
def test_borders_of_the_step(cols, name):
    """127 steps exactly, a little above, ties, zeros, the smallest and the largest numbers of the type."""
    tiny, top = {"fp32": (2.0 ** -149, float(np.finfo(np.float32).max)), "fp16": (2.0 ** -24, 65504.0), "bf16": (2.0 ** -133, 255 * 2.0 ** 120)}[name]
    rows = [[127.0, 1.0, 0.5, 1.5, 2.5, -127.0], [127.5, 1.0, -3.0], [128.0, 64.0, 63.5], [0.0, -0.0], [tiny, -tiny, tiny * 3], [top, -top, top / 2],
            [1.0, 127 / 128, 1 / 256], [2.0 ** -14, 2.0 ** -20], [top, tiny], [254.0, 127.0, 253.0]]
    x = np.zeros((len(rows), cols))
    for i, r in enumerate(rows):
        x[i, 32:32 + len(r)] = r
        x[i, 3] = r[0]
    check(x, name)
    assert G.status_clear() == 0


@pytest.mark.parametrize("name", sorted(TYPES))
@pytest.mark.parametrize("cols", [96, 70])
def test_infinities_and_nan_mark_their_block_alone(cols, name):
    x = np.random.default_rng(3).normal(size=(40, cols))
    x[3, 5], x[9, 40], x[12, 69], x[12, 64], x[20, 31] = np.nan, np.inf, -np.inf, 1.0, np.nan
    exps = G.host(check(x, name))
    assert (exps == 255).sum() == 4
    assert G.status_clear() == eoq.EOQ_DEV_NONFINITE and G.status_clear() == 0


def test_integer_sums():
    rng = np.random.default_rng(5)
    a = rng.integers(-2 ** 20, 2 ** 20, (90, 48)).astype(np.int32)
    a[0, 0], a[1, 1], a[2, 2] = 2 ** 31 - 1, -2 ** 31, 127 << 9
    codes, exps = save(G.dev(a), eoq.EOQ_I32, src_exp=-14)
    want_codes, want_exps, _ = R.block_form(a.astype(np.float32).astype(np.float64) * 2.0 ** -14)
    assert np.array_equal(G.host(codes), want_codes) and np.array_equal(G.host(exps), want_exps)


def test_addresses_beyond_32_bits():
    """The last rows of a tensor of more than 2^32 elements, told by their stride."""
    free, _ = torch.cuda.mem_get_info()
    if free < 24 << 30:
        pytest.skip("needs 24 GB of free device memory")
    rows, stride, cols = 4, (1 << 31) + 16, 64
    x = torch.empty(rows * stride, dtype=torch.bfloat16, device="cuda:0")
    v = torch.as_strided(x, (rows, cols), (stride, 1))
    v.copy_(torch.randn(rows, cols, device="cuda:0"))
    codes, exps = save(v, eoq.EOQ_BF16, stride=stride)
    want_codes, want_exps, back = R.block_form(v.double().cpu().numpy())
    assert np.array_equal(G.host(codes), want_codes) and np.array_equal(G.host(exps), want_exps)
    v.zero_()
    eoq.eoq_ckpt_load(G.handle(), codes, exps, rows, cols, v, eoq.EOQ_BF16, stride)
    assert np.array_equal(v.double().cpu().numpy(), back)


def test_captured_and_on_another_stream():
    x = torch.randn(512, 128, device="cuda:0")
    codes, exps, back = G.zeros((512, 128), torch.int8), G.zeros((512, 4), torch.uint8), G.zeros((512, 128), torch.float32)

    def step():
        eoq.eoq_ckpt_save(G.handle(), x, eoq.EOQ_F32, 0, 512, 128, 128, codes, exps)
        eoq.eoq_ckpt_load(G.handle(), codes, exps, 512, 128, back, eoq.EOQ_F32, 128)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (1, 2):
        x.copy_(torch.randn(512, 128, generator=torch.Generator().manual_seed(seed)).to("cuda:0"))
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(G.host(back), R.block_form(G.host(x))[2].astype(np.float32))
