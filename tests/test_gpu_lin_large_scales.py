"""Forward passes of tokens whose scales are far from one: the sum times a token's scale may be beyond what an fp32 number holds, the output is not."""
import pytest
import torch

import lin_reference as ref
from gpu_util import status_clear
from paper_2105_13890_b200 import build, eoq
from test_gpu_lin import Layer, handle

build.build_lib()
pytestmark = pytest.mark.gpu
DEV = "cuda:0"
# a few tokens; single blocks of 32, 64 and 128 columns, pairs; sums in parts, joined in 32 and in 64 bits
SIZES = [(3, 40, 50), (8, 2048, 40), (1, 4096, 70), (40, 70, 33), (33, 4096, 40), (60, 300, 200), (300, 384, 257), (1000, 40, 33), (700, 512, 600), (700, 8200, 300), (6, 140000, 64),
         (2500, 100, 1000), (3000, 200, 512), (5000, 600, 500)]
TOPS = [3e38, 1e36, 1e33, 2.0 ** 100, 2.0 ** 99.5, 1e29, 1e15, 1.0, 1e-20, 1e-36]      # (2^93 is the scale from which tokens are large: magnitudes of 2^100)


def large(rows, c_in, c_out, dtype, bias=True):
    """Tokens of all sizes, channels of several that bring the outputs back among the numbers."""
    l = Layer(rows, c_in, c_out, dtype, bias)
    top = torch.tensor(TOPS, device=DEV)[torch.arange(rows, device=DEV) % len(TOPS)]
    x = l.x.float()
    l.x.copy_(x / x.abs().amax(1, keepdim=True) * top[:, None])
    small = torch.tensor([1e-3, 1e-10, 1e-30], device=DEV)[torch.arange(c_out, device=DEV) % 3]
    l.w.copy_(l.w / l.w.abs().amax(1, keepdim=True) * small[:, None] / c_in)
    l.code_weights()
    return l


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
@pytest.mark.parametrize("rows,c_in,c_out", SIZES)
def test_outputs_are_numbers(rows, c_in, c_out, dtype):
    l = large(rows, c_in, c_out, dtype)
    status_clear()
    l.forward(keep=False)
    assert status_clear() == 0 and bool(torch.isfinite(l.y).all())
    l.check_forward()
    y = l.y.clone()
    l.forward()
    l.check_codes()
    assert torch.equal(l.y, y)
    eoq.eoq_lin_fwd(handle(), l.desc, None, l.x_codes, l.x_scales, l.w_codes, l.w_scales, l.bias, l.y, l.ws)
    assert torch.equal(l.y, y)


@pytest.mark.parametrize("rows,c_in,c_out", SIZES)
def test_sums_of_zero(rows, c_in, c_out):
    """Nothing but the bias, however large the two scales are."""
    l = Layer(rows, c_in, c_out, torch.float32)
    l.x[:, 0], l.x[:, 1:] = 3e38, 0.0
    l.w[:, 0], l.w[:, 1:] = 0.0, 1e30
    l.code_weights()
    l.forward(keep=False)
    assert torch.equal(l.y, l.bias.expand(rows, c_out))


@pytest.mark.parametrize("rows,c_in,c_out", SIZES)
def test_outputs_that_no_number_holds(rows, c_in, c_out):
    """Infinities of the sums' signs; the rows beside them are as they should be."""
    l = Layer(rows, c_in, c_out, torch.float32)
    l.x[0] = 3e38
    l.w.copy_(l.w.abs())
    l.w[1::2] *= -1.0
    l.w.mul_(1000.0 / l.w.abs().amin(1, keepdim=True))
    l.code_weights()
    l.forward(keep=False)
    assert torch.equal(l.y[0].cpu(), torch.where(torch.arange(c_out) % 2 == 0, float("inf"), float("-inf")))
    y, bound = ref.forward(*l.oracle(), l.bias, torch.float32)
    ref.near(l.y[1:], y[1:], bound[1:], "y")


@pytest.mark.parametrize("c_in", [40, 2000])
def test_same_bits_whichever_kernel(c_in):
    whole = large(1200, c_in, 600, torch.float32)
    whole.forward(keep=False)
    for rows in (1, 8, 40, 130, 700):
        l = Layer(rows, c_in, 600, torch.float32)
        l.x.copy_(whole.x[:rows])
        eoq.eoq_lin_fwd(handle(), l.desc, l.x, None, None, whole.w_codes, whole.w_scales, whole.bias, l.y, l.ws)
        assert torch.equal(l.y, whole.y[:rows])
