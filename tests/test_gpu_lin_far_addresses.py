"""Integer linear layers and gradients whose tensors, codes and rows lie beyond 32 bits of bytes or elements; the ends are compared."""
import pytest
import torch

import lin_reference as ref
from gpu_util import handle, status_clear
from paper_2105_13890_b200 import build, eoq
from test_gpu_grad import NORM
from test_gpu_lin import DEV

build.build_lib()
pytestmark = pytest.mark.gpu
ROWS, WIDE, NARROW, END = 33_001, 66_000, 48, 40      # 2.18 G elements


def test_forward_of_long_rows():
    """Tokens, and their codes, of more than 2^31 bytes."""
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    x = torch.empty(ROWS, WIDE, dtype=torch.bfloat16, device=DEV).normal_(generator=g)
    w = torch.randn(NARROW, WIDE, generator=g, device=DEV)
    desc = eoq.lin_desc(ROWS, WIDE, NARROW, eoq.EOQ_BF16)
    pitch = eoq.lin_pitch(WIDE)
    w_codes, w_scales = torch.empty(NARROW, pitch, dtype=torch.int8, device=DEV), torch.empty(NARROW, device=DEV)
    x_codes, x_scales = torch.empty(ROWS, pitch, dtype=torch.int8, device=DEV), torch.empty(ROWS, device=DEV)
    y = torch.empty(ROWS, NARROW, dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(eoq.eoq_lin_workspace_size(desc, eoq.EOQ_LIN_FWD), dtype=torch.uint8, device=DEV)
    status_clear()
    eoq.eoq_lin_quantize(handle(), w, eoq.EOQ_F32, NARROW, WIDE, WIDE, w_codes, w_scales)
    eoq.eoq_lin_fwd(handle(), desc, x, x_codes, x_scales, w_codes, w_scales, None, y, ws)
    assert status_clear() == 0
    wc, wsc = ref.codes_of(w)
    for at in (slice(0, END), slice(ROWS - END, ROWS)):
        codes, scales = ref.codes_of(x[at])
        assert torch.equal(x_codes[at, :WIDE].double(), codes) and torch.equal(x_scales[at].double(), scales)
        want, bound = ref.forward(codes, scales, wc, wsc, None, torch.bfloat16)
        ref.near(y[at], want, bound, "y")


def test_step_of_a_wide_output():
    """Outputs and errors, and both of their codes, of more than 2^31 bytes."""
    g = torch.Generator(device=DEV)
    g.manual_seed(2)
    x = torch.randn(ROWS, NARROW, generator=g, device=DEV).half()
    w = torch.randn(WIDE, NARROW, generator=g, device=DEV)
    desc = eoq.lin_desc(ROWS, NARROW, WIDE, eoq.EOQ_F16)
    w_codes, w_scales = torch.empty(WIDE, NARROW, dtype=torch.int8, device=DEV), torch.empty(WIDE, device=DEV)
    x_codes, x_scales = torch.empty(ROWS, NARROW, dtype=torch.int8, device=DEV), torch.empty(ROWS, device=DEV)
    ws = torch.empty(max(eoq.eoq_lin_workspace_size(desc, k) for k in (eoq.EOQ_LIN_FWD, eoq.EOQ_LIN_BWD)), dtype=torch.uint8, device=DEV)
    y = torch.empty(ROWS, WIDE, dtype=torch.float16, device=DEV)
    status_clear()
    eoq.eoq_lin_quantize(handle(), w, eoq.EOQ_F32, WIDE, NARROW, NARROW, w_codes, w_scales)
    eoq.eoq_lin_fwd(handle(), desc, x, x_codes, x_scales, w_codes, w_scales, None, y, ws)
    xc, xs = ref.codes_of(x)
    wc, wsc = ref.codes_of(w)
    for at in (slice(0, END), slice(ROWS - END, ROWS)):
        want, bound = ref.forward(xc[at], xs[at], wc, wsc, None, torch.float16)
        ref.near(y[at], want, bound, "y")
    dy = y.normal_(generator=g)
    dx, dw, db = torch.empty(ROWS, NARROW, dtype=torch.float16, device=DEV), torch.empty(WIDE, NARROW, device=DEV), torch.empty(WIDE, device=DEV)
    eoq.eoq_lin_bwd(handle(), desc, dy, x_codes, x_scales, w_codes, w_scales, dx, dw, db, ws)
    assert status_clear() == 0
    for at in (slice(0, END), slice(ROWS - END, ROWS)):
        want = ref.backward(dy[at], xc[at], xs[at], wc, wsc, torch.float16)
        ref.near(dx[at], *want["dx"], "dx")
    for at in (slice(0, END), slice(WIDE - END, WIDE)):
        want = ref.backward(dy[:, at], xc, xs, wc[at], wsc[at], torch.float16)
        ref.near(dw[at], *want["dw"], "dw")
        ref.near(db[at], *want["db"], "db")


@pytest.mark.parametrize("dtype,size", [(torch.float16, (1 << 32) + 12_345), (torch.float32, (1 << 31) + 12_345)], ids=str)
def test_gradients_of_many_elements(dtype, size):
    """One tensor beyond 2^31 or 2^32 elements, from an odd address on, clipped in place; its first and last pieces are not whole."""
    flat = torch.zeros(size + 3, dtype=dtype, device=DEV)
    t = flat[3:]
    spots = torch.tensor([0, 1, 5000, (1 << 31) - 1, 1 << 31, size - 5000, size - 1], device=DEV)
    t[spots] = torch.arange(1, 8, device=DEV).to(dtype)
    flat[:3] = 9.0
    l = eoq.grad_list([t])
    ws, norm = torch.empty(eoq.eoq_grad_workspace_size(l), dtype=torch.uint8, device=DEV), torch.empty(1, device=DEV)
    whole = 140.0 ** 0.5
    status_clear()
    eoq.eoq_grad_norm(handle(), l, norm, ws)
    assert abs(float(norm) - whole) <= NORM * whole
    eoq.eoq_grad_clip(handle(), l, 1.0, norm, ws)
    assert status_clear() == 0
    want = torch.arange(1, 8, device=DEV).double() / whole
    # (two products and a norm in fp32, as in every clip)
    ref.near(t[spots], want, (8 * 2.0 ** -24 + ref.HALF[dtype]) * want)
    assert int(torch.count_nonzero(t)) == 7 and bool((flat[:3] == 9.0).all())
