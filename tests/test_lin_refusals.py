"""Calls of the integer linear layers and of the gradients' norm that are refused, told without a device: every check but the handle's comes before any device work."""
import ctypes

import pytest

from paper_2105_13890_b200 import build, eoq
from test_float_operator_refusals import A, At

build.build_lib()
ODD = At((1 << 12) + 1)


def desc(**k):
    v = {"rows": 9, "c_in": 40, "c_out": 24, "dtype": eoq.EOQ_BF16}
    v.update(k)
    return eoq.lin_desc(**v)


def quantize(src=A, dtype=eoq.EOQ_BF16, rows=3, cols=40, stride=40, codes=A, scales=A):
    return eoq.eoq_lin_quantize(0, src, dtype, rows, cols, stride, codes, scales, stream=0, check=False)


def fwd(d=None, x=A, x_codes=A, x_scales=A, w_codes=A, w_scales=A, bias=A, y=A, ws=A):
    return eoq.eoq_lin_fwd(0, d or desc(), x, x_codes, x_scales, w_codes, w_scales, bias, y, ws, stream=0, check=False)


def bwd(d=None, dy=A, x_codes=A, x_scales=A, w_codes=A, w_scales=A, dx=A, dw=A, dbias=A, ws=A):
    return eoq.eoq_lin_bwd(0, d or desc(), dy, x_codes, x_scales, w_codes, w_scales, dx, dw, dbias, ws, stream=0, check=False)


@pytest.mark.parametrize("change,status", [
    (dict(rows=0), eoq.EOQ_ERR_BAD_ARG), (dict(c_in=0), eoq.EOQ_ERR_BAD_ARG), (dict(c_out=-4), eoq.EOQ_ERR_BAD_ARG), (dict(dtype=eoq.EOQ_I32), eoq.EOQ_ERR_BAD_ARG),
    (dict(dtype=-1), eoq.EOQ_ERR_BAD_ARG), (dict(x_stride=39), eoq.EOQ_ERR_BAD_ARG), (dict(y_stride=23), eoq.EOQ_ERR_BAD_ARG), (dict(dy_stride=1), eoq.EOQ_ERR_BAD_ARG),
    (dict(dx_stride=39), eoq.EOQ_ERR_BAD_ARG), (dict(rows=(1 << 30) + 1), eoq.EOQ_ERR_UNSUPPORTED), (dict(c_in=(1 << 20) + 1), eoq.EOQ_ERR_UNSUPPORTED),
    (dict(c_out=(1 << 20) + 1), eoq.EOQ_ERR_UNSUPPORTED), (dict(rows=1 << 30, c_in=1025), eoq.EOQ_ERR_UNSUPPORTED), (dict(rows=1 << 30, c_out=1025), eoq.EOQ_ERR_UNSUPPORTED),
    (dict(c_in=1 << 20, c_out=(1 << 14) + 1), eoq.EOQ_ERR_UNSUPPORTED), (dict(x_stride=(1 << 30) + 1), eoq.EOQ_ERR_UNSUPPORTED)])
def test_descriptors(change, status):
    d = desc(**change)
    assert fwd(d) == status and bwd(d) == status
    for which in (eoq.EOQ_LIN_FWD, eoq.EOQ_LIN_BWD):
        with pytest.raises(eoq.EoqError) as e:
            eoq.eoq_lin_workspace_size(d, which)
        assert e.value.status == status


def test_sizes_that_no_field_holds():
    for k in (dict(rows=-1), dict(rows=1 << 64), dict(c_in=1 << 31), dict(x_stride=1 << 64)):
        with pytest.raises(OverflowError):
            desc(**k)
    with pytest.raises(OverflowError):
        quantize(cols=1 << 32)
    with pytest.raises(eoq.EoqError) as e:
        eoq.eoq_lin_workspace_size(desc(), 2)
    assert e.value.status == eoq.EOQ_ERR_BAD_ARG
    with pytest.raises(TypeError):
        fwd(eoq.conv_desc(1, 8, 8, 16, 16, 3, 3))


def test_quantize():
    assert quantize() == eoq.EOQ_ERR_BAD_ARG          # all is well but the handle
    for k in (dict(src=None), dict(codes=None), dict(scales=None), dict(rows=0), dict(cols=0), dict(cols=-1), dict(stride=39), dict(dtype=eoq.EOQ_I32), dict(dtype=9)):
        assert quantize(**k) == eoq.EOQ_ERR_BAD_ARG
    for k in (dict(rows=(1 << 30) + 1), dict(cols=(1 << 20) + 1, stride=1 << 21), dict(stride=(1 << 30) + 1), dict(rows=-1)):
        assert quantize(**k) == eoq.EOQ_ERR_UNSUPPORTED
    for k in (dict(src=ODD), dict(src=At((1 << 12) + 2), dtype=eoq.EOQ_F32), dict(codes=At((1 << 12) + 8)), dict(scales=At((1 << 12) + 2))):
        assert quantize(**k) == eoq.EOQ_ERR_ALIGNMENT


def test_forward():
    assert fwd() == eoq.EOQ_ERR_BAD_ARG
    for k in (dict(x_codes=None), dict(x_scales=None), dict(x=None, x_codes=None, x_scales=None), dict(w_codes=None), dict(w_scales=None), dict(y=None)):
        assert fwd(**k) == eoq.EOQ_ERR_BAD_ARG
    for k in (dict(x=ODD), dict(y=ODD), dict(bias=At((1 << 12) + 2)), dict(x_codes=At((1 << 12) + 8)), dict(w_codes=At((1 << 12) + 8)), dict(x_scales=ODD), dict(w_scales=ODD)):
        assert fwd(**k) == eoq.EOQ_ERR_ALIGNMENT
    need = eoq.eoq_lin_workspace_size(desc(), eoq.EOQ_LIN_FWD)
    assert need % 256 == 0 and need > 0
    for ws in (None, At(1 << 12, need - 1), At((1 << 12) + 128)):
        assert fwd(ws=ws) == eoq.EOQ_ERR_WORKSPACE


def test_backward():
    assert bwd() == eoq.EOQ_ERR_BAD_ARG
    for k in (dict(dy=None), dict(dx=None, dw=None, dbias=None), dict(w_codes=None), dict(w_scales=None), dict(x_codes=None), dict(x_scales=None)):
        assert bwd(**k) == eoq.EOQ_ERR_BAD_ARG
    for k in (dict(dy=ODD), dict(dx=ODD), dict(dw=At((1 << 12) + 8)), dict(dbias=ODD), dict(x_codes=At((1 << 12) + 8)), dict(w_codes=At((1 << 12) + 8)), dict(x_scales=ODD),
              dict(w_scales=ODD)):
        assert bwd(**k) == eoq.EOQ_ERR_ALIGNMENT
    need = eoq.eoq_lin_workspace_size(desc(), eoq.EOQ_LIN_BWD)
    for ws in (None, At(1 << 12, need - 1), At((1 << 12) + 128)):
        assert bwd(ws=ws) == eoq.EOQ_ERR_WORKSPACE
    # what is not asked for needs nothing
    assert bwd(w_codes=None, w_scales=None, dx=None, ws=None) == eoq.EOQ_ERR_WORKSPACE
    assert bwd(x_codes=None, x_scales=None, dw=None, ws=None) == eoq.EOQ_ERR_WORKSPACE


class Grads:
    """Stands in for a list of gradients at addresses."""

    def __init__(self, g, sizes, dtypes=None, to=None):
        n = self.num = len(g)
        self.g, self.sizes, self.dtypes = (ctypes.c_void_p * n)(*g), (ctypes.c_size_t * n)(*sizes), (ctypes.c_int * n)(*(dtypes or [eoq.EOQ_F32] * n))
        self.to = None if to is None else (ctypes.c_void_p * n)(*to)


def grads(l, norm=A, ws=A, max_norm=1.0):
    st = eoq.eoq_grad_clip(0, l, max_norm, norm, ws, stream=0, check=False)
    if l.to is None and max_norm == 1.0:
        assert eoq.eoq_grad_norm(0, l, norm, ws, stream=0, check=False) == st
    return st


def test_gradients():
    p = 1 << 12
    assert grads(Grads([p, p], [3, 4])) == eoq.EOQ_ERR_BAD_ARG          # all is well but the handle
    good = Grads([p, 0, p], [3, 0, 4])
    assert grads(good, ws=None) == eoq.EOQ_ERR_WORKSPACE                  # (a tensor without elements needs no address)
    for l in (Grads([], []), Grads([p, 0], [3, 4]), Grads([p], [3], [eoq.EOQ_I32]), Grads([p], [3], [-1]), Grads([p], [3], to=[0])):
        assert grads(l, ws=None) == eoq.EOQ_ERR_BAD_ARG
    assert grads(good, norm=None) == eoq.EOQ_ERR_BAD_ARG
    assert grads(good, max_norm=-1.0) == eoq.EOQ_ERR_BAD_ARG and grads(good, max_norm=float("nan"), ws=None) == eoq.EOQ_ERR_BAD_ARG
    assert grads(Grads([p + 2], [3])) == eoq.EOQ_ERR_ALIGNMENT and grads(Grads([p + 1], [3], [eoq.EOQ_F16])) == eoq.EOQ_ERR_ALIGNMENT
    assert grads(Grads([p], [3], to=[p + 2])) == eoq.EOQ_ERR_ALIGNMENT and grads(good, norm=At(p + 2)) == eoq.EOQ_ERR_ALIGNMENT
    assert grads(Grads([p], [(1 << 40) + 1])) == eoq.EOQ_ERR_UNSUPPORTED and grads(Grads([p] * 20, [1 << 40] * 20)) == eoq.EOQ_ERR_UNSUPPORTED
    need = eoq.eoq_grad_workspace_size(good)
    assert grads(good, ws=At(p, need // 2)) == eoq.EOQ_ERR_WORKSPACE and grads(good, ws=At(p + 128)) == eoq.EOQ_ERR_WORKSPACE


def test_lists_of_gradients():
    import torch

    t = torch.zeros(4, 6)
    for bad in ([t[:, :3]], [t.t()]):
        with pytest.raises(ValueError):
            eoq.grad_list(bad)
    with pytest.raises(TypeError):
        eoq.grad_list([t.double()])
    for out in ([], [torch.zeros(5)], [torch.zeros(24).half()], [torch.zeros(6, 8)[:, :4]]):
        with pytest.raises(ValueError):
            eoq.grad_list([t], out)
    l = eoq.grad_list([t, t.half()[1]], [t, torch.zeros(6).half()])
    assert l.num == 2 and list(l.sizes) == [24, 6] and list(l.dtypes) == [eoq.EOQ_F32, eoq.EOQ_F16]
