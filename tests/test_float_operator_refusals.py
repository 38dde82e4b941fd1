"""Calls of the floating-point operators that are refused, told without a device: every check but the handle's comes before any device work."""
import pytest

from paper_2105_13890_b200 import build, eoq

build.build_lib()


class At:
    """Stands in for a tensor at an address."""

    def __init__(self, address, bytes_=1 << 30):
        self.address, self.bytes_ = address, bytes_

    def data_ptr(self):
        return self.address

    def numel(self):
        return self.bytes_

    def element_size(self):
        return 1


A = At(1 << 12)


def desc(**k):
    v = {"n": 2, "hw": 9, "c": 64, "groups": 8, "dtype": eoq.EOQ_BF16, "act": eoq.EOQ_ACT_SILU}
    v.update(k)
    return eoq.gn_desc(**v)


BAD_DESC = [
    (dict(n=0), eoq.EOQ_ERR_BAD_ARG), (dict(hw=0), eoq.EOQ_ERR_BAD_ARG), (dict(c=0), eoq.EOQ_ERR_BAD_ARG), (dict(n=-1), eoq.EOQ_ERR_BAD_ARG),
    (dict(groups=0), eoq.EOQ_ERR_BAD_ARG), (dict(groups=7), eoq.EOQ_ERR_BAD_ARG), (dict(dtype=4), eoq.EOQ_ERR_BAD_ARG),
    (dict(dtype=-1), eoq.EOQ_ERR_BAD_ARG), (dict(act=3), eoq.EOQ_ERR_BAD_ARG), (dict(eps=-1e-5), eoq.EOQ_ERR_BAD_ARG),
    (dict(eps=float("nan")), eoq.EOQ_ERR_BAD_ARG), (dict(x_stride=63), eoq.EOQ_ERR_BAD_ARG), (dict(y_stride=1), eoq.EOQ_ERR_BAD_ARG),
    (dict(dy_stride=8), eoq.EOQ_ERR_BAD_ARG), (dict(dx_stride=60), eoq.EOQ_ERR_BAD_ARG), (dict(n=(1 << 30) + 1), eoq.EOQ_ERR_UNSUPPORTED),
    (dict(hw=(1 << 30) + 1), eoq.EOQ_ERR_UNSUPPORTED), (dict(c=(1 << 20) + 8), eoq.EOQ_ERR_UNSUPPORTED), (dict(x_exp=-14), eoq.EOQ_ERR_RANGE),
    (dict(dtype=eoq.EOQ_I32, x_exp=61), eoq.EOQ_ERR_RANGE), (dict(x_stride=1 << 31), eoq.EOQ_ERR_UNSUPPORTED),
]


def fwd(d, x=A, y=A, gamma=A, beta=A, stats=A, codes=None, exps=None, ws=A):
    return eoq.eoq_gn_fwd(0, d, x, gamma, beta, y, stats, codes, exps, ws, stream=0, check=False)


def bwd(d, dy=A, dy_exp=None, x=A, codes=None, exps=None, gamma=A, beta=A, stats=A, dx=A, dgamma=A, dbeta=A, ws=A):
    return eoq.eoq_gn_bwd(0, d, dy, dy_exp, x, codes, exps, gamma, beta, stats, dx, dgamma, dbeta, ws, stream=0, check=False)


@pytest.mark.parametrize("change,status", BAD_DESC)
def test_group_norm_descriptors(change, status):
    d = desc(**change)
    assert fwd(d) == status and bwd(d) == status
    with pytest.raises(eoq.EoqError) as e:
        eoq.eoq_gn_workspace_size(d)
    assert e.value.status == status


def test_group_norm_pointers():
    d, odd = desc(), At((1 << 12) + 1)
    assert fwd(d) == eoq.EOQ_ERR_BAD_ARG          # all is well but the handle
    assert fwd(d, x=odd) == eoq.EOQ_ERR_ALIGNMENT and fwd(d, y=odd) == eoq.EOQ_ERR_ALIGNMENT
    assert fwd(d, gamma=At((1 << 12) + 2)) == eoq.EOQ_ERR_ALIGNMENT and fwd(d, stats=At((1 << 12) + 4)) == eoq.EOQ_ERR_ALIGNMENT
    assert fwd(d, codes=A) == eoq.EOQ_ERR_BAD_ARG and fwd(d, x=None) == eoq.EOQ_ERR_BAD_ARG
    need = eoq.eoq_gn_workspace_size(d)
    assert fwd(d, ws=None) == eoq.EOQ_ERR_WORKSPACE and fwd(d, ws=At(1 << 12, need // 2)) == eoq.EOQ_ERR_WORKSPACE
    assert fwd(d, ws=At((1 << 12) + 128)) == eoq.EOQ_ERR_WORKSPACE and need % 256 == 0
    assert bwd(d, dy=odd) == eoq.EOQ_ERR_ALIGNMENT and bwd(d, dx=odd) == eoq.EOQ_ERR_ALIGNMENT and bwd(d, dgamma=odd) == eoq.EOQ_ERR_ALIGNMENT
    assert bwd(d, ws=At(1 << 12, 256)) == eoq.EOQ_ERR_WORKSPACE
    # int8 errors carry an exponent, the other types none; x or its 8-bit form, not both
    for k in (dict(stats=None), dict(x=None), dict(codes=A, exps=A), dict(x=None, codes=A), dict(dy_exp=A)):
        assert bwd(d, **k) == eoq.EOQ_ERR_BAD_ARG
    assert bwd(desc(dtype=eoq.EOQ_I32, x_exp=-14), dy=odd, dy_exp=A, dx=odd) == eoq.EOQ_ERR_ALIGNMENT
    with pytest.raises(TypeError):
        eoq.eoq_gn_fwd(0, eoq.conv_desc(1, 8, 8, 16, 16, 3, 3), A, A, A, A, workspace=A, stream=0)


def test_eight_bit_form():
    def save(src=A, dtype=eoq.EOQ_F16, src_exp=0, rows=4, cols=40, stride=40, codes=A, exps=A):
        return eoq.eoq_ckpt_save(0, src, dtype, src_exp, rows, cols, stride, codes, exps, stream=0, check=False)

    def load(codes=A, exps=A, rows=4, cols=40, dst=A, dtype=eoq.EOQ_F16, stride=0):
        return eoq.eoq_ckpt_load(0, codes, exps, rows, cols, dst, dtype, stride, stream=0, check=False)

    for k in (dict(), dict(src=None), dict(rows=0), dict(cols=0), dict(cols=-8), dict(stride=39), dict(dtype=4), dict(dtype=-1), dict(codes=None),
              dict(exps=None)):
        assert save(**k) == eoq.EOQ_ERR_BAD_ARG, k
    for k in (dict(), dict(dst=None), dict(rows=0), dict(cols=0), dict(stride=8), dict(dtype=eoq.EOQ_I32), dict(codes=None), dict(exps=None)):
        assert load(**k) == eoq.EOQ_ERR_BAD_ARG, k
    assert save(src=At(4097)) == eoq.EOQ_ERR_ALIGNMENT and load(dst=At(4098), dtype=eoq.EOQ_F32) == eoq.EOQ_ERR_ALIGNMENT
    assert save(cols=(1 << 20) + 1, stride=0) == eoq.EOQ_ERR_UNSUPPORTED and save(rows=(1 << 40) + 1) == eoq.EOQ_ERR_UNSUPPORTED
    assert save(src_exp=-14) == eoq.EOQ_ERR_RANGE and save(dtype=eoq.EOQ_I32, src_exp=-61) == eoq.EOQ_ERR_RANGE



def test_sizes_that_no_int_holds():
    """Not cut to 32 bits on their way into the library."""
    for cols in (40 + (1 << 32), 40 - (1 << 32)):
        with pytest.raises(OverflowError):
            eoq.eoq_ckpt_save(0, A, eoq.EOQ_F16, 0, 4, cols, 40, A, A, stream=0, check=False)
        with pytest.raises(OverflowError):
            eoq.eoq_ckpt_load(0, A, A, 4, cols, A, eoq.EOQ_F16, 0, stream=0, check=False)
        with pytest.raises(OverflowError):
            eoq.eoq_ckpt_wgrad(0, A, eoq.EOQ_BF16, 64, cols, 0, A, A, 64, A, A, stream=0, check=False)
    with pytest.raises(OverflowError):
        eoq.gn_desc(1 + (1 << 32), 4, 8, 2, eoq.EOQ_F16)


def test_weight_gradient():
    def call(dy=A, dtype=eoq.EOQ_BF16, rows=4096, c_out=32, dy_stride=32, codes=A, exps=A, c_in=64, dw=A, ws=A):
        return eoq.eoq_ckpt_wgrad(0, dy, dtype, rows, c_out, dy_stride, codes, exps, c_in, dw, ws, stream=0, check=False)

    for k in (dict(), dict(dy=None), dict(rows=0), dict(c_out=0), dict(c_in=-1), dict(dy_stride=31), dict(dtype=eoq.EOQ_I32), dict(dtype=-1),
              dict(codes=None), dict(exps=None), dict(dw=None)):
        assert call(**k) == eoq.EOQ_ERR_BAD_ARG, k
    assert call(dy=At(4097)) == eoq.EOQ_ERR_ALIGNMENT and call(dw=At(4100)) == eoq.EOQ_ERR_ALIGNMENT
    assert call(rows=(1 << 36) + 1) == eoq.EOQ_ERR_UNSUPPORTED and call(c_in=(1 << 20) + 1) == eoq.EOQ_ERR_UNSUPPORTED
    need = eoq.eoq_ckpt_wgrad_workspace_size(4096, 32, 64, eoq.EOQ_BF16)
    assert need > 0 and need % 256 == 0
    assert call(ws=None) == eoq.EOQ_ERR_WORKSPACE and call(ws=At(1 << 12, need // 2)) == eoq.EOQ_ERR_WORKSPACE and call(ws=At(4112)) == eoq.EOQ_ERR_WORKSPACE
    with pytest.raises(eoq.EoqError):
        eoq.eoq_ckpt_wgrad_workspace_size(0, 32, 64, eoq.EOQ_BF16)
