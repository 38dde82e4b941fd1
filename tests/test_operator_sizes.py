"""Sizes that an int or a size_t does not hold raise in the binding of the floating-point operators instead of being cut."""
import pytest

from paper_2105_13890_b200 import build, eoq

build.build_lib()


@pytest.mark.parametrize("rows,c_out,c_in,dtype", [(64, 8 + (1 << 32), 16, eoq.EOQ_BF16), (64, 8, 16 + (1 << 32), eoq.EOQ_BF16), (64, 8, 16, eoq.EOQ_F16 + (1 << 32)),
                                                   (64 + (1 << 64), 8, 16, eoq.EOQ_BF16), (64 - (1 << 64), 8, 16, eoq.EOQ_BF16), (64, 8 - (1 << 32), 16, eoq.EOQ_BF16)])
def test_workspace_of_the_weight_gradient(rows, c_out, c_in, dtype):
    assert eoq.eoq_ckpt_wgrad_workspace_size(64, 8, 16, eoq.EOQ_BF16) >= 0
    with pytest.raises(OverflowError):
        eoq.eoq_ckpt_wgrad_workspace_size(rows, c_out, c_in, dtype)


@pytest.mark.parametrize("field,size", [("n", 1 + (1 << 32)), ("hw", 4 - (1 << 32)), ("c", 8 + (1 << 32)), ("x_stride", 8 + (1 << 64)), ("y_stride", (1 << 64)),
                                        ("dy_stride", 8 - (1 << 64)), ("dx_stride", -1)])
def test_descriptor_of_a_group_norm(field, size):
    whole = dict(n=1, hw=4, c=8, groups=2, dtype=eoq.EOQ_F16)
    assert eoq.eoq_gn_workspace_size(eoq.gn_desc(**whole)) > 0
    with pytest.raises(OverflowError):
        eoq.gn_desc(**{**whole, field: size})
