"""Outputs of the query and key calls whose rows would fall on each other are refused
before anything is enqueued."""
import pytest

import paper_2606_27216_amd as hm
from paper_2606_27216_amd import train_ops as ops

P = 0x10000  # a pointer that no call may follow
GOOD = ops._HEADS.pack(P, 512, 128, 64)
ARGS = ops._QK.pack(2, 4, 2, 2, 64, 64, 0, hm.F32, hm.F32, ops.I64, P, P, P, P, 100, P, 1e-6)


@pytest.mark.parametrize("strides", [(0, 128, 64), (512, 0, 64), (512, 128, 0)])
@pytest.mark.parametrize("which", [0, 1])
def test_output_strides_of_zero(strides, which):
    L = hm.lib()
    outs = [GOOD, GOOD]
    outs[which] = ops._HEADS.pack(P, *strides)
    assert L.himuon_qk_norm_rope(ARGS, GOOD, GOOD, *outs, None) == hm.ERR_INVALID_ARG
    assert L.himuon_qk_norm_rope_grad(ARGS, GOOD, GOOD, GOOD, GOOD, *outs, P, P, P, 1 << 40, None) == hm.ERR_INVALID_ARG
