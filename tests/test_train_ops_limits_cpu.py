"""Sizes that a launch or a kernel's indexes cannot hold: refused before anything is
enqueued. (No call may follow a pointer here, nor reach a device.)"""
import pytest
from test_train_ops_cpu import HEADS, P, _qk

import paper_2606_27216_amd as hm

MOST = 1 << 30


@pytest.mark.parametrize("hq,hk", [(2 ** 31 - 1, 2 ** 31 - 1), (2 ** 31 - 1, 1), (1, 2 ** 31 - 1), (MOST, MOST), (MOST, 1), (MOST - 8, 9)])
def test_heads_of_queries_and_keys(hq, hk):
    """Their number together is a 32-bit one in the kernels."""
    L = hm.lib()
    args = _qk(hq=hq, hk=hk)
    assert L.himuon_qk_norm_rope(args, HEADS, HEADS, HEADS, HEADS, None) == hm.ERR_UNSUPPORTED
    assert L.himuon_qk_norm_rope_grad(args, *[HEADS] * 6, P, P, P, 1 << 40, None) == hm.ERR_UNSUPPORTED
