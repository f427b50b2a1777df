"""Sizes that a launch or a kernel's indexes cannot hold: refused before anything is
enqueued. (No call may follow a pointer here, nor reach a device.)"""
import pytest
from test_train_ops_cpu import GRAD, HEADS, P, WGRAD, _call, _qk

import paper_2606_27216_amd as hm

MOST = 1 << 30


@pytest.mark.parametrize("hq,hk", [(2 ** 31 - 1, 2 ** 31 - 1), (2 ** 31 - 1, 1), (1, 2 ** 31 - 1), (MOST, MOST), (MOST, 1), (MOST - 8, 9)])
def test_heads_of_queries_and_keys(hq, hk):
    """Their number together is a 32-bit one in the kernels."""
    L = hm.lib()
    args = _qk(hq=hq, hk=hk)
    assert L.himuon_qk_norm_rope(args, HEADS, HEADS, HEADS, HEADS, None) == hm.ERR_UNSUPPORTED
    assert L.himuon_qk_norm_rope_grad(args, *[HEADS] * 6, P, P, P, 1 << 40, None) == hm.ERR_UNSUPPORTED


@pytest.mark.parametrize("n,dim", [(600, 65535 * 512 + 1), (5000, 1 << 26), ((1 << 30) - 1, 32 * 512 + 1)])
def test_sums_of_a_tables_gradient(n, dim):
    """More columns or chunks than the sums' launches hold: known before the sort is enqueued."""
    L = hm.lib()
    assert _call("embed_grad", GRAD, n=n, dim=dim, ld_grad=dim, ld_out=dim, ws_bytes=1 << 60) == hm.ERR_UNSUPPORTED
    assert L.himuon_embed_grad_workspace_size(n, 10, dim) == 0
    assert L.himuon_embed_grad_workspace_size(600, 10, 65535 * 512) > 0


@pytest.mark.parametrize("dtype", [hm.F32, hm.BF16])
@pytest.mark.parametrize("n", [0, 64, 100000])
def test_tiles_of_a_weight_gradient(n, dtype):
    """More tiles than a launch holds: known before the gradient is laid out."""
    rows, cols = (1 << 26) - 8192, (1 << 26) - 8191
    assert _call("weight_grad", WGRAD, n=n, out=rows, cols=cols, ld_grad=rows, ld_dw=cols, dtype=dtype,
                 ws_bytes=1 << 60) == hm.ERR_UNSUPPORTED
    assert hm.lib().himuon_weight_grad_workspace_size(n, rows, cols, P, rows, dtype) == 0
