"""attention's sizes and results at their limits, on a machine without a GPU: refused before anything
is enqueued."""
import pytest
from test_block_ops_cpu import BIG, HEADS, P, _attn, _backward

import paper_2606_27216_amd as hm
from paper_2606_27216_amd import train_ops


def _place(n):
    return train_ops._HEADS.pack(n * P, 64 * 4 * 12, 64 * 4, 64)


@pytest.mark.parametrize("places", [(2, 2, 3), (2, 3, 2), (2, 3, 3)])
def test_gradients_in_each_others_place(places):
    """Two results in one array would be written by two blocks at a time."""
    assert _backward(_attn(), [HEADS] * 5 + [_place(n) for n in places]) == hm.ERR_INVALID_ARG
    # (a side without tokens has no place)
    none = train_ops._HEADS.pack(0, 64 * 4 * 12, 64 * 4, 64)
    assert _backward(_attn(q_len=0, k_len=0), [none] * 8, lse=None, ws=None, ws_bytes=0) == hm.OK



@pytest.mark.parametrize("batch,q_len,heads,size", [(1 << 20, 1 << 20, 1 << 19, 1 << 62)] + [
    (n, n, h, 0) for n in (1 << 20, 1 << 30) for h in ((1 << 28) + 1, (1 << 29) + 1, (1 << 30) - 1, (1 << 31) - 1)])
def test_statistics_past_64_bits(batch, q_len, heads, size):
    """batch * q_len * q_heads rows of eight bytes: more than 2^62 bytes are no size of a workspace."""
    args = _attn(batch=batch, q_len=q_len, k_len=1, hq=heads, hk=heads)
    assert hm.lib().himuon_attention_grad_workspace_size(args) == size
    if size == 0:
        assert _backward(args, ws_bytes=BIG) == hm.ERR_UNSUPPORTED
