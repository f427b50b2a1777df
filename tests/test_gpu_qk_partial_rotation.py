"""qk_norm_rope and its gradient where a part of a head is rotated, at sizes that cut runs of
eight pairs, mix rotated and other pairs in one (neighbouring pairs) or leave fewer than
eight of a kind. Bounds as in test_gpu_qk_norm_rope."""
import pytest
from test_gpu_qk_norm_rope import EPS, _case, _check_backward, _check_forward

import paper_2606_27216_amd as hm

pytestmark = pytest.mark.gpu

SHAPES = [(2, 33, 12, 4, 256, 148), (1, 19, 48, 8, 256, 148), (1, 30, 3, 1, 112, 74), (2, 17, 9, 3, 128, 120), (1, 25, 20, 5, 144, 114),
          (1, 7, 4, 2, 512, 486), (1, 9, 40, 8, 498, 250), (3, 11, 2, 2, 16, 6), (2, 8, 5, 1, 14, 4), (1, 15, 6, 2, 130, 2), (2, 21, 3, 3, 36, 20)]


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dtype,gains", [("f32", "f32"), ("bf16", "f32")])
@pytest.mark.parametrize("inter", [False, True])
def test_both_directions(shape, dtype, gains, inter):
    import torch
    q, k, gq, gk, wq, wk, cos, sin, pos = _case(*shape, dtype, gains, "heads", seed=9, table=40)
    pos[0, 0] = 39  # (the tables' last row)
    print(f"[gpu-case] qk {shape} {dtype} {inter}", flush=True)
    oq, ok = hm.qk_norm_rope(q, k, wq, wk, cos, sin, pos, eps=EPS, interleaved=inter)
    _check_forward(oq, q, wq, cos, sin, pos, inter, dtype)
    _check_forward(ok, k, wk, cos, sin, pos, inter, dtype)
    dq, dk, dwq, dwk = hm.qk_norm_rope_grad(gq, gk, q, k, wq, wk, cos, sin, pos, eps=EPS, interleaved=inter)
    _check_backward(dq, dwq, gq, q, wq, cos, sin, pos, inter, dtype, gains)
    _check_backward(dk, dwk, gk, k, wk, cos, sin, pos, inter, dtype, gains)
    hm.qk_norm_rope(q, k, wq, wk, cos, sin, pos, eps=EPS, interleaved=inter, out=(q, k))
    assert torch.equal(q, oq) and torch.equal(k, ok)
