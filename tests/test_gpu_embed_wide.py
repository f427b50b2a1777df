"""embed_grad of short batches of wide rows: batches that are not sorted whose blocks take
several parts of the columns in turn (more than 2048 / tokens parts of 512), and sorted ones
of at most 2048 tokens, whose joins have blocks of four waves with eight columns a lane, in
each size of a chunk. Bounds as in test_gpu_embed_ops."""
import pytest
from test_gpu_embed_ops import _check_grad, _dt, _ids, _rand

import paper_2606_27216_amd as hm

pytestmark = pytest.mark.gpu

#          not sorted                                       chunks of 8,      8,              16,             32
SHAPES = [(400, 5000, 4100), (300, 90, 4096), (512, 40, 2561), (1500, 3000, 2051), (513, 300, 1025), (2000, 100, 5000), (2048, 64, 9500)]


@pytest.mark.parametrize("n,rows,width", SHAPES)
@pytest.mark.parametrize("kind", ["mixed", "one"])
@pytest.mark.parametrize("dtype,out", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
def test_gradient(n, rows, width, kind, dtype, out):
    import torch
    tokens = _ids(n, rows, 60, kind, "i32" if n % 2 else "i64")
    grad = _rand((n, width + 3), dtype, 61)[:, 2:2 + width]
    print(f"[gpu-case] embed_grad {n} {rows} {width} {kind} {dtype} {out}", flush=True)
    got = hm.embed_grad(tokens, grad, rows, scale=1.5, dtype=_dt(out))
    _check_grad(got, tokens, grad, rows, 1.5, out)
    space = _rand((rows, width + 4), out, 62)
    before = space.clone()
    hm.embed_grad(tokens, grad, rows, out=space[:, 1:1 + width], accumulate=True)
    assert torch.equal(space[:, 0], before[:, 0]) and torch.equal(space[:, 1 + width:], before[:, 1 + width:])
    _check_grad(space[:, 1:1 + width], tokens, grad, rows, 1.0, out, base=before[:, 1:1 + width])
    hm.embed_grad(tokens, grad, rows, scale=1.5, out=space[:, 1:1 + width])
    assert torch.equal(space[:, 1:1 + width], got)
    assert torch.equal(space[:, 0], before[:, 0]) and torch.equal(space[:, 1 + width:], before[:, 1 + width:])
