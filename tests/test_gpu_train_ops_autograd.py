"""embed and qk_norm_rope where autograd records: the gradients are, bit for bit, those of
embed_grad and qk_norm_rope_grad, whatever the upstream gradient's strides."""
import pytest

import paper_2606_27216_amd as hm

pytestmark = pytest.mark.gpu


def _rand(shape, dtype, seed):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*shape, generator=gen, device="cuda").to({"f32": torch.float32, "bf16": torch.bfloat16}[dtype])


def _upstream(y, kind, seed):
    """A gradient of y, whole, with its last two axes' strides swapped, or one value expanded."""
    import torch
    g = _rand(y.shape, "f32", seed).to(y.dtype)
    if kind == "swapped" and y.dim() > 1:
        return g.transpose(-1, -2).contiguous().transpose(-1, -2)
    return g.flatten()[:1].view([1] * y.dim()).expand(y.shape) if kind == "expanded" else g


KINDS = ["whole", "swapped", "expanded"]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("shape", [(), (1,), (700,), (3, 500), (0,)], ids=str)
def test_embed(shape, dtype, kind):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(1)
    tokens = torch.randint(-3, 90, shape, generator=gen, device="cuda")
    table = _rand((80, 72), dtype, 2)
    print(f"[gpu-case] embed under autograd {shape} {dtype} {kind}", flush=True)
    want = hm.embed(tokens, table, scale=3.0)
    assert not want.requires_grad
    leaf = table.clone().requires_grad_()
    got = hm.embed(tokens, leaf, scale=3.0)
    assert got.requires_grad and torch.equal(got.detach(), want)
    g = _upstream(want, kind if tokens.numel() else "whole", 3)
    got.backward(g)
    assert torch.equal(leaf.grad, hm.embed_grad(tokens.view(-1), g.reshape(-1, 72).contiguous(), 80, scale=3.0))


@pytest.mark.parametrize("dtype,gains", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("inter", [False, True])
def test_qk_norm_rope(dtype, gains, kind, inter):
    import torch
    x = _rand((2, 33, 10, 64), dtype, 4)
    wq, wk = _rand((64,), gains, 5), _rand((64,), gains, 6)
    cos, sin = _rand((50, 16), "f32", 7), _rand((50, 16), "f32", 8)
    pos = torch.randint(-5, 50, (2, 33), generator=torch.Generator(device="cuda").manual_seed(9), device="cuda")
    print(f"[gpu-case] qk under autograd {dtype} {gains} {kind} {inter}", flush=True)
    args = (x[:, :, :6], x[:, :, 6:8], wq, wk)
    rest = (cos, sin, pos, 1e-5, inter)
    want = hm.qk_norm_rope(*args, *rest)
    g = [_upstream(y, kind, 10 + i) for i, y in enumerate(want)]
    grads = hm.qk_norm_rope_grad(*(t.contiguous() for t in g), *args, *rest)
    leaf = x.clone().requires_grad_()
    lq, lk = wq.clone().requires_grad_(), wk.clone().requires_grad_()
    got = hm.qk_norm_rope(leaf[:, :, :6], leaf[:, :, 6:8], lq, lk, *rest)
    assert all(y.requires_grad and torch.equal(y.detach(), w) for y, w in zip(got, want))
    torch.autograd.backward(got, g)
    assert torch.equal(leaf.grad[:, :, :6], grads[0]) and torch.equal(leaf.grad[:, :, 6:8], grads[1])
    assert bool((leaf.grad[:, :, 8:] == 0).all())
    assert torch.equal(lq.grad, grads[2]) and torch.equal(lk.grad, grads[3])


def test_one_output_or_one_gain_alone():
    """The output that is not used gives no gradient; a gain alone may ask for one."""
    import torch
    q, k, w = _rand((40, 4, 32), "f32", 11), _rand((40, 2, 32), "f32", 12), _rand((32,), "f32", 13)
    cos, sin, g = _rand((40, 16), "f32", 14), _rand((40, 16), "f32", 15), _rand((40, 2, 32), "f32", 16)
    want = hm.qk_norm_rope_grad(torch.zeros_like(q), g, q, k, w, w, cos, sin)
    lq, lk, lw = q.clone().requires_grad_(), k.clone().requires_grad_(), w.clone().requires_grad_()
    hm.qk_norm_rope(lq, lk, w, lw, cos, sin)[1].backward(g)
    assert bool((lq.grad == 0).all()) and torch.equal(lk.grad, want[1]) and torch.equal(lw.grad, want[3])
    lw = w.clone().requires_grad_()
    hm.qk_norm_rope(q, k, w, lw, cos, sin)[1].backward(g)
    assert torch.equal(lw.grad, want[3])


def test_where_nothing_is_recorded():
    """Without recording, and into tensors that are given, the results are the same and carry no graph."""
    import torch
    tokens = torch.arange(20, device="cuda")
    table = _rand((20, 24), "bf16", 17).requires_grad_()
    q, k, w = _rand((20, 2, 32), "bf16", 18).requires_grad_(), _rand((20, 1, 32), "bf16", 19), _rand((32,), "f32", 20)
    cos, sin = _rand((20, 16), "f32", 21), _rand((20, 16), "f32", 22)
    with torch.no_grad():
        rows, heads = hm.embed(tokens, table), hm.qk_norm_rope(q, k, w, w, cos, sin)
    assert not rows.requires_grad and not heads[0].requires_grad
    into = torch.empty_like(rows)
    assert hm.embed(tokens, table, out=into) is into and not into.requires_grad and torch.equal(into, rows)
    into = tuple(torch.empty_like(h) for h in heads)
    got = hm.qk_norm_rope(q, k, w, w, cos, sin, out=into)
    assert all(a is b and not a.requires_grad and torch.equal(a, h) for a, b, h in zip(got, into, heads))


def test_on_another_stream():
    import torch
    tokens, table, g = torch.arange(300, device="cuda") % 77, _rand((77, 40), "f32", 23), _rand((300, 40), "f32", 24)
    q, k, w = _rand((300, 2, 64), "f32", 25), _rand((300, 1, 64), "f32", 26), _rand((64,), "f32", 27)
    cos, sin = _rand((300, 32), "f32", 28), _rand((300, 32), "f32", 29)
    leaf, lq = table.clone().requires_grad_(), q.clone().requires_grad_()
    want, want_q = hm.embed_grad(tokens, g, 77), hm.qk_norm_rope_grad(q, k, q, k, w, w, cos, sin)[0]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    rows = hm.embed(tokens, leaf, stream=side)
    heads = hm.qk_norm_rope(lq, k, w, w, cos, sin, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    torch.autograd.backward((rows, *heads), (g, q, k))
    torch.cuda.synchronize()
    assert torch.equal(leaf.grad, want) and torch.equal(lq.grad, want_q)


def test_gradients_of_gradients_are_refused():
    import torch
    table = _rand((9, 8), "f32", 30).requires_grad_()
    y = hm.embed(torch.arange(9, device="cuda"), table)
    (grad,) = torch.autograd.grad((y * y).sum(), table, create_graph=True)
    with pytest.raises(RuntimeError):
        grad.sum().backward()
