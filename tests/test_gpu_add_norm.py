"""add_norm and its gradient against the definition in 64 bits.

Tolerances: a sum of n products in fp32 is off by at most n 2^-24 of the sum of their
magnitudes; r takes half of its argument's relative error; a store is off by half a step.
"""
import pytest

torch = pytest.importorskip("torch")
import paper_2606_27216_amd as hm

pytestmark = pytest.mark.gpu
T = {"f32": torch.float32, "bf16": torch.bfloat16}
U = 2.0 ** -24


def half(dtype):
    return torch.finfo(dtype).eps / 2


def make(rows, width, dtype, gain, seed, ld=None):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def one(scale):
        t = torch.randn(rows, ld or width, generator=gen, device="cuda") * scale
        return t.to(T[dtype])[:, :width]
    x, res, gy, gh = one(1.0), one(2.0), one(0.1), one(0.1)
    w = (1 + 0.3 * torch.randn(width, generator=gen, device="cuda")).to(T[gain])
    return x, res, gy, gh, w


def close(got, want, tol):
    assert got.shape == want.shape
    off = (got.double() - want).abs()
    bad = off > tol
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} off, worst {float((off / tol.clamp_min(1e-300)).max()):.3g} times the tolerance"


SIZES = [(1, 1), (1, 64), (3, 7), (5, 100), (33, 512), (70, 513), (40, 1000), (9, 1024), (17, 1025), (65, 2048), (31, 2500), (12, 4096),
         (7, 5001), (3, 8192), (5, 8200), (3, 16384), (2, 16391), (700, 640)]


@pytest.mark.parametrize("dtype,gain", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("rows,width", SIZES)
def test_forward_and_backward(rows, width, dtype, gain):
    print("[gpu-case] add_norm", rows, width, dtype, gain, flush=True)
    for residual, ld in ((True, None), (False, width + 3), (True, width + 8)):
        x, res, gy, gh, w = make(rows, width, dtype, gain, rows + width, ld)
        h, y = hm.add_norm(x, res if residual else None, w)
        s = x.double() + (res.double() if residual else 0.0)
        r = (s.square().mean(1, keepdim=True) + 1e-6).rsqrt()
        e = half(T[dtype])
        if residual:
            close(h, s, s.abs() * (e + 2 * U))
        else:
            assert h is x
        # (the addition 2 U, the mean (width + 4) U / 2, root, reciprocal and products 8 U)
        want = s * r * w.double()
        close(y, want, want.abs() * (e + (width / 2 + 12) * U))
        H = h.double()
        r = (H.square().mean(1, keepdim=True) + 1e-6).rsqrt()
        for up in (gh, None):
            dh, dw = hm.add_norm_grad(gy, h, w, g_h=up)
            G, W = gy.double(), w.double()
            part = r * (G * W - H * r * r * (G * W * H).mean(1, keepdim=True))
            size = r * ((G * W).abs() + H.abs() * r * r * (G * W * H).abs().mean(1, keepdim=True))
            want = part + (0 if up is None else up.double())
            close(dh, want, want.abs() * e + size * (3 * width / 2 + 24) * U + want.abs() * 2 * U + 1e-38)
            want = (G * H * r).sum(0)
            close(dw, want, want.abs() * half(w.dtype) + (G * H * r).abs().sum(0) * (rows + width / 2 + 16) * U + 1e-38)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,width", [(1, 40), (32, 64), (33, 100), (95, 1000), (64, 4096), (130, 2049), (40, 20000)])
def test_packed_output_is_the_stored_ones(rows, width, dtype):
    print("[gpu-case] add_norm pack", rows, width, dtype, flush=True)
    x, res, _, _, w = make(rows, width, dtype, "f32", 5)
    h, y, codes, exps = hm.add_norm(x, res, w, pack=True)
    h2, y2 = hm.add_norm(x, res, w)
    assert torch.equal(h, h2) and torch.equal(y, y2)
    want = hm.act_pack(y)
    assert torch.equal(codes, want[0]) and torch.equal(exps, want[1])
    _, y3, codes, exps = hm.add_norm(x, None, w, pack=True)
    want = hm.act_pack(y3)
    assert torch.equal(codes, want[0]) and torch.equal(exps, want[1])


def test_in_place_and_shapes():
    x, res, gy, gh, w = make(24, 300, "bf16", "f32", 3)
    h, y = hm.add_norm(x, res, w)
    dh, dw = hm.add_norm_grad(gy, h, w, g_h=gh)
    a, b, c = x.clone(), res.clone(), gy.clone()
    out = hm.add_norm(a, b, w, out=(b, a))
    assert out[0] is b and torch.equal(b, h) and torch.equal(a, y)
    got, _ = hm.add_norm_grad(c, h, w, g_h=gh, out=c)
    assert torch.equal(got, dh)
    h3, y3 = hm.add_norm(x.view(2, 3, 4, 300), res.view(2, 3, 4, 300), w)
    assert y3.shape == (2, 3, 4, 300) and torch.equal(y3.view(24, 300), y) and torch.equal(h3.view(24, 300), h)
    assert hm.add_norm(x[:0], res[:0], w)[1].shape == (0, 300)
    assert not hm.add_norm_grad(gy[:0], h[:0], w)[1].any()


def test_large_and_tiny_rows():
    """Rows whose squares pass fp32's range are infinite as the formula's sum is; tiny ones go by eps."""
    w = torch.ones(256, device="cuda")
    x = torch.full((2, 256), 1e-12, device="cuda")
    want = 1e-12 / (1e-24 + 1e-6) ** 0.5
    assert torch.allclose(hm.add_norm(x, None, w)[1], torch.full_like(x, want), rtol=1e-5, atol=0)
    assert not hm.add_norm(torch.zeros(2, 256, device="cuda"), None, w)[1].any()


def test_autograd_and_differences():
    """Gradients through autograd against the definition's differences in 64 bits."""
    x, res, gy, gh, w = make(6, 90, "f32", "f32", 11)
    x, res, w = x.clone().requires_grad_(), res.clone().requires_grad_(), w.requires_grad_()
    h, y = hm.add_norm(x, res, w)
    ((h * gh).sum() + (y * gy).sum()).backward()
    assert torch.equal(x.grad, res.grad)

    def loss(a, b, c):
        s = a + b
        return ((s * gh.double()).sum() + (s * (s.square().mean(1, keepdim=True) + 1e-6).rsqrt() * c * gy.double()).sum())
    gen = torch.Generator(device="cuda").manual_seed(1)
    args = [t.detach().double() for t in (x, res, w)]
    step = 1e-5
    for i, g in enumerate((x.grad, res.grad, w.grad)):
        d = torch.randn(args[i].shape, generator=gen, device="cuda", dtype=torch.float64)
        up, down = list(args), list(args)
        up[i], down[i] = args[i] + step * d, args[i] - step * d
        want = float(loss(*up) - loss(*down)) / (2 * step)
        # (differences: step^2; fp32: some 100 U of the terms' magnitudes)
        assert abs(float((g.double() * d).sum()) - want) < 1e-7 + 200 * U * float((g.double() * d).abs().sum())
    x.grad = w.grad = None
    same, y = hm.add_norm(x, None, w, pack=True)[:2]
    assert same is x
    (y * gy).sum().backward()
    want = hm.add_norm_grad(gy, x.detach(), w.detach())
    assert torch.equal(x.grad, want[0]) and torch.equal(w.grad, want[1])
