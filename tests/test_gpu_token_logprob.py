"""token_logprob and its gradient against the definition in 64 bits.

Tolerances: z = scale x is off by U |z|, its distance to the maximum by U of both; an
exponential of base 2 by 2 U and its argument's error; the sums of n terms by n U at the worst.
"""
import math

import pytest

torch = pytest.importorskip("torch")
import paper_2606_27216_amd as hm

pytestmark = pytest.mark.gpu
T = {"f32": torch.float32, "bf16": torch.bfloat16}
U = 2.0 ** -24


def make(rows, vocab, dtype, seed, ld=None):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    z = torch.randn(rows, ld or vocab, generator=gen, device="cuda") * (1 + 3 * torch.rand(rows, 1, generator=gen, device="cuda"))
    t = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
    return z.to(T[dtype])[:, :vocab], t


def ordered(x, k):
    """The k largest by (value, first index), as a stable sort gives them."""
    return torch.sort(x.double(), dim=1, descending=True, stable=True).indices[:, :k]


def check(z, t, top, scale):
    rows, vocab = z.shape
    got = hm.token_logprob(z, t, top=top, scale=scale)
    s = z.double() * scale
    lp = torch.log_softmax(s, 1)
    size = float(s[s.isfinite()].abs().max()) + 1
    tol = (8 * size + vocab + 16) * U
    at = t.clamp(0)[:, None].long()
    want = lp.gather(1, at)[:, 0]
    assert float((got[0].double() - want).abs().max()) <= tol
    entropy = -torch.where(lp == -math.inf, 0.0, lp.exp() * lp).sum(1)
    assert float((got[1].double() - entropy).abs().max()) <= tol * (2 + math.log(vocab + 1))
    assert float((got[2].double() - torch.logsumexp(s, 1)).abs().max()) <= tol
    if top:
        best = ordered(z, top)
        assert torch.equal(got[4], best)
        near = (got[3].double() - lp.gather(1, best)).abs()
        assert float(near[lp.gather(1, best) > -math.inf].max()) <= tol
    return got


SIZES = [(1, 1), (3, 2), (5, 7), (4, 63), (9, 64), (70, 511), (33, 513), (6, 2048), (5, 2049), (130, 5003), (3, 16384), (4, 16385),
         (2, 32000), (3, 128000), (1, 130001)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab", SIZES)
def test_forward_and_backward(rows, vocab, dtype):
    print("[gpu-case] token_logprob", rows, vocab, dtype, flush=True)
    for top, scale, ld in ((0, 1.0, None), (min(5, vocab), 0.7, vocab + 5), (min(64, vocab), 1.0, vocab + 8), (1, 2.0, None)):
        z, t = make(rows, vocab, dtype, rows + vocab + top, ld)
        got = check(z, t, top, scale)
        gen = torch.Generator(device="cuda").manual_seed(9)
        gl, gh = (torch.randn(rows, generator=gen, device="cuda") for _ in range(2))
        for a, b in ((gl, gh), (gl, None), (None, gh)):
            d = hm.token_logprob_grad(a, b, z, t, got[2], got[1], scale=scale)
            s = z.double() * scale
            lp = s - got[2].double()[:, None]
            p = lp.exp()
            delta = torch.zeros_like(p).scatter_(1, t[:, None], 1.0)
            A = 0.0 if a is None else a.double()[:, None]
            B = 0.0 if b is None else b.double()[:, None]
            H = got[1].double()[:, None]
            want = scale * (A * (delta - p) - B * p * (lp + H))
            e = (3 * (float(s.abs().max()) + float(got[2].abs().max())) + 8) * U  # of a probability
            size = scale * (abs(A) * (p * e + (delta + p) * 4 * U) + abs(B) * p * ((lp.abs() + H) * (e + 6 * U) + e))
            off = (d.double() - want).abs()
            assert bool((off <= size * 1.1 + want.abs() * torch.finfo(T[dtype]).eps / 2 + 1e-37).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [50, 300, 3000, 20000])
def test_ties_masks_and_special_values(vocab, dtype):
    print("[gpu-case] token_logprob special", vocab, dtype, flush=True)
    k = 20
    z, t = make(12, vocab, dtype, 3)
    z = z.contiguous()
    z[0] = 0.5                                    # all equal: the first indices
    z[1] = torch.arange(vocab, device="cuda") % 3  # three values
    z[2, 5:] = -math.inf                          # fewer finite logits than alternatives
    t[2] = 3
    z[3, ::2] = -math.inf                         # half of the vocabulary masked
    t[3] = 1
    z[4] = torch.finfo(T[dtype]).min              # a mask of the type's lowest value
    z[4, 7] = 1.0
    z[5] = -0.0
    z[5, ::5] = 0.0                               # zeros of both signs are equal
    z[6] = torch.arange(vocab, device="cuda").flip(0) / 8.0
    z[7] = torch.arange(vocab, device="cuda") / 8.0
    z[8] = 1e4 + z[8] if dtype == "f32" else z[8]
    got = check(z[[0, 1, 3, 5, 6, 7, 9]].contiguous(), t[[0, 1, 3, 5, 6, 7, 9]].contiguous(), k, 1.0)
    got = hm.token_logprob(z, t, top=k)
    assert torch.equal(got[4], ordered(z, k))
    assert bool((got[3][2, 5:] == -math.inf).all()) and bool(got[3][2, :5].isfinite().all())
    assert float(got[0][4]) == -math.inf or float(got[0][4]) < -1e30
    assert float(got[1][4]) == 0.0
    d = hm.token_logprob_grad(torch.ones(12, device="cuda"), torch.ones(12, device="cuda"), z, t, got[2], got[1])
    assert bool(d[2].isfinite().all()) and not d[2, 5:].any() and bool(d[3].isfinite().all()) and not d[3, ::2].any()
    # NaN: the largest; the row's numbers are NaN, the others' are not
    z[9, 11] = math.nan
    z[9, 30] = -math.nan
    again = hm.token_logprob(z, t, top=k)
    assert again[4][9, :2].tolist() == [11, 30] and bool(again[0][9].isnan()) and bool(again[3][9].isnan().all())
    others = [i for i in range(12) if i != 9]
    for a, b in zip(got, again):
        assert torch.equal(a[others], b[others])


@pytest.mark.parametrize("vocab", [1, 5, 64, 3000, 20000])
def test_nan_at_the_first_token(vocab):
    print("[gpu-case] token_logprob first NaN", vocab, flush=True)
    z, t = make(6, vocab, "f32", 12)
    z[2, 0] = math.nan
    z[4] = math.nan
    k = min(vocab, 64)
    got = hm.token_logprob(z, t, top=k)
    want = ordered(torch.where(z.isnan(), math.inf, z), k)
    assert torch.equal(got[4], want)
    for r in (2, 4):
        assert all(bool(x[r].isnan().all()) for x in got[:4])
    assert all(bool(x[[0, 1, 3, 5]].isfinite().all()) for x in got[:4])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [33, 3000, 20000, 70000])
def test_logits_far_from_zero(vocab, dtype):
    # lse rounds by 2^-24 of itself, which leaves the probabilities to the logits' distances: products
    # with c = log2 e of distances to the maximum (6 U of up to D), sums of vocab terms
    print("[gpu-case] token_logprob far", vocab, dtype, flush=True)
    gen = torch.Generator(device="cuda").manual_seed(vocab)
    near = torch.randint(0, 9, (10, vocab), generator=gen, device="cuda").float()
    t = torch.randint(0, vocab, (10,), generator=gen, device="cuda")
    low = torch.finfo(T[dtype]).min
    z = torch.stack([near[0] - 2.0 ** (10 if dtype == "bf16" else 20), near[1] + 2.0 ** (10 if dtype == "bf16" else 20), near[2] * 512 - 1e6,
                     torch.full_like(near[3], -1e9), torch.full_like(near[4], low), near[5], near[6] * 512 + 1e5, near[7] - 5000, near[8] + 5000,
                     near[9]]).to(T[dtype])
    z[4, ::2] = -math.inf if vocab > 33 else low
    z[9, ::3] = low
    t[4], t[9] = 1, 1
    s = z.double()
    lp = torch.log_softmax(s, 1)
    p = lp.exp()
    H = -torch.where(p == 0, 0.0, p * lp).sum(1)
    got = hm.token_logprob(z, t, top=min(vocab, 20))
    D = (s.amax(1, keepdim=True) - s).clamp(0, 200) + math.log(vocab) + 1  # (beyond: a probability of less than e^-150)
    tol = (6 * D + vocab + 16) * U
    at = t[:, None]
    assert bool(((got[0].double() - lp.gather(1, at)[:, 0]).abs() <= tol.gather(1, at)[:, 0] + 4 * U * lp.gather(1, at)[:, 0].abs()).all())
    assert bool(((got[1].double() - H).abs() <= (p * (tol * (lp.abs().clamp(0, 300) + 2))).sum(1) + tol.amin(1) * (H + 2)).all())
    lse = torch.logsumexp(s, 1)
    assert bool(((got[2].double() - lse).abs() <= tol.amin(1) + 2 * U * lse.abs()).all())
    assert torch.equal(got[4], ordered(z, min(vocab, 20)))
    gl, gh = (torch.randn(10, generator=gen, device="cuda") for _ in range(2))
    for a, b, out in ((gl, gh, None), (gl, None, z.clone()), (None, gh, None)):
        d = hm.token_logprob_grad(a, b, z if out is None else out, t, got[2], got[1], out=out)
        delta = torch.zeros_like(p).scatter_(1, at, 1.0)
        A, B = (0.0 if x is None else x.double()[:, None] for x in (a, b))
        E = got[1].double()[:, None]
        L = lp.clamp_min(-1e30)
        want = A * (delta - p) - B * p * (L + E)
        e = tol + 2.0 ** -13  # (an lse below 1024 is off by 2^-14 or less, and so is a sum of two)
        size = abs(A) * (p * e + (delta + p) * 4 * U) + abs(B) * p * ((L.abs() + E) * (e + 6 * U) + e)
        assert bool(((d.double() - want).abs() <= size * 1.1 + want.abs() * torch.finfo(T[dtype]).eps / 2 + 1e-37).all())


def test_rows_not_in_use_and_empty_rows():
    z, t = make(40, 700, "f32", 4)
    t[::3] = -1
    t[1] = 700
    off = (t < 0) | (t >= 700)
    want = hm.token_logprob(torch.where(off[:, None], 0.0, z), t, top=3)
    z[off] = math.nan                              # they are not read
    z[2] = -math.inf                               # in use, and nothing left
    got = hm.token_logprob(z, t.int(), top=3)
    for a in got[:4]:
        assert not a[off].any()
    assert bool((got[4][off] == -1).all())
    assert float(got[0][2]) == -math.inf and float(got[1][2]) == 0.0 and float(got[2][2]) == -math.inf
    assert got[4][2].tolist() == [0, 1, 2] and bool((got[3][2] == -math.inf).all())
    rest = ~off
    rest[2] = False
    for a, b in zip(got, want):
        assert torch.equal(a[rest], b[rest])
    g = torch.ones(40, device="cuda")
    d = hm.token_logprob_grad(g, g, z, t, got[2], got[1])
    assert not d[off].any() and not d[2].any() and bool(d.isfinite().all())
    same = z.clone()
    assert torch.equal(hm.token_logprob_grad(g, g, same, t, got[2], got[1], out=same), d)
    assert hm.token_logprob(z[:0], t[:0], top=2)[4].shape == (0, 2)


def test_autograd_and_differences():
    z, t = make(24, 333, "f32", 8)
    z = z.clone().view(4, 6, 333).requires_grad_()
    t = t.view(4, 6)
    t[0, 0] = -1
    lp, entropy, lse = hm.token_logprob(z, t, scale=1.3)
    assert not lse.requires_grad
    (-lp.mean() - 0.1 * entropy.sum()).backward()

    def loss(x):
        p = torch.log_softmax(x * 1.3, -1)
        on = (t >= 0).double()
        return -(p.gather(-1, t.clamp(0)[..., None])[..., 0] * on).mean() + 0.1 * ((p.exp() * p).sum(-1) * on).sum()
    x, step = z.detach().double(), 1e-5
    gen = torch.Generator(device="cuda").manual_seed(1)
    for _ in range(3):
        d = torch.randn(x.shape, generator=gen, device="cuda", dtype=torch.float64)
        want = float(loss(x + step * d) - loss(x - step * d)) / (2 * step)
        assert abs(float((z.grad.double() * d).sum()) - want) < 1e-7 + 200 * U * float((z.grad.double() * d).abs().sum())
    z.grad = None
    hm.token_logprob(z, t, top=4)[1].sum().backward()  # (the entropy alone)
    assert bool(z.grad.isfinite().all()) and not z.grad[0, 0].any()
