"""act_pack, act_unpack and weight_grad against their definitions in 64 bits.

Packing has one right answer for finite values. The weight gradient's products are
exact; the fp32 accumulation of T terms (three times as many for an fp32 gradient)
is off by at most T 2^-23 of the terms' sizes whatever its order and rounding, and the
result is rounded once to its type. Rounding errors of either sign add up like sqrt(T):
4 sqrt(T) 2^-23 bounds the relative distance of the whole matrix."""
import pytest

import paper_2606_27216_amd as hm

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
ROUND = {"f32": 2 * U, "bf16": 2.0 ** -8 + 2 * U}


def _dt(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


def _rand(shape, dtype, seed, scale=1.0):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (scale * torch.randn(*shape, generator=gen, device="cuda")).to(_dt(dtype))


def _exp2(n):
    import torch
    return ((n.long() + 1023) << 52).view(torch.float64)


def _definition(x):
    """(values, exponents) of finite x [T, C] in 64 bits: the least e in -100 .. 119 with max |x| <= 448
    2^e; values rounded to nearest even with three mantissa bits, at least 2^-9 apart, at most 448."""
    import torch
    x = x.double()
    T, C = x.shape
    groups = -(-T // 32)
    p = torch.zeros(groups * 32, C, dtype=torch.float64, device=x.device)
    p[:T] = x
    p = p.view(groups, 32, C)
    top = p.abs().amax(1)
    e = torch.full_like(top, -100).long()
    for k in range(-100, 119):
        e = torch.where(top > 448.0 * 2.0 ** k, k + 1, e)
    v = (p / _exp2(e)[:, None]).clamp(-448.0, 448.0)
    step = _exp2((torch.frexp(v)[1] - 4).clamp_min(-9))
    return (torch.round(v / step) * step * _exp2(e)[:, None]).view(-1, C)[:T], e


def _data(T, C, dtype, kind, seed):
    import torch
    x = _rand((T, C), "f32", seed)
    gen = torch.Generator(device="cuda").manual_seed(seed + 1)
    if kind == "wide":  # every binade, zeros among them
        x = x * _exp2(torch.randint(-120, 120, (T, C), generator=gen, device="cuda")).float()
        x[torch.rand(T, C, generator=gen, device="cuda") < 0.2] = 0.0
        x[:, ::7] = 0.0
    if kind == "edges":  # halfway between codes, at the ends of an exponent's range
        pick = torch.tensor([448.0, 449.0, 464.0, 255.0, 17.0, 19.0, 1.0625, 0.0009765625, 0.0029296875, 3.0e38, 1e-38, -1.0],
                            device="cuda")
        x = pick[torch.randint(0, 12, (T, C), generator=gen, device="cuda")]
    return x.to(_dt(dtype))


SIZES = [(1, 1), (31, 5), (32, 64), (33, 257), (100, 1003), (777, 130), (64, 4096)]


@pytest.mark.parametrize("T,C", SIZES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["gauss", "wide", "edges"])
def test_pack_and_unpack(T, C, dtype, kind):
    import torch
    x = _data(T, C, dtype, kind, 3)
    print(f"[gpu-case] act_pack {T} {C} {dtype} {kind}", flush=True)
    codes, exps = hm.act_pack(x)
    want, e = _definition(x)
    assert codes.shape == (-(-T // 32), C, 32) and torch.equal(exps.long() - 127, e)
    for out in ("f32", "bf16"):
        assert torch.equal(hm.act_unpack(codes, exps, T, dtype=_dt(out)).double(), want)
    # the values of the codes themselves, and zeros behind the last token
    v = codes.view(torch.float8_e4m3fn).double() * _exp2(exps.long() - 127)[:, :, None]
    v = v.transpose(1, 2).reshape(-1, C)
    assert torch.equal(v[:T], want) and bool((v[T:] == 0).all())


def test_strides_and_no_tokens():
    import torch
    x = _rand((70, 90), "bf16", 4)[:, 3:80]
    codes, exps = hm.act_pack(x)
    assert torch.equal(codes, hm.act_pack(x.contiguous())[0])
    space = torch.full((70, 100), 5.0, device="cuda")
    hm.act_unpack(codes, exps, 70, out=space[:, 1:78])
    assert torch.equal(space[:, 1:78].double(), _definition(x)[0])
    assert bool((space[:, 0] == 5).all()) and bool((space[:, 78:] == 5).all())
    codes, exps = hm.act_pack(x[:0])
    assert codes.shape == (0, 77, 32) and hm.act_unpack(codes, exps, 0).shape == (0, 77)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_infinities_and_nan_stay_where_they_are(dtype):
    import torch
    x = _rand((50, 40), dtype, 5)
    x[3, 7], x[40, 7], x[45, 8], x[0, 9] = float("nan"), float("inf"), -float("inf"), float("nan")
    bad = ~torch.isfinite(x)
    want, e = _definition(torch.where(bad, 0.0, x.double()))
    codes, exps = hm.act_pack(x)
    got = hm.act_unpack(codes, exps, 50, dtype=torch.float32).double()
    assert torch.equal(exps.long() - 127, e)
    assert bool(torch.isnan(got[bad]).all()) and torch.equal(got[~bad], want[~bad])


def _check_wgrad(got, grad, codes, exps, out, terms=1, base=None):
    import torch
    T = grad.shape[0]
    x = hm.act_unpack(codes, exps, T, dtype=torch.float32).double()
    g = grad.double()
    want, size = g.t().contiguous() @ x, g.abs().t().contiguous() @ x.abs()
    if base is not None:
        want, size = want + base.double(), size + base.double().abs()
    n = max(T, 1) * terms + 1
    err = (got.double() - want).abs()
    bound = n * 2 * U * size + ROUND[out] * want.abs()
    assert bool((err <= bound).all()), float((err - bound).max())
    assert float(err.norm()) <= (4 * n ** 0.5 * 2 * U + ROUND[out]) * max(float(want.norm()), 1e-300)


WSIZES = [(1, 1, 1), (5, 3, 70), (32, 64, 64), (33, 100, 31), (257, 130, 129), (1111, 1003, 777), (4096, 256, 128), (640, 515, 1028),
          (96, 2048, 1024), (20000, 72, 40)]


@pytest.mark.parametrize("T,O,C", WSIZES)
@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("f32", "bf16")])
def test_weight_gradient(T, O, C, dtype, out):
    import torch
    grad = _rand((T, O), dtype, 6, 1e-3)
    codes, exps = hm.act_pack(_data(T, C, "bf16", "gauss", 7))
    print(f"[gpu-case] weight_grad {T} {O} {C} {dtype} {out}", flush=True)
    got = hm.weight_grad(grad, codes, exps, dtype=_dt(out))
    _check_wgrad(got, grad, codes, exps, out, 3 if dtype == "f32" else 1)
    assert torch.equal(got, hm.weight_grad(grad, codes, exps, dtype=_dt(out)))  # the same from call to call


# every kernel that serves larger results, whole and cut: two groups of waves to a tile, split
# or not; 128-tiles; 256-tiles, split or not
LARGE = [(300, 1500, 2100), (512, 2048, 2048), (9000, 700, 1000), (4100, 1024, 1096), (200, 3000, 2200), (256, 4096, 2304),
         (1100, 3300, 3000), (1024, 3328, 3328), (8200, 4000, 2040)]


@pytest.mark.parametrize("T,O,C", LARGE)
@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
def test_large_weight_gradient(T, O, C, dtype, out):
    import torch
    grad = _rand((T, O), dtype, 23, 1e-3)
    codes, exps = hm.act_pack(_data(T, C, "bf16", "gauss", 24))
    print(f"[gpu-case] weight_grad {T} {O} {C} {dtype} {out}", flush=True)
    got = hm.weight_grad(grad, codes, exps, dtype=_dt(out))
    _check_wgrad(got, grad, codes, exps, out, 3 if dtype == "f32" else 1)
    assert torch.equal(got, hm.weight_grad(grad, codes, exps, dtype=_dt(out)))


@pytest.mark.parametrize("T,O,C", [(300, 1500, 2100), (9000, 700, 1000), (200, 3000, 2200), (1100, 3300, 3000)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_weight_gradient_strides_and_accumulation(T, O, C, dtype):
    import torch
    for cut in (1, 8):
        grad = _rand((T, O + 16), dtype, 25)[:, cut:cut + O]
        codes, exps = hm.act_pack(_data(T, C, "bf16", "gauss", 26))
        space = _rand((O, C + 9), "f32", 27)
        before = space.clone()
        view = space[:, 2:2 + C]
        hm.weight_grad(grad, codes, exps, out=view, accumulate=True)
        assert torch.equal(space[:, :2], before[:, :2]) and torch.equal(space[:, 2 + C:], before[:, 2 + C:])
        _check_wgrad(view, grad, codes, exps, "f32", 3 if dtype == "f32" else 1, base=before[:, 2:2 + C])


@pytest.mark.parametrize("T,O,C", [(300, 1500, 2104), (200, 3000, 2200), (1100, 3304, 3000)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_weight_gradient_infinities_and_nan(T, O, C, dtype):
    """As below, where the last group of tokens is cut."""
    import torch
    grad, x = _rand((T, O), dtype, 28), _rand((T, C), "bf16", 29)
    x[T - 1] = x[T - 1].abs() + 0.5
    x[T - 1, ::2] *= -1
    clean = hm.weight_grad(grad, *hm.act_pack(x), dtype=torch.float32)
    x2, g2 = x.clone(), grad.clone()
    g2[T - 1, 9] = float("inf")
    g2[0, 777] = float("nan")
    x2[2, 33] = float("nan")
    got = hm.weight_grad(g2, *hm.act_pack(x2), dtype=torch.float32)
    cols = torch.arange(C, device="cuda") != 33
    rows = torch.ones(O, dtype=torch.bool, device="cuda")
    rows[9] = rows[777] = False
    assert torch.equal(got[9][cols], (x2[T - 1].float() * float("inf"))[cols])
    assert bool(torch.isnan(got[:, 33]).all()) and bool(torch.isnan(got[777]).all())
    assert torch.equal(got[rows][:, cols], clean[rows][:, cols])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_weight_gradient_strides_and_accumulation(dtype):
    """Rows of the gradient and of the result at any address; added to what is there."""
    import torch
    for T, O, C, cut in ((300, 200, 136, 1), (300, 200, 136, 8), (95, 77, 45, 3)):
        grad = _rand((T, O + 16), dtype, 8)[:, cut:cut + O]
        codes, exps = hm.act_pack(_data(T, C, "bf16", "gauss", 9))
        for out in ("f32", "bf16"):
            space = _rand((O, C + 9), out, 10)
            before = space.clone()
            view = space[:, 2:2 + C]
            hm.weight_grad(grad, codes, exps, out=view, accumulate=True)
            assert torch.equal(space[:, :2], before[:, :2]) and torch.equal(space[:, 2 + C:], before[:, 2 + C:])
            _check_wgrad(view, grad, codes, exps, out, 3 if dtype == "f32" else 1, base=before[:, 2:2 + C])
            hm.weight_grad(grad, codes, exps, out=view)
            _check_wgrad(view, grad, codes, exps, out, 3 if dtype == "f32" else 1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [40, 64, 3000])
def test_weight_gradient_infinities_and_nan_stay_in_their_row_or_column(dtype, T):
    """The last token's gradient (beside the empty places of a last group) infinite in
    one row: infinities of the input's signs; a NaN in one column of the input."""
    import torch
    O, C = 70, 50
    grad, x = _rand((T, O), dtype, 11), _rand((T, C), "bf16", 12)
    x[T - 1] = x[T - 1].abs() + 0.5
    x[T - 1, ::2] *= -1
    clean = hm.weight_grad(grad, *hm.act_pack(x), dtype=torch.float32)
    x2, g2 = x.clone(), grad.clone()
    g2[T - 1, 9] = float("inf")
    x2[2, 33] = float("nan")
    got = hm.weight_grad(g2, *hm.act_pack(x2), dtype=torch.float32)
    ref = x2[T - 1].float() * float("inf")
    cols = torch.arange(C, device="cuda") != 33
    rows = torch.arange(O, device="cuda") != 9
    assert torch.equal(got[9][cols], ref[cols])
    assert bool(torch.isnan(got[:, 33]).all())
    assert torch.equal(got[rows][:, cols], clean[rows][:, cols])


def test_past_32_bits():
    """Activations, codes and gradients of more than 2^31 elements."""
    import torch
    T, C = 66000, 33000
    x = torch.empty(T, C, dtype=torch.bfloat16, device="cuda")
    x[:64] = _rand((64, C), "bf16", 40)
    for i in range(64, T, 6000):
        x[i:i + 6000] = x[(i // 64) % 7]
    x[T - 90:] = _rand((90, C), "bf16", 41)
    codes, exps = hm.act_pack(x)
    last = hm.act_pack(x[T - T % 32 - 64:].contiguous())
    assert torch.equal(codes[-3:], last[0]) and torch.equal(exps[-3:], last[1])
    back = hm.act_unpack(codes, exps, T)
    assert torch.equal(back[T - 40:], hm.act_unpack(*last, T % 32 + 64)[-40:])
    del back
    # the gradient's last columns, and the input's, alone
    small = _rand((T, 40), "bf16", 42, 1e-3)
    packed = hm.act_pack(small)
    wide = hm.weight_grad(x, *packed, dtype=torch.float32)  # x as the gradient
    _check_wgrad(wide[-33:], x[:, -33:], *packed, "f32")
    tall = hm.weight_grad(small, codes, exps, dtype=torch.float32)
    part = (codes[:, -50:].contiguous(), exps[:, -50:].contiguous())
    _check_wgrad(tall[:, -50:], small, *part, "f32")


def test_weight_gradient_extreme_values():
    """fp32 gradients near the ends of the range: no term overflows on the way."""
    import torch
    T, O, C = 64, 40, 36
    grad = torch.zeros(T, O, device="cuda")
    grad[7] = 3.4e38
    grad[9, ::2] = 1e-30
    x = torch.zeros(T, C, device="cuda", dtype=torch.bfloat16)
    x[7] = 0.25
    codes, exps = hm.act_pack(x)
    got = hm.weight_grad(grad, codes, exps)
    assert torch.equal(got, (grad[7].double()[:, None] * x[7].double()[None]).float())


def test_weight_gradient_of_no_tokens():
    import torch
    g = torch.empty(0, 10, device="cuda")
    codes, exps = hm.act_pack(torch.empty(0, 7, device="cuda"))
    out = torch.ones(10, 7, device="cuda")
    hm.weight_grad(g, codes, exps, out=out, accumulate=True)
    assert bool((out == 1).all())
    hm.weight_grad(g, codes, exps, out=out)
    assert bool((out == 0).all())


def test_weight_gradient_against_differences():
    """A bilinear form: its change along a direction of the weights."""
    import torch
    T, O, C = 333, 64, 96
    grad, x, d = _rand((T, O), "f32", 13), _rand((T, C), "bf16", 14), _rand((O, C), "f32", 15)
    codes, exps = hm.act_pack(x)
    v = hm.act_unpack(codes, exps, T, dtype=torch.float32).double()
    y = v @ d.double().t().contiguous()  # the change of the layer's outputs along d
    along, size = (grad.double() * y).sum(), (grad.double().abs().t().contiguous() @ v.abs() * d.double().abs()).sum()
    inner = (hm.weight_grad(grad, codes, exps).double() * d.double()).sum()
    assert abs(float(along - inner)) <= (3 * T + 4) * 2 * U * float(size)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_streams_and_graph_replay(dtype):
    import torch
    for T, O, C in ((700, 320, 200), (4096, 128, 128)):
        grad, x = _rand((T, O), dtype, 16), _rand((T, C), "bf16", 17)
        want = hm.weight_grad(grad, *hm.act_pack(x))
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        packed = hm.act_pack(x, stream=side)
        got = hm.weight_grad(grad, *packed, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(want, got)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            packed = hm.act_pack(x)
            got = hm.weight_grad(grad, *packed)
            back = hm.act_unpack(*packed, T)
        for i in range(4):
            grad.copy_(_rand((T, O), dtype, 20 + i))
            x.copy_(_rand((T, C), "bf16", 30 + i))
            graph.replay()
            torch.cuda.synchronize()
            eager = hm.act_pack(x)
            assert torch.equal(got, hm.weight_grad(grad, *eager)) and torch.equal(back, hm.act_unpack(*eager, T))


def test_the_gradient_goes_into_the_optimizer():
    """weight_grad writes the buffer that HiMuon.step reads: the same step as from the
    product formed elsewhere with the same bits."""
    import torch
    T, O, C = 512, 256, 128
    grad, x = _rand((T, O), "bf16", 18), _rand((T, C), "bf16", 19)
    packed = hm.act_pack(x)
    w1 = _rand((O, C), "bf16", 20)
    w2, buf = w1.clone(), torch.empty_like(w1)
    a, b = hm.HiMuon([w1], T=128), hm.HiMuon([w2], T=128)
    hm.weight_grad(grad, *packed, out=buf)
    a.step([buf])
    b.step([hm.weight_grad(grad, *packed)])
    assert torch.equal(w1, w2) and bool(torch.isfinite(w1).all())


def test_refusals():
    import torch
    x = _rand((64, 32), "bf16", 21)
    codes, exps = hm.act_pack(x)
    for bad in (x.t(), x.cpu(), x[0]):
        with pytest.raises(ValueError):
            hm.act_pack(bad)
    with pytest.raises(TypeError):
        hm.act_pack(x.half())
    with pytest.raises(ValueError):
        hm.act_unpack(codes, exps, 65)
    with pytest.raises(ValueError):
        hm.act_unpack(codes, exps[:, :31], 64)
    with pytest.raises(ValueError):
        hm.act_unpack(codes.int(), exps, 64)
    g = _rand((64, 16), "bf16", 22)
    with pytest.raises(ValueError):
        hm.weight_grad(g[:32], codes, exps)
    with pytest.raises(ValueError):
        hm.weight_grad(g, codes, exps, accumulate=True)
    with pytest.raises(ValueError):
        hm.weight_grad(g, codes, exps, out=torch.empty(16, 31, device="cuda"))
    with pytest.raises(TypeError):
        hm.weight_grad(g.half(), codes, exps)
    with pytest.raises(hm.HimuonError) as e:
        hm.weight_grad(_rand((300, 1501), "bf16", 22), *hm.act_pack(_rand((300, 2100), "bf16", 22)),
                       workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    assert e.value.status == hm.ERR_WORKSPACE
