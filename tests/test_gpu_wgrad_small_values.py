"""weight_grad of gradients near the small end of their type.

A bf16 gradient is an operand as it stands, subnormal or not. An fp32 one is cut into three
bf16 terms: all of its bits from 2^-133 on count, so an element from 2^-110 on is exact and a
smaller one off by less than 2^-133. The rest of the bound is test_gpu_act8's, and the last
bit of fp32 (2^-149) for every term and rounding."""
import pytest
from test_gpu_act8 import _exp2, _rand

import paper_2606_27216_amd as hm

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def _gradient(T, O, low, high, dtype, seed):
    """Values of full precision in the binades low .. high of each column, of either sign."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    m = 1.0 + torch.randint(0, 1 << 23, (T, O), generator=gen, device="cuda").double() * 2.0 ** -23
    e = torch.randint(low, high + 1, (T, O), generator=gen, device="cuda")
    sign = torch.randint(0, 2, (T, O), generator=gen, device="cuda") * 2 - 1
    return (sign * m * _exp2(e)).to({"f32": torch.float32, "bf16": torch.bfloat16}[dtype])


@pytest.mark.parametrize("T,O,C", [(64, 40, 36), (300, 1500, 2100), (200, 3000, 2200), (2101, 3100, 4103)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("low,high", [(-110, -100), (-126, -111), (-140, -127)])
def test_small_gradients(T, O, C, dtype, low, high):
    import torch
    grad = _gradient(T, O, low, high, dtype, 70)
    x = (_rand((T, C), "f32", 71) * 2.0 ** 40).bfloat16()
    codes, exps = hm.act_pack(x)
    print(f"[gpu-case] weight_grad {T} {O} {C} {dtype} 2^{low} .. 2^{high}", flush=True)
    got = hm.weight_grad(grad, codes, exps, dtype=torch.float32).double()
    v = hm.act_unpack(codes, exps, T, dtype=torch.float32).double()
    want, size = grad.double().t().contiguous() @ v, grad.double().abs().t().contiguous() @ v.abs()
    n = T * (3 if dtype == "f32" else 1) + 1
    bound = n * 2 * U * size + 2 * U * want.abs() + n * 2.0 ** -149
    if dtype == "f32" and low < -110:
        bound += 2.0 ** -133 * v.abs().sum(0)
    err = (got - want).abs()
    assert bool((err <= bound).all()), float((err - bound).max())
    if high < -126 and dtype == "bf16":
        assert bool((want != 0).any()) and bool((got != 0).any())  # subnormal operands count
