"""weight_grad on the kernel of the largest results (256-tiles), with and without partial sums:
stores, cut tiles and a cut last group of tokens, several rounds over the chip, any row
stride, accumulation, infinities and NaN. Bounds as in test_gpu_act8; which kernel each of
these sizes runs on is held by test_wgrad_plan_cpu."""
import pytest
from test_gpu_act8 import _check_wgrad, _data, _dt, _rand

import paper_2606_27216_amd as hm

pytestmark = pytest.mark.gpu

# one round of tiles, the gradient read in place and laid out; three rounds
WHOLE = [(2100, 3104, 4100), (2101, 3100, 4103), (1911, 5000, 8101)]
SPLIT = [(8200, 4000, 2040), (8213, 4001, 2041)]  # two partial sums


@pytest.mark.parametrize("T,O,C", WHOLE + SPLIT)
@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("f32", "bf16")])
def test_weight_gradient(T, O, C, dtype, out):
    import torch
    grad = _rand((T, O), dtype, 50, 1e-3)
    codes, exps = hm.act_pack(_data(T, C, "bf16", "gauss", 51))
    print(f"[gpu-case] weight_grad {T} {O} {C} {dtype} {out}", flush=True)
    got = hm.weight_grad(grad, codes, exps, dtype=_dt(out))
    _check_wgrad(got, grad, codes, exps, out, 3 if dtype == "f32" else 1)
    assert torch.equal(got, hm.weight_grad(grad, codes, exps, dtype=_dt(out)))


@pytest.mark.parametrize("T,O,C", WHOLE[:2] + SPLIT)
@pytest.mark.parametrize("dtype,out", [("bf16", "f32"), ("bf16", "bf16"), ("f32", "f32")])
def test_strides_and_accumulation(T, O, C, dtype, out):
    """Rows of the gradient that start on 16 bytes and that do not, into rows with a stride."""
    import torch
    for cut in (1, 8):
        pitch = (O + 23) // 8 * 8
        grad = _rand((T, pitch), dtype, 52)[:, cut:cut + O]
        codes, exps = hm.act_pack(_data(T, C, "bf16", "gauss", 53))
        print(f"[gpu-case] weight_grad {T} {O} {C} {dtype} {out} cut {cut}", flush=True)
        space = _rand((O, C + 9), out, 54)
        before = space.clone()
        view = space[:, 2:2 + C]
        hm.weight_grad(grad, codes, exps, out=view, accumulate=True)
        assert torch.equal(space[:, :2], before[:, :2]) and torch.equal(space[:, 2 + C:], before[:, 2 + C:])
        _check_wgrad(view, grad, codes, exps, out, 3 if dtype == "f32" else 1, base=before[:, 2:2 + C])


@pytest.mark.parametrize("T,O,C", WHOLE[:2] + SPLIT)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_infinities_and_nan_stay_in_their_row_or_column(T, O, C, dtype):
    """In the last group of tokens, which is cut, and in the first."""
    import torch
    grad, x = _rand((T, O), dtype, 55), _rand((T, C), "bf16", 56)
    x[T - 1] = x[T - 1].abs() + 0.5
    x[T - 1, ::2] *= -1
    print(f"[gpu-case] weight_grad {T} {O} {C} {dtype} infinities", flush=True)
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
