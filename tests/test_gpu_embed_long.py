"""embed_grad of long batches, where the tiles' counts of the sort are added up in a
launch of their own. Gradients are whole numbers and small, so that every sum in fp32 is
exact and has to be equal."""
import pytest

import paper_2606_27216_amd as hm

pytestmark = pytest.mark.gpu


def _want(tokens, grad, rows):
    import torch
    ok = (tokens >= 0) & (tokens < rows)
    return torch.zeros(rows, grad.shape[1], dtype=torch.int64, device="cuda").index_add_(0, tokens[ok].long(), grad[ok].long())


# around the last length without that launch, one digit to three, few bins, a whole number of tiles
@pytest.mark.parametrize("n,rows,width,kind", [(98304, 777, 24, "uniform"), (98305, 777, 24, "uniform"), (99001, 3, 40, "uniform"),
                                               (131072, 50000, 16, "uniform"), (200003, 1500000, 8, "uniform"),
                                               (300001, 1000, 520, "one"), (1000003, 33000, 8, "few"), (150000, 1, 9, "none")])
def test_long_batches(n, rows, width, kind):
    import torch
    print(f"[gpu-case] embed_grad {n} {rows} {width} {kind}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(n)
    tokens = torch.randint(-(rows // 9), rows + rows // 9 + 1, (n,), generator=gen, device="cuda")
    if kind == "one":
        tokens[::3] = rows // 2
    elif kind == "few":
        tokens = torch.where(torch.rand(n, generator=gen, device="cuda") < 0.9, tokens % 7, tokens)
    elif kind == "none":
        tokens = torch.full_like(tokens, -1)
    grad = torch.randint(-8, 9, (n, width), generator=gen, device="cuda").bfloat16()
    got = hm.embed_grad(tokens, grad, rows, dtype=torch.float32)
    assert torch.equal(got.long(), _want(tokens, grad, rows))
    assert torch.equal(hm.embed_grad(tokens.int(), grad, rows, out=got.clone(), accumulate=True), 2 * got)
