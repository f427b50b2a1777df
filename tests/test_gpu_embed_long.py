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


# around the lengths at which the sort changes, whole and cut parts of 1024, one digit and two
# (1023 and 1024 rows), and a table whose zeros are set by smaller blocks
@pytest.mark.parametrize("n,rows,width,kind", [(4096, 50000, 24, "uniform"), (4097, 50000, 24, "uniform"), (5120, 1024, 24, "few"),
                                               (5121, 1023, 24, "few"), (5121, 1024, 24, "few"), (7000, 3000, 72, "one"),
                                               (9000, 2000, 8, "none"), (33333, 130000, 16, "uniform"), (49151, 1500, 8, "few"),
                                               (49152, 50000, 8, "uniform"), (49153, 50000, 8, "uniform"),
                                               (20000, 55000, 1000, "few")])
def test_lengths_of_each_sort(n, rows, width, kind):
    import torch
    print(f"[gpu-case] embed_grad {n} {rows} {width} {kind}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(n + rows)
    tokens = torch.randint(-(rows // 9), rows + rows // 9 + 1, (n,), generator=gen, device="cuda")
    if kind == "one":
        tokens[::3] = rows // 2
    elif kind == "few":
        tokens = torch.where(torch.rand(n, generator=gen, device="cuda") < 0.7, tokens % 11, tokens)
    elif kind == "none":
        tokens = torch.full_like(tokens, rows)
    grad = torch.randint(-8, 9, (n, width), generator=gen, device="cuda").bfloat16()
    want = _want(tokens, grad, rows)
    got = hm.embed_grad(tokens, grad, rows, dtype=torch.float32)
    assert torch.equal(got.long(), want)
    wide = torch.full((rows, width + 5), 3.0, device="cuda")
    out = hm.embed_grad(tokens.int(), grad.float(), rows, scale=2.0, out=wide[:, 2:2 + width])
    assert torch.equal(out, 2 * got) and bool((wide[:, :2] == 3).all()) and bool((wide[:, 2 + width:] == 3).all())
    assert torch.equal(hm.embed_grad(tokens, grad, rows, out=got.clone(), accumulate=True), 2 * got)
