"""attention and its gradient against the definition in 64 bits where a wave has 32 rows of its own and
walks over many tiles of the other side: the kernels of large batches, in every form that they have (heads
of 64, 128 and 256 columns, whole and cut; aligned or not; heads to a group). Tolerances are
test_gpu_attention's."""
import math

import pytest

torch = pytest.importorskip("torch")
import paper_2606_27216_amd as hm
from test_gpu_attention import check, make

pytestmark = pytest.mark.gpu

# (batch, queries, keys, heads, key heads, head, type, layout)
BATCHES = [
    # whole heads, aligned: tiles by DMA, many of them on their way
    (5, 520, 520, 8, 4, 64, "bf16", "tokens"), (5, 520, 520, 8, 4, 128, "bf16", "heads"), (5, 520, 520, 8, 4, 256, "bf16", "tokens"),
    (13, 520, 520, 16, 8, 64, "f32", "heads"), (13, 520, 520, 16, 8, 128, "f32", "tokens"), (13, 520, 520, 16, 8, 256, "f32", "tokens"),
    # one, three and forty heads to a group; sides of different lengths
    (10, 700, 333, 4, 4, 128, "bf16", "fused"), (12, 333, 700, 9, 3, 128, "bf16", "tokens"), (20, 130, 640, 40, 1, 64, "bf16", "tokens"),
    (22, 1025, 333, 8, 8, 64, "f32", "tokens"), (33, 333, 700, 9, 3, 128, "f32", "tokens"),
    (12, 400, 333, 6, 3, 256, "bf16", "heads"), (60, 333, 520, 3, 3, 256, "f32", "heads"),
    # heads that are no whole tile, and rows that are not aligned
    (6, 520, 520, 8, 4, 80, "bf16", "tokens"), (5, 520, 520, 8, 4, 200, "bf16", "tokens"), (13, 520, 520, 16, 8, 80, "f32", "tokens"),
    (13, 333, 520, 16, 8, 136, "f32", "tokens"), (6, 520, 520, 8, 4, 64, "bf16", "odd"), (5, 520, 520, 8, 4, 128, "bf16", "odd"),
    (12, 333, 333, 9, 3, 256, "bf16", "odd"), (13, 520, 520, 16, 8, 64, "f32", "odd"), (20, 520, 260, 18, 9, 128, "f32", "odd"),
    (13, 520, 520, 8, 8, 256, "f32", "odd"),
]

# (starts, tokens, heads, key heads, head, type)
PACKED = [
    ([0, 700, 700, 1300, 1333, 3000], 3040, 8, 4, 128, "bf16"), ([10, 1010, 2600], 2600, 15, 5, 64, "bf16"),
    ([0, 1500, 2300, 2400], 2410, 10, 5, 256, "bf16"), ([0, 3000, 3001, 4100, 7000], 7000, 18, 9, 128, "f32"),
    ([5, 2500, 6900], 7000, 9, 9, 64, "f32"), ([0, 1500, 3300, 6900], 7000, 9, 9, 256, "f32"),
]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("case", BATCHES, ids=str)
def test_batches(case, causal):
    print("[gpu-case] attention tiles", case, causal, flush=True)
    batch, nq, nk, hq, hk, dim, dtype, layout = case
    check(*make((batch,), nq, nk, hq, hk, dim, dtype, layout, dim), causal=causal)


@pytest.mark.parametrize("case", BATCHES[:13], ids=str)
def test_padded_batches(case):
    """Lengths from none to all, a part of them long: the last whole tile of either side anywhere."""
    print("[gpu-case] attention tiles padded", case, flush=True)
    batch, nq, nk, hq, hk, dim, dtype, layout = case
    q, k, v, g = make((batch,), nq, nk, hq, hk, dim, dtype, layout, dim + 1)
    gen = torch.Generator(device="cuda").manual_seed(batch)
    n, m = (torch.randint(c // 2, c + 1, (batch,), generator=gen, device="cuda") for c in (nq, nk))
    n[1], m[2] = 0, 0
    n[3], m[3] = nq, nk
    out, lse, _ = check(q, k, v, g, q_lengths=n, k_lengths=m)
    grads = hm.attention_grad(g, q, k, v, out, lse, q_lengths=n, k_lengths=m)
    # tokens that are not in use are not read, whatever they hold
    off = [torch.arange(c, device="cuda")[None] >= x[:, None] for c, x in ((nq, n), (nk, m))]
    dirty = [t.clone() for t in (q, k, v, g, out)]
    for t, i, x in zip(dirty, (0, 1, 1, 0, 0), (math.nan, math.inf, math.nan, -math.inf, math.nan)):
        t[off[i]] = x
    again = hm.attention(*dirty[:3], q_lengths=n, k_lengths=m)
    assert torch.equal(again[0], out) and torch.equal(again[1], lse)
    for a, b in zip(hm.attention_grad(dirty[3], *dirty[:3], dirty[4], lse, q_lengths=n, k_lengths=m), grads):
        assert torch.equal(a, b)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("case", PACKED, ids=str)
def test_packed(case, causal):
    print("[gpu-case] attention tiles packed", case, causal, flush=True)
    starts, tokens, hq, hk, dim, dtype = case
    s = torch.tensor(starts, dtype=torch.int32, device="cuda")
    check(*make((), tokens, tokens, hq, hk, dim, dtype, "tokens", tokens), causal=causal, q_starts=s)
