"""token_logprob and its gradient where sums or an lse are large, against 64 bits."""
import math

import pytest

torch = pytest.importorskip("torch")
import paper_2606_27216_amd as hm

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def test_a_row_of_more_masked_tokens_than_a_float_holds_times_their_distance():
    """Two tokens beside 2^29 of the type's lowest value: a distance of 3e38 and a count of 5e8 leave
    the entropy of the two."""
    print("[gpu-case] token_logprob wide masks", flush=True)
    vocab, last = 1 << 29, (1 << 29) - 8 * 512 + 3590  # (the last wave's, whose maximum is joined last)
    z = torch.full((1, vocab), torch.finfo(torch.bfloat16).min, dtype=torch.bfloat16, device="cuda")
    z[0, last], z[0, last + 1] = 2.0, 1.0
    got = hm.token_logprob(z, torch.tensor([last], device="cuda"))
    p = 1 / (1 + math.exp(-1.0))
    want = (math.log(p), -p * math.log(p) - (1 - p) * math.log(1 - p), 2.0 - math.log(p))
    for a, b in zip(got, want):  # (numbers of about one, some ten roundings)
        assert abs(float(a) - b) < 32 * U


@pytest.mark.parametrize("vocab", [40, 700, 9000, 33000])
@pytest.mark.parametrize("shift", [-900.0, -500.0, -60.0, 25.0, 40.0, 500.0, 1000.0])
def test_fp32_gradient_of_uncentred_logits(shift, vocab):
    """Logits far from zero: lse, given in fp32, is off by up to 2^-24 of itself, a probability by as
    much of its own size. Up to an lse of 32 that is 2^-20 and is granted; beyond, a probability is as near
    as the logits' distances make it. With D = |log p| + log(vocab): the distance, its product and the
    subtraction of the sum's logarithm 4 U D; the sum vocab / 256 U (a thread's terms) and 8 U (the tree); the
    exponentials in it, by their weights, 32 U; its logarithm (below 16, one step of 2^-20) 12 U; the last
    exponential 4 U: 56, say 64 U."""
    print("[gpu-case] token_logprob_grad uncentred", shift, vocab, flush=True)
    gen = torch.Generator(device="cuda").manual_seed(vocab)
    rows = 6
    z = torch.randn(rows, vocab, generator=gen, device="cuda") * 2 + shift
    t = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
    _, entropy, lse = hm.token_logprob(z, t)
    gl, gh = (torch.randn(rows, generator=gen, device="cuda") for _ in range(2))
    lp = torch.log_softmax(z.double(), 1)
    p, E = lp.exp(), entropy.double()[:, None]
    delta = torch.zeros_like(p).scatter_(1, t[:, None], 1.0)
    D = lp.abs() + math.log(vocab)
    e = 4 * U * D + (vocab / 256 + 64) * U + 2.0 ** -20
    for a, b in ((gl, None), (gl, gh)):
        d = hm.token_logprob_grad(a, b, z, t, lse, entropy)
        A, B = (0.0 if x is None else x.double()[:, None] for x in (a, b))
        want = A * (delta - p) - B * p * (lp + E)
        size = abs(A) * (p * e + (delta + p) * 4 * U) + abs(B) * p * ((lp.abs() + E) * (e + 6 * U) + e)
        off = (d.double() - want).abs()
        assert bool((off <= size + want.abs() * U + 1e-37).all()), f"worst {float((off / (size + want.abs() * U + 1e-37)).max()):.3g} times the tolerance"
