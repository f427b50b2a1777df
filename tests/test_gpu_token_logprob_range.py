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
