"""The training-step operators called for another stream than the current one: what they
allocate is that stream's memory. A block that the current stream has just given up, and
may still read, is not among it."""
import pytest

import paper_2606_27216_amd as hm

pytestmark = pytest.mark.gpu


def _calls():
    import torch
    r = lambda *s: torch.randn(*s, device="cuda").bfloat16()
    tokens, table, g = torch.randint(0, 500, (1024,), device="cuda"), r(500, 512), r(1024, 512)
    q, k, w, cos, sin = r(1, 256, 8, 64), r(1, 256, 2, 64), r(64), torch.rand(256, 32, device="cuda"), torch.rand(256, 32, device="cuda")
    codes, exps = hm.act_pack(g)
    return {"embed": lambda s: hm.embed(tokens, table, stream=s), "embed_grad": lambda s: hm.embed_grad(tokens, g, 500, stream=s),
            "qk": lambda s: hm.qk_norm_rope(q, k, w, w, cos, sin, stream=s),
            "qk_grad": lambda s: hm.qk_norm_rope_grad(q, k, q, k, w, w, cos, sin, stream=s),
            "pack": lambda s: hm.act_pack(g, stream=s), "unpack": lambda s: hm.act_unpack(codes, exps, 1024, stream=s),
            "weight_grad": lambda s: hm.weight_grad(g, codes, exps, stream=s)}


@pytest.mark.parametrize("name", ["embed", "embed_grad", "qk", "qk_grad", "pack", "unpack", "weight_grad"])
def test_memory_is_the_streams_own(name):
    import torch
    print(f"[gpu-case] {name} on another stream", flush=True)
    call, side = _calls()[name], torch.cuda.Stream()
    several = lambda r: r if isinstance(r, tuple) else (r,)
    want = [t.clone() for t in several(call(None))]
    torch.cuda.synchronize()
    given_up = [torch.empty_like(t) for t in want]
    blocks = {t.data_ptr() for t in given_up}
    del given_up
    got = several(call(side))
    assert not blocks & {t.data_ptr() for t in got}
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert torch.cuda.current_stream() != side
