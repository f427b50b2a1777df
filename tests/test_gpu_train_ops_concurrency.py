"""The training-step operators from several host threads, each on its own stream and its own
data: the results are, bit for bit, those of the same calls made alone."""
import threading

import pytest

import paper_2606_27216_amd as hm

pytestmark = pytest.mark.gpu


def _data(seed):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda").bfloat16()
    return {"tokens": torch.randint(-1, 500, (7000,), generator=gen, device="cuda"), "g": r(7000, 264), "few": r(90, 264),
            "q": r(2, 200, 12, 128), "k": r(2, 200, 2, 128), "w": r(128), "x": r(1000, 1500), "dy": r(1000, 2100), "small": r(1000, 72),
            "cos": torch.rand(200, 64, generator=gen, device="cuda"), "sin": torch.rand(200, 64, generator=gen, device="cuda")}


def _calls(d, stream):
    args = (d["q"], d["k"], d["w"], d["w"], d["cos"], d["sin"])
    out = [hm.embed(d["tokens"], d["few"], scale=2.0, stream=stream), hm.embed_grad(d["tokens"], d["g"], 500, stream=stream),
           hm.embed_grad(d["tokens"][:90], d["few"], 500, stream=stream)]
    out += hm.qk_norm_rope(*args, stream=stream)
    out += hm.qk_norm_rope_grad(d["q"], d["k"], *args, stream=stream)
    packed = hm.act_pack(d["x"], stream=stream)
    out += [*packed, hm.act_unpack(*packed, 1000, stream=stream), hm.weight_grad(d["dy"], *packed, stream=stream),
            hm.weight_grad(d["small"], *packed, stream=stream), hm.weight_grad(d["dy"].float(), *packed, stream=stream)]
    return out


def test_threads_on_their_own_streams_match_single_calls():
    import torch
    print("[gpu-case] training-step operators from four threads", flush=True)
    data = [_data(60 + i) for i in range(4)]
    torch.cuda.synchronize()
    want = [_calls(d, None) for d in data]
    torch.cuda.synchronize()
    bad = []

    def work(i):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                for _ in range(5):
                    got = _calls(data[i], stream)
                    stream.synchronize()
                    if not all(torch.equal(a, b) for a, b in zip(got, want[i])):
                        bad.append(i)
        except Exception as e:  # reported below
            bad.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad, bad
