"""The operators of a decoder block together, as a training step uses them: against the same
model in torch's own operations, on other streams, in captured graphs and from several threads."""
import importlib.util
import os
import threading

import pytest

torch = pytest.importorskip("torch")
import paper_2606_27216_amd as hm

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("train_block", os.path.join(ROOT, "examples", "train_block.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_the_examples_gradients_are_a_plain_models():
    """Inputs held in 8 bits (3 mantissa bits: 2^-4 of a value at most, 2^-5.8 in the mean
    square) and bf16 roundings on other paths leave the directions within a few percent."""
    print("[gpu-case] block plain", flush=True)
    ex = _example()
    tokens = ex.Walks(4).batch()

    class Plain(ex.Block):
        def linear(self, name, x):
            return x @ self.weights[name].t()

        def embed(self, tokens):
            return self.table[tokens] * ex.math.sqrt(ex.WIDTH)

        def norm_rope(self, q, k):
            out = []
            for x, w in ((q, self.gains[0]), (k, self.gains[1])):
                x = x.float()
                a, b = (x * torch.rsqrt(x.pow(2).mean(-1, keepdim=True) + ex.EPS) * w).chunk(2, -1)
                c, s = self.cos[None, :, None], self.sin[None, :, None]
                out.append(torch.cat([a * c - b * s, b * c + a * s], -1).bfloat16())
            return out

        def add_norm(self, x, residual, i):
            h = x if residual is None else x + residual
            f = h.float()
            return h, (f * torch.rsqrt(f.pow(2).mean(-1, keepdim=True) + ex.EPS) * self.norm_gains[i]).bfloat16()

        def attention(self, q, k, v):
            q, k, v = (t.float().transpose(1, 2) for t in (q, k, v))
            k, v = (t.repeat_interleave(ex.HEADS // ex.KV_HEADS, 1) for t in (k, v))
            s = q @ k.transpose(-1, -2).contiguous() / ex.HEAD ** 0.5
            mask = torch.ones(s.shape[-2:], dtype=torch.bool, device=s.device).tril()
            return (s.masked_fill(~mask, float("-inf")).softmax(-1) @ v).transpose(1, 2).bfloat16()

        def logprob(self, logits, tokens):
            lp = torch.log_softmax(logits.float(), -1).gather(-1, tokens.clamp(0)[..., None])[..., 0]
            return lp * (tokens >= 0)

    def run(block):
        loss = block.loss(tokens)
        loss.backward()
        return loss.detach()
    block, plain = ex.Block(3), Plain(3)
    for w in plain.weights.values():
        w.requires_grad_()
    got, want = run(block), run(plain)
    assert abs(float(got - want)) < 2e-2 * float(want)
    pairs = [(block.grads[n], plain.weights[n].grad) for n in block.grads] + [(block.table.grad, plain.table.grad)]
    pairs += [(a.grad, b.grad) for a, b in zip(block.gains + block.norm_gains, plain.gains + plain.norm_gains)]
    for a, b in pairs:
        a, b = a.double().flatten(), b.double().flatten()
        assert float(a @ b / (a.norm() * b.norm())) > 0.99
        assert abs(float(a.norm() / b.norm()) - 1) < 0.05


def chain(st):
    """norm, attention, norm with 8-bit output, loss, and all the backward passes."""
    x, res, w, q, k, v, g, starts, logits, tokens, gl = st
    h, y, codes, exps = hm.add_norm(x, res, w, pack=True)
    out, lse = hm.attention(q, k, v, q_starts=starts)
    few, few_lse = hm.attention(q[None, :1], k[None], v[None])
    lp = hm.token_logprob(logits, tokens, top=7)
    return (h, y, codes, exps, out, lse, few, few_lse, *lp, *hm.add_norm_grad(y, h, w, g_h=res),
            *hm.attention_grad(g, q, k, v, out, lse, q_starts=starts),
            hm.token_logprob_grad(gl, gl, logits, tokens, lp[2], lp[1]))


def state(seed, dtype):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def r(*shape):
        return torch.randn(*shape, generator=gen, device="cuda").to(dtype)
    cut = torch.tensor([0, 70 + seed, 300, 511], device="cuda")
    t = torch.randint(-1, 3000, (90,), generator=gen, device="cuda")
    return [r(200, 1500), r(200, 1500), r(1500).float(), r(512, 8, 64), r(512, 2, 64), r(512, 2, 64), r(512, 8, 64), cut, r(90, 3000), t,
            r(90).float()]


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b)) and len(a) == len(b)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_other_streams(dtype):
    print("[gpu-case] block streams", dtype, flush=True)
    st = state(1, dtype)
    want = chain(st)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = chain(st)
    side.synchronize()
    assert same(got, want)
    side.wait_stream(torch.cuda.current_stream())
    a = hm.attention(*st[3:6], q_starts=st[7], stream=side)
    b = hm.add_norm(st[0], st[1], st[2], pack=True, stream=side)
    c = hm.token_logprob(st[8], st[9], top=7, stream=side)
    d = hm.attention_grad(st[6], *st[3:6], want[4], want[5], q_starts=st[7], stream=side)
    e = hm.add_norm_grad(want[1], want[0], st[2], g_h=st[1], stream=side)
    side.synchronize()
    assert same([*b, *a], want[:6]) and same(c, want[8:13]) and same([*e, *d], want[13:18])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_captured_and_replayed(dtype):
    """Two graphs, replayed in turn several times with eager work between, on inputs that change."""
    print("[gpu-case] block graphs", dtype, flush=True)
    states = [state(s, dtype) for s in (1, 2)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        chain(states[0])
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for st in states:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs = chain(st)
        graphs.append((g, outs, st))
    for turn in range(3):
        for g, outs, st in graphs:
            fresh = state(10 + turn, dtype)
            for a, b in zip(st, fresh):
                a.copy_(b)
            want = chain(fresh)
            g.replay()
            torch.cuda.synchronize()
            assert same(outs, want), turn


def test_from_several_threads():
    print("[gpu-case] block threads", flush=True)
    states = [state(s, torch.bfloat16) for s in range(4)]
    want = [chain(st) for st in states]
    torch.cuda.synchronize()
    got, errors = [None] * 4, []

    def work(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(10):
                    got[i] = chain(states[i])
                torch.cuda.current_stream().synchronize()
        except Exception as e:  # (reported below)
            errors.append(e)
    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors
    for a, b in zip(got, want):
        assert same(a, b)


def test_offsets_past_32_bits():
    """Rows whose elements lie beyond 2^32 bytes (and 2^31 elements): a cache of long sequences, wide logits."""
    print("[gpu-case] block far offsets", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(3)
    rows, vocab = 40000, 128000  # 10 GB of bf16
    logits = torch.empty(rows, vocab, dtype=torch.bfloat16, device="cuda")
    logits[-3:] = torch.randn(3, vocab, generator=gen, device="cuda").bfloat16()
    tokens = torch.full((rows,), -1, device="cuda")
    tokens[-3:] = torch.tensor([5, 100, 127999], device="cuda")
    got = hm.token_logprob(logits, tokens, top=3)
    want = hm.token_logprob(logits[-3:].clone(), tokens[-3:].clone(), top=3)
    for a, b in zip(got, want):
        assert torch.equal(a[-3:], b)
    ones = torch.ones(rows, device="cuda")
    d = hm.token_logprob_grad(ones, None, logits, tokens, got[2], got[1], out=logits)
    assert bool(d[-3:].isfinite().all()) and bool(d[-3:].any(1).all()) and bool((d[:5] == 0).all())
    del logits, d
    k = torch.empty(3, 150000, 8, 128 * 16, dtype=torch.bfloat16, device="cuda")[..., :128]  # tokens 32 KB apart: 4.9 GB to a sequence
    k[:, -200:] = torch.randn(3, 200, 8, 128, generator=gen, device="cuda").bfloat16()
    q = torch.randn(3, 200, 8, 128, generator=gen, device="cuda").bfloat16()
    s = torch.tensor([150000 - 200, 150000], device="cuda")
    a = hm.attention(q[2], k[2], k[2], q_starts=torch.tensor([0, 200], device="cuda"), k_starts=s)
    b = hm.attention(q[2], k[2, -200:].contiguous(), k[2, -200:].contiguous())
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    g = torch.randn(200, 8, 128, generator=gen, device="cuda").bfloat16()
    x = hm.attention_grad(g, q[2], k[2], k[2], *a, q_starts=torch.tensor([0, 200], device="cuda"), k_starts=s)
    near = k[2].contiguous()  # (as many tokens: the sums' order goes by the sizes)
    y = hm.attention_grad(g, q[2], near, near, *b, q_starts=torch.tensor([0, 200], device="cuda"), k_starts=s)
    for c, d in zip(x, y):
        assert torch.equal(c, d)
    assert not x[1][:-200].any()


def test_tensors_of_different_devices_or_shapes_are_refused():
    x, w = torch.zeros(4, 8, device="cuda"), torch.ones(8, device="cuda")
    q, k = torch.zeros(2, 4, 2, 8, device="cuda"), torch.zeros(2, 4, 1, 8, device="cuda")
    n = torch.tensor([4, 4], device="cuda")
    t = torch.zeros(4, dtype=torch.int64, device="cuda")
    f = torch.zeros(4, device="cuda")
    bad = [lambda: hm.add_norm(x, x[:2], w), lambda: hm.add_norm(x, x.bfloat16(), w), lambda: hm.add_norm(x, x, w[:4]),
           lambda: hm.add_norm(x, x, w.cpu()), lambda: hm.add_norm(x.t(), None, w[:4]), lambda: hm.add_norm(x, None, w, out=(x, x)),
           lambda: hm.add_norm_grad(x[:2], x, w), lambda: hm.attention(q, k, k[:1]), lambda: hm.attention(q, k[..., :4], k[..., :4]),
           lambda: hm.attention(k.expand(2, 4, 1, 8), q, q), lambda: hm.attention(q, k, k, q_starts=n),
           lambda: hm.attention(q, k, k, q_lengths=n[:1]), lambda: hm.attention(q, k, k, q_lengths=n, k_lengths=n.int()),
           lambda: hm.attention(q, k, k, q_lengths=n.cpu()), lambda: hm.attention(q[0], k[0][:3], k[0][:3], q_starts=n),
           lambda: hm.attention(q[0], k[0], k[0], k_starts=n), lambda: hm.token_logprob(x, t[:2]), lambda: hm.token_logprob(x, t, top=9),
           lambda: hm.token_logprob(x, t, top=-1), lambda: hm.token_logprob_grad(f[:2], None, x, t, f, f),
           lambda: hm.token_logprob_grad(f, f, x, t, f, None), lambda: hm.token_logprob_grad(f.double(), None, x, t, f, f)]
    for call in bad:
        with pytest.raises((ValueError, TypeError)):
            call()
    for call in (lambda: hm.add_norm(x.half(), None, w), lambda: hm.token_logprob(x, t.float()), lambda: hm.attention(q.half(), k.half(), k.half())):
        with pytest.raises((ValueError, TypeError)):
            call()
    with pytest.raises(hm.HimuonError):
        hm.attention(q, k, k, scale=-1.0)
    with pytest.raises(hm.HimuonError):
        hm.token_logprob(x, t, scale=0.0)
    with pytest.raises(hm.HimuonError):
        hm.attention(torch.zeros(1, 4, 1, 300, device="cuda"), *[torch.zeros(1, 4, 1, 300, device="cuda")] * 2)
