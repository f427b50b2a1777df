"""The operators that a decoder block's training step needs beside those of
``perf/operators.py``, as they are measured: what each of them computes, the calls that
users make, their inputs and their work.

A case is a dict of plain values. "op" is the operator:

    norm          the residual's addition and the norm of the sum ("pack": in 8 bits too)
    norm_grad     its backward pass
    attn          attention, grouped heads, causal or not
    attn_grad     its backward pass
    logprob       log probabilities of given tokens, entropies, most likely tokens
    logprob_grad  their backward pass

"dtype" is the storage type ("f32", "bf16"). Widths, head counts and token counts are
those of this repository's workloads (the 7B-style layer, the Qwen3 blocks, batches of
16 x 1024 tokens a GPU) or generic.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}
EPS = 1e-6
GROUP = 32  # tokens of a column that share an exponent


def _norm(name, tokens, width, dtype, gain, residual=True, pack=False):
    return {"name": name, "op": "norm", "tokens": tokens, "width": width, "dtype": dtype, "gain": gain, "residual": residual,
            "pack": pack}


def _norm_grad(name, tokens, width, dtype, gain, residual=True):
    return {"name": name, "op": "norm_grad", "tokens": tokens, "width": width, "dtype": dtype, "gain": gain,
            "residual": residual}


def _attn(name, op, form, batch, seq, keys, heads, kv_heads, dim, dtype, causal=True, layout="tokens"):
    return {"name": name, "op": op, "form": form, "batch": batch, "seq": seq, "keys": keys, "heads": heads,
            "kv_heads": kv_heads, "dim": dim, "dtype": dtype, "causal": causal, "layout": layout}


def _logprob(name, op, tokens, vocab, dtype, ids="drawn", top=0, entropy=True, scale=1.0):
    return {"name": name, "op": op, "tokens": tokens, "vocab": vocab, "dtype": dtype, "ids": ids, "top": top,
            "entropy": entropy, "scale": scale}


def listed():
    return [
        # generation while a run is evaluated: one token of each of 32 sequences
        _norm("norm_decode_32x4096", 32, 4096, "bf16", "bf16"),
        # a training batch of 16 x 1024 tokens; the norm's output is kept in 8 bits for the weight gradient
        _norm("norm_pack_train_16384x4096", 16384, 4096, "bf16", "f32", pack=True),
        # a small model in fp32, odd sizes
        _norm_grad("norm_grad_odd_f32", 1500, 1003, "f32", "f32"),
        # the training batch's backward pass, with the gradient that comes along the residual
        _norm_grad("norm_grad_train_16384x4096", 16384, 4096, "bf16", "f32"),
        # eight sequences of their own lengths, one new token each, against the keys and values held so far
        _attn("attn_decode_8x4096_32_8", "attn", "cache", 8, 1, 4096, 32, 8, 128, "bf16"),
        # documents of different lengths packed into one batch of 8192 tokens
        _attn("attn_packed_8192_32_8", "attn", "packed", 5, 8192, 8192, 32, 8, 128, "bf16"),
        # packed fp32 documents, a head that is no power of two
        _attn("attn_grad_odd_f32", "attn_grad", "packed", 7, 901, 901, 12, 4, 80, "f32"),
        # the backward pass of 16 x 1024 tokens, gradients as the output projection leaves them
        _attn("attn_grad_train_16x1024_16_8", "attn_grad", "batch", 16, 1024, 1024, 16, 8, 128, "bf16"),
        # sampled tokens' log probabilities with their alternatives, odd sizes, some positions padded (id -1)
        _logprob("logprob_odd_f32", "logprob", 700, 5003, "f32", ids="padded", top=5, scale=1.25),
        # scoring 4096 tokens with a large vocabulary
        _logprob("logprob_score_4096x128000", "logprob", 4096, 128000, "bf16", top=20),
        # the loss's backward pass for a small batch in fp32, with a term on the entropy
        _logprob("logprob_grad_odd_f32", "logprob_grad", 700, 5003, "f32", ids="padded", scale=1.25),
        # the loss's backward pass of 8 x 1024 tokens
        _logprob("logprob_grad_train_8192x32000", "logprob_grad", 8192, 32000, "bf16", entropy=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """Half of the widths are multiples of 64, the others anything."""
    n = _log(rng, lo, hi)
    return max(64, 64 * round(n / 64)) if rng.random() < 0.5 else n


def draw(rng):
    """One more case: any operator, both storage types, one token to 32768."""
    while True:
        op = rng.choice(["norm", "norm_grad", "attn", "attn", "attn_grad", "attn_grad", "logprob", "logprob_grad"])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        if op in ("norm", "norm_grad"):
            case = _norm("", _log(rng, 1, 32768), _width(rng, 64, 8192), dtype, rng.choice([dtype, "f32"]), rng.random() < 0.8,
                         rng.random() < 0.5)
            if op == "norm_grad":
                case["op"] = op
                del case["pack"]
        elif op in ("attn", "attn_grad"):
            dim = rng.choice([64, 128, 128, 128, 256, 2 * rng.randint(20, 128)])
            kv = rng.choice([1, 2, 4, 8, rng.randint(1, 12)])
            form = rng.choice(["batch", "padded", "packed"] + (["cache"] if op == "attn" else []))
            batch = _log(rng, 1, 32)
            seq = _log(rng, 1, 4096)
            if form == "packed":
                seq = min(8192, seq * batch)
            if form == "cache":
                seq = rng.choice([1, 1, 1, rng.randint(2, 16)])
            keys = _log(rng, 64, 32768) if form == "cache" else seq
            case = _attn("", op, form, batch, seq, keys, kv * rng.randint(1, 6), kv, dim, dtype,
                         True if form == "cache" else rng.random() < 0.8, rng.choice(["tokens", "heads"]))
        else:
            case = _logprob("", op, _log(rng, 1, 16384), _width(rng, 100, 130000), dtype, rng.choice(["drawn", "padded"]),
                            rng.choice([0, 1, 5, rng.randint(1, 50)]) if op == "logprob" else 0, rng.random() < 0.7,
                            rng.choice([1.0, 1.0, 0.7]))
        del case["name"]
        most = [work(c) for c in listed() if c["op"] == op]
        w = work(case)
        pairs = case["batch"] * case["heads"] * case["seq"] * case["keys"] if "heads" in case else 0
        if all(w[k] <= max(m[k] for m in most) for k in w) and w["bytes"] >= 2048 and pairs <= 1 << 31:
            return case


def _randn(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda")


def _heads(gen, case, rows, heads, dtype):
    """[batch, rows, heads, dim] (a packed batch: [rows, heads, dim]), stored so or heads before tokens."""
    lead = () if case["form"] == "packed" else (case["batch"],)
    if case["layout"] == "heads":
        return _randn(gen, *lead, heads, rows, case["dim"]).to(dtype).transpose(-3, -2)
    return _randn(gen, *lead, rows, heads, case["dim"]).to(dtype)


def _pow2(e):
    """2 ** e in 32 bits, exactly."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _held(x):
    """The values, in 32 bits, that 8 bits hold of x [T, C]: 32 tokens of a column share the
    least power of two with max |x| <= 448 2^e."""
    T, C = x.shape
    nb = -(-T // GROUP)
    x = torch.nn.functional.pad(x.float(), (0, 0, 0, nb * GROUP - T)).view(nb, GROUP, C)
    m, k = torch.frexp(x.abs().amax(1, keepdim=True))
    e = (k - 9 + (m > 0.875).int()).clamp(-100, 119)
    q = (x * _pow2(-e)).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)
    return (q.float() * _pow2(e)).view(-1, C)[:T]


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1000003 * seed + 41)
    op, dt = case["op"], TYPES[case["dtype"]]
    st = {"case": case}
    if op in ("norm", "norm_grad"):
        T, C = case["tokens"], case["width"]
        x = _randn(gen, T, C) * torch.where(torch.rand(C, generator=gen, device="cuda") < 0.01, 30.0, 1.0)
        st["gain"] = (1.0 + 0.2 * _randn(gen, C)).to(TYPES[case["gain"]])
        st["x"] = x.to(dt)
        if op == "norm":
            st["residual"] = (2.0 * _randn(gen, T, C)).to(dt) if case["residual"] else None
        else:
            st["g_y"] = (0.01 * _randn(gen, T, C)).to(dt)
            st["g_h"] = (0.01 * _randn(gen, T, C)).to(dt) if case["residual"] else None
    elif op in ("attn", "attn_grad"):
        B, S, K = case["batch"], case["seq"], case["keys"]
        st["q"], st["k"] = 1.2 * _heads(gen, case, S, case["heads"], dt), _heads(gen, case, K, case["kv_heads"], dt)
        st["v"] = 0.7 * _heads(gen, case, K, case["kv_heads"], dt)
        where = {}
        if case["form"] == "packed":  # documents of all lengths, some of them empty, some tokens behind the last one
            cut = torch.randint(0, S + 1, (B,), generator=gen, device="cuda").sort().values
            where["q_starts"] = torch.cat([cut.new_zeros(1), cut[1:], cut.new_full((1,), S - S // 50)]).clamp_max(S - S // 50).int()
        if case["form"] == "padded":
            where["q_lengths"] = where["k_lengths"] = torch.randint(1, S + 1, (B,), generator=gen, device="cuda").int()
        if case["form"] == "cache":
            where["k_lengths"] = torch.randint(min(K, max(S, K // 2)), K + 1, (B,), generator=gen, device="cuda").int()
        st["where"] = where
        if op == "attn_grad":
            st["out"], st["lse"] = _attention(st)
            st["g"] = (0.01 * _heads(gen, dict(case, layout="tokens"), S, case["heads"], torch.float32)).to(dt)
    else:
        N, V = case["tokens"], case["vocab"]
        z = _randn(gen, N, V)
        # tokens: likely ones; the distributions run from flat to sharp
        z.mul_(1.0 + 2.5 * torch.rand(N, 1, generator=gen, device="cuda"))
        t = (z + 2.0 * _randn(gen, N, V)).argmax(1) if N * V < 1 << 26 else torch.randint(0, V, (N,), generator=gen, device="cuda")
        if case["ids"] == "padded":
            t[torch.rand(N, generator=gen, device="cuda") < 0.15] = -1
        st["logits"], st["tokens"] = z.to(dt), t
        if op == "logprob_grad":
            del z
            st["lse"], st["entropy"] = _lse_entropy(st["logits"].float() * case["scale"])
            on = (t >= 0).float()
            st["entropy"] = st["entropy"] * on
            st["g"] = -(0.5 + torch.rand(N, generator=gen, device="cuda")) / N
            st["g_entropy"] = 0.01 * _randn(gen, N) / N if case["entropy"] else None
    return st


def _visible(st):
    """[B, S, K] truth values: whether a query sees a key (a packed batch: B = 1)."""
    case, w = st["case"], st["where"]
    S, K = case["seq"], case["keys"]
    i, j = torch.arange(S, device="cuda"), torch.arange(K, device="cuda")
    if case["form"] == "packed":
        cuts = w["q_starts"].long()
        doc = torch.searchsorted(cuts, i, right=True)
        see = (doc[:, None] == doc[None, :]) & (i < cuts[-1])[:, None]
        if case["causal"]:
            see = see & (j[None, :] <= i[:, None])
        return see[None]
    every = torch.ones(case["batch"], dtype=torch.long, device="cuda")
    n_q, n_k = w.get("q_lengths", S * every).long()[:, None, None], w.get("k_lengths", K * every).long()[:, None, None]
    see = (i[None, :, None] < n_q) & (j[None, None, :] < n_k)
    if case["causal"]:
        see = see & (j[None, None, :] <= i[None, :, None] + n_k - n_q)
    return see


def _by_heads(t, heads):
    """[B, heads, rows, dim] in 32 bits; keys and values repeated for the heads that share them."""
    t = t.float() if t.dim() == 4 else t.float()[None]
    return t.transpose(1, 2).repeat_interleave(heads // t.shape[2], 1)


def _back(t, like):
    t = t.transpose(1, 2)
    return t if like.dim() == 4 else t[0]


def _attention(st):
    case, dt = st["case"], st["q"].dtype
    q, k, v = (_by_heads(st[n], case["heads"]) for n in ("q", "k", "v"))
    see = _visible(st)[:, None]
    s = torch.matmul(q, k.transpose(-1, -2)).mul_(case["dim"] ** -0.5).masked_fill_(~see, float("-inf"))
    m = s.amax(-1, keepdim=True).clamp_min(-1e30)
    p = s.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, v) / total.clamp_min(1e-37)
    return _back(out, st["q"]).to(dt).contiguous(), _back(m + total.log(), st["q"]).squeeze(-1).contiguous()


def _shared(t, kv_heads, like):
    """Gradients of keys or values: summed over the heads that share them."""
    B, H, S, D = t.shape
    return _back(t.view(B, kv_heads, H // kv_heads, S, D).sum(2), like).to(like.dtype)


def _attention_grad(st):
    case, c = st["case"], st["case"]["dim"] ** -0.5
    q, k, v, g, o = (_by_heads(st[n], case["heads"]) for n in ("q", "k", "v", "g", "out"))
    lse = _by_heads(st["lse"].unsqueeze(-1), case["heads"])
    see = _visible(st)[:, None]
    p = torch.matmul(q, k.transpose(-1, -2)).mul_(c).sub_(lse.clamp_min(-1e30)).masked_fill_(~see, float("-inf")).exp_()
    dv = torch.matmul(p.transpose(-1, -2), g)
    ds = torch.matmul(g, v.transpose(-1, -2)).sub_((g * o).sum(-1, keepdim=True)).mul_(p)
    del p
    dq, dk = c * torch.matmul(ds, k), c * torch.matmul(ds.transpose(-1, -2), q)
    return [_back(dq, st["q"]).to(st["q"].dtype), _shared(dk, case["kv_heads"], st["k"]), _shared(dv, case["kv_heads"], st["v"])]


def _lse_entropy(z):
    """log of the sum of exponentials, and the entropy of the distribution."""
    m = z.amax(-1, keepdim=True)
    e = (z - m).exp()
    total = e.sum(-1)
    mean = (e * (z - m)).sum(-1) / total
    return m[:, 0] + total.log(), total.log() - mean


def _top(x, k):
    """Indices of the k largest of each row, equal ones by index."""
    bits = x.float().view(torch.int32).long()
    order = torch.where(bits < 0, -(bits & 0x7fffffff), bits)
    index = torch.arange(x.shape[1], device=x.device)
    return ((order << 32) + ((1 << 31) - 1 - index)).topk(k, 1).indices


def _plain(st):
    case = st["case"]
    op, dt = case["op"], TYPES[case["dtype"]]
    if op == "norm":
        h = st["x"].float()
        if case["residual"]:
            h = h + st["residual"].float()
        y = (h * torch.rsqrt((h * h).mean(-1, keepdim=True) + EPS) * st["gain"].float()).to(dt)
        return [h.to(dt), y] + ([_held(y).to(dt)] if case["pack"] else [])
    if op == "norm_grad":
        h, g = st["x"].float(), st["g_y"].float()
        r = torch.rsqrt((h * h).mean(-1, keepdim=True) + EPS)
        n, gw = h * r, g * st["gain"].float()
        dx = r * (gw - n * (gw * n).mean(-1, keepdim=True))
        if case["residual"]:
            dx = dx + st["g_h"].float()
        return [dx.to(dt), (g * n).sum(0).to(st["gain"].dtype)]
    if op == "attn":
        return list(_attention(st))
    if op == "attn_grad":
        return _attention_grad(st)
    t = st["tokens"]
    on = (t >= 0) & (t < case["vocab"])
    at = t.clamp(0)[:, None]
    z = st["logits"].float() * case["scale"]
    if op == "logprob":
        lse, entropy = _lse_entropy(z)
        out = [(z.gather(1, at)[:, 0] - lse) * on, entropy * on, lse * on]
        if case["top"]:
            best = _top(st["logits"], case["top"])
            out += [(z.gather(1, best) - lse[:, None]) * on[:, None], torch.where(on[:, None], best, -1)]
        return out
    log_p = z.sub_(st["lse"][:, None])
    p = log_p.exp()
    gl = (st["g"] * on)[:, None]
    d = p * -gl
    if case["entropy"]:
        d -= (st["g_entropy"] * on)[:, None] * p * (log_p + st["entropy"][:, None])
    d.scatter_add_(1, at, gl)
    return (d * case["scale"]).to(dt)


def run(st):
    if not own:
        return _plain(st)
    import paper_2606_27216_amd as hm

    case = st["case"]
    op = case["op"]
    if op == "norm":
        got = hm.add_norm(st["x"], st["residual"], st["gain"], eps=EPS, pack=case["pack"])
        if not case["pack"]:
            return list(got)
        h, y, codes, exps = got
        return [h, y, hm.act_unpack(codes, exps, case["tokens"], dtype=y.dtype)]
    if op == "norm_grad":
        return list(hm.add_norm_grad(st["g_y"], st["x"], st["gain"], g_h=st["g_h"], eps=EPS))
    if op == "attn":
        return list(hm.attention(st["q"], st["k"], st["v"], causal=case["causal"], **st["where"]))
    if op == "attn_grad":
        return list(hm.attention_grad(st["g"], st["q"], st["k"], st["v"], st["out"], st["lse"], causal=case["causal"],
                                      **st["where"]))
    if op == "logprob":
        return list(hm.token_logprob(st["logits"], st["tokens"], top=case["top"], scale=case["scale"]))
    return hm.token_logprob_grad(st["g"], st["g_entropy"], st["logits"], st["tokens"], st["lse"], st["entropy"],
                                 scale=case["scale"])


def _pairs(case):
    """Visible pairs of a query and a key that the drawn lengths are expected to give, and the
    queries and keys in use."""
    B, S, K = case["batch"], case["seq"], case["keys"]
    if case["form"] == "packed":  # B pieces between uniform cuts: the mean of a piece's square
        n = S - S // 50
        pairs, q, k = 2 * n * n / (B + 1) if B > 1 else n * n, n, n
    elif case["form"] == "padded":
        pairs, q, k = B * S * S / 3, B * S / 2, B * S / 2
    elif case["form"] == "cache":
        pairs, q, k = B * S * K * 0.75, B * S, B * K * 0.75
    else:
        pairs, q, k = B * S * K, B * S, B * K
    if case["causal"] and case["form"] != "cache":
        pairs /= 2
    return pairs, q, k


def work(case):
    op, es = case["op"], SIZE[case["dtype"]]
    if op in ("norm", "norm_grad"):
        n = case["tokens"] * case["width"]
        if op == "norm_grad":
            return {"bytes": n * es * (4 if case["residual"] else 3) + 2 * case["width"] * SIZE[case["gain"]], "flops": 12 * n}
        held = -(-case["tokens"] // GROUP) * case["width"] * (GROUP + 1)
        extra = 2 * held + n * es if case["pack"] else 0  # the codes written, read again and restored
        return {"bytes": n * es * (4 if case["residual"] else 2) + extra, "flops": 6 * n}
    if op in ("attn", "attn_grad"):
        pairs, q, k = _pairs(case)
        H, G, D = case["heads"], case["kv_heads"], case["dim"]
        if op == "attn":
            return {"bytes": int((2 * q * H + 2 * k * G) * D * es + 4 * q * H), "flops": int(4 * D * H * pairs)}
        return {"bytes": int((4 * q * H + 4 * k * G) * D * es + 4 * q * H), "flops": int(10 * D * H * pairs)}
    n = int(case["tokens"] * (0.85 if case["ids"] == "padded" else 1.0)) * case["vocab"]
    if op == "logprob":
        return {"bytes": n * es + case["tokens"] * (20 + 12 * case["top"]), "flops": 5 * n}
    return {"bytes": (n + case["tokens"] * case["vocab"]) * es + 24 * case["tokens"], "flops": 6 * n}


def _exp2(n):
    """2 ** n in 64 bits, exactly, for whole numbers n."""
    return ((n.long() + 1023) << 52).view(torch.float64)


def _exact_held(x):
    """What 8 bits hold of x [T, C], from the definition in 64 bits."""
    out = torch.empty_like(x)
    for i in range(0, x.shape[0], GROUP):
        part = x[i:i + GROUP]
        top = part.abs().amax(0)
        e = torch.ceil(torch.log2(top.clamp_min(2.0 ** -200) / 448.0))
        e = torch.where(top > 448.0 * _exp2(e), e + 1, torch.where(top <= 448.0 * _exp2(e - 1), e - 1, e))
        unit = _exp2(e.clamp(-100, 119))
        v = (part / unit).clamp(-448.0, 448.0)
        step = _exp2(torch.frexp(v)[1].sub(4).clamp_min(-9))  # of three bits after the leading one
        out[i:i + GROUP] = torch.round(v / step) * step * unit
    return out


def _pieces(st):
    """(queries, keys) of each sequence as slices of the flattened tokens."""
    case, w = st["case"], st["where"]
    S, K = case["seq"], case["keys"]
    if case["form"] == "packed":
        cuts = w["q_starts"].tolist()
        return [(slice(a, b), slice(a, b)) for a, b in zip(cuts, cuts[1:])]
    n_q = w["q_lengths"].tolist() if "q_lengths" in w else [S] * case["batch"]
    n_k = w["k_lengths"].tolist() if "k_lengths" in w else [K] * case["batch"]
    return [(slice(b * S, b * S + n_q[b]), slice(b * K, b * K + n_k[b])) for b in range(case["batch"])]


def _exact_attention(st):
    """Sequence by sequence and head by head, the softmax and (by autograd) the gradients in 64 bits."""
    case, grad = st["case"], st["case"]["op"] == "attn_grad"
    H, G, D = case["heads"], case["kv_heads"], case["dim"]
    q, k, v = (st[n].reshape(-1, st[n].shape[-2], D) for n in ("q", "k", "v"))
    f64 = {"dtype": torch.float64, "device": "cuda"}
    out, lse = torch.zeros(q.shape, **f64), torch.full(q.shape[:2], float("-inf"), **f64)
    dq, dk, dv = (torch.zeros(t.shape, **f64) for t in (q, k, v))
    g = st["g"].reshape(q.shape) if grad else None
    for rows, keys in _pieces(st):
        n, m = rows.stop - rows.start, keys.stop - keys.start
        if n == 0 or m == 0:
            continue
        hide = torch.ones(n, m, dtype=torch.bool, device="cuda").triu(m - n + 1) if case["causal"] else None
        for h in range(H):
            a, b, c = (t.detach().double().requires_grad_(grad) for t in (q[rows, h], k[keys, h * G // H], v[keys, h * G // H]))
            s = torch.mm(a, b.t().contiguous()) / math.sqrt(D)
            if hide is not None:
                s = s.masked_fill(hide, float("-inf"))
            o = torch.mm(torch.softmax(s, 1), c)
            if grad:
                da, db, dc = torch.autograd.grad(o, (a, b, c), g[rows, h].double())
                dq[rows, h] = da
                dk[keys, h * G // H] += db
                dv[keys, h * G // H] += dc
            else:
                out[rows, h] = o
                lse[rows, h] = torch.logsumexp(s, 1)
    if grad:
        return [dq.view(st["q"].shape), dk.view(st["k"].shape), dv.view(st["v"].shape)]
    return [out.view(st["q"].shape), lse.view(st["q"].shape[:-1])]


def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    if op == "norm":
        h = st["x"].double() + (st["residual"].double() if case["residual"] else 0.0)
        y = h / torch.sqrt(h.square().sum(1, keepdim=True) / case["width"] + EPS) * st["gain"].double()
        return [h, y] + ([_exact_held(y.to(TYPES[case["dtype"]]).double())] if case["pack"] else [])
    if op == "norm_grad":
        h, w = st["x"].double().requires_grad_(), st["gain"].double().requires_grad_()
        y = h / torch.sqrt(h.square().sum(1, keepdim=True) / case["width"] + EPS) * w
        dh, dw = torch.autograd.grad(y, (h, w), st["g_y"].double())
        return [dh + (st["g_h"].double() if case["residual"] else 0.0), dw]
    if op in ("attn", "attn_grad"):
        return _exact_attention(st)
    N, V, t = case["tokens"], case["vocab"], st["tokens"]
    step = max(1, (1 << 27) // V)
    parts = []
    for i in range(0, N, step):
        z = st["logits"][i:i + step].double() * case["scale"]
        on = (t[i:i + step] >= 0).double()
        at = t[i:i + step].clamp(0)[:, None]
        if op == "logprob":
            lp = torch.log_softmax(z, 1)
            part = [lp.gather(1, at)[:, 0] * on, -(lp.exp() * lp).sum(1) * on, torch.logsumexp(z, 1) * on]
            if case["top"]:
                part.append(lp.topk(case["top"], 1).values * on[:, None])
            parts.append(part)
            continue
        z.requires_grad_()
        lp = torch.log_softmax(z, 1)
        loss = (lp.gather(1, at)[:, 0] * on * st["g"][i:i + step].double()).sum()
        if case["entropy"]:
            loss = loss - ((lp.exp() * lp).sum(1) * on * st["g_entropy"][i:i + step].double()).sum()
        (d,) = torch.autograd.grad(loss, z)
        parts.append([(d * case["scale"]).to(torch.float32 if N * V > 1 << 28 else torch.float64)])
    outs = [torch.cat(p) for p in zip(*parts)]
    if op == "logprob_grad":
        return outs[0]
    return outs + ([None] if case["top"] else [])
