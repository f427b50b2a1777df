"""The operators of a training step around the optimizer, as they are measured: what
each of them computes, the calls that users make, their inputs and their work.

A case is a dict of plain values. "op" is the operator:

    embed        rows of a token table, scaled
    embed_grad   the table's gradient
    qk           per-head norms of queries and keys and the position rotation
    qk_grad      their backward pass
    pack         an activation held in 8 bits for the backward pass, and restored
    wgrad        a weight matrix's gradient from an activation held in 8 bits

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


def _embed(name, tokens, vocab, dim, dtype, ids="zipf", scale=1.0):
    return {"name": name, "op": "embed", "tokens": tokens, "vocab": vocab, "dim": dim, "dtype": dtype, "ids": ids,
            "scale": scale}


def _embed_grad(name, tokens, vocab, dim, dtype, out, ids="zipf", scale=1.0):
    return dict(_embed(name, tokens, vocab, dim, dtype, ids, scale), op="embed_grad", out=out)


def _qk(name, op, batch, seq, heads, kv_heads, dim, rot, dtype, gains, pairs="halves", start="documents", layout="tokens"):
    return {"name": name, "op": op, "batch": batch, "seq": seq, "heads": heads, "kv_heads": kv_heads, "dim": dim,
            "rot": rot, "dtype": dtype, "gains": gains, "pairs": pairs, "start": start, "layout": layout}


def _pack(name, tokens, cols, dtype, data="gauss"):
    return {"name": name, "op": "pack", "tokens": tokens, "cols": cols, "dtype": dtype, "data": data}


def _wgrad(name, tokens, rows, cols, dtype, out, data="gauss"):
    return {"name": name, "op": "wgrad", "tokens": tokens, "rows": rows, "cols": cols, "dtype": dtype, "out": out,
            "data": data}


def listed():
    return [
        # generation while a run is evaluated: one token of each of 32 sequences
        _embed("embed_decode_32x4096", 32, 32000, 4096, "bf16"),
        # a training batch of 16 x 1024 tokens, table scaled by sqrt(width)
        _embed("embed_train_16384x2560", 16384, 128000, 2560, "bf16", scale=math.sqrt(2560.0)),
        # a small model's table in fp32, odd sizes, some positions padded (id -1)
        _embed_grad("embed_grad_odd_f32", 1500, 5003, 1003, "f32", "f32", ids="padded"),
        # the same training batch's gradient: a few tokens make up much of the batch
        _embed_grad("embed_grad_train_16384x4096", 16384, 32000, 4096, "bf16", "bf16", scale=64.0),
        # eight sequences, one token each, at positions of their own
        _qk("qk_decode_8", "qk", 8, 1, 32, 8, 128, 128, "bf16", "bf16", start="each"),
        # a 7B-style layer's queries and keys, 8 x 1024 tokens
        _qk("qk_train_8x1024_32_32", "qk", 8, 1024, 32, 32, 128, 128, "bf16", "f32"),
        # partial rotation of neighbouring elements, a head that is no power of two, fp32
        _qk("qk_grad_odd_f32", "qk_grad", 3, 259, 12, 4, 80, 40, "f32", "f32", pairs="neighbours"),
        # grouped heads, 16 x 1024 tokens, gradients as attention leaves them (heads before tokens)
        _qk("qk_grad_train_16x1024_16_8", "qk_grad", 16, 1024, 16, 8, 128, 128, "bf16", "bf16", layout="heads"),
        # a hidden state of a small model in fp32, odd sizes
        _pack("pack_odd_f32", 777, 1000, "f32", data="outliers"),
        # the widest activation of a 7B-style layer: the input of its down projection
        _pack("pack_train_8192x11008", 8192, 11008, "bf16", data="heavy"),
        # fp32 gradients, sizes that are no multiples of anything
        _wgrad("wgrad_odd_f32", 1111, 1003, 777, "f32", "f32", data="outliers"),
        # the gradient of a 7B-style layer's up projection, 8 x 1024 tokens
        _wgrad("wgrad_train_8192x11008x4096", 8192, 11008, 4096, "bf16", "bf16"),
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
        op = rng.choice(["embed", "embed_grad", "qk", "qk_grad", "pack", "wgrad", "wgrad"])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        if op in ("embed", "embed_grad"):
            case = {"op": op, "tokens": _log(rng, 1 if op == "embed" else 16, 32768), "vocab": _log(rng, 300, 130000),
                    "dim": _width(rng, 64, 5120), "dtype": dtype, "ids": rng.choice(["zipf", "zipf", "uniform", "padded", "one"]),
                    "scale": rng.choice([1.0, 1.0, 45.25])}
            if op == "embed_grad":
                case["out"] = rng.choice([dtype, "f32"])
        elif op in ("qk", "qk_grad"):
            dim = rng.choice([64, 128, 128, 128, 256, 2 * rng.randint(20, 128)])
            kv = rng.choice([1, 2, 4, 8, rng.randint(1, 12)])
            case = _qk("", op, _log(rng, 1, 32), _log(rng, 1, 4096), kv * rng.randint(1, 6), kv, dim,
                       dim if rng.random() < 0.7 else 2 * rng.randint(1, dim // 2), dtype, rng.choice([dtype, "f32"]),
                       rng.choice(["halves", "halves", "neighbours"]), rng.choice(["documents", "each"]),
                       rng.choice(["tokens", "heads"]))
            del case["name"]
        else:
            case = {"op": op, "tokens": _log(rng, 8, 32768), "cols": _width(rng, 64, 11008), "dtype": dtype,
                    "data": rng.choice(["gauss", "heavy", "outliers"])}
            if op == "wgrad":
                case.update(rows=_width(rng, 64, 11008), out=rng.choice([dtype, "f32"]))
        most = [work(c) for c in listed() if c["op"] == op]
        w = work(case)
        if all(w[k] <= max(m[k] for m in most) for k in w) and w["bytes"] >= 4096:
            return case


def _probabilities(case, device="cpu"):
    """Probability of each token: frequencies fall as 1 / rank."""
    V = case["vocab"]
    p = torch.ones(V, dtype=torch.float64, device=device)
    if case["ids"] in ("zipf", "padded"):
        p /= torch.arange(V, dtype=torch.float64, device=device) + 2.7
    return p / p.sum()


def _tokens(case, gen):
    N, V = case["tokens"], case["vocab"]
    if case["ids"] == "one":  # a batch of nothing but one token
        return torch.randint(0, V, (1,), generator=gen, device="cuda").repeat(N)
    t = torch.multinomial(_probabilities(case, "cuda"), N, replacement=True, generator=gen)
    if case["ids"] == "padded":
        t[torch.rand(N, generator=gen, device="cuda") < 0.15] = -1
    return t


def _activation(T, C, data, dtype, gen):
    x = torch.randn(T, C, generator=gen, device="cuda")
    if data == "heavy":  # products of a gate and a value: many near zero, some large
        x *= torch.nn.functional.silu(torch.randn(T, C, generator=gen, device="cuda"))
    if data == "outliers":  # a few columns far above the others
        x *= torch.where(torch.rand(C, generator=gen, device="cuda") < 0.01, 60.0, 1.0)
    return x.to(TYPES[dtype])


def _positions(case, gen):
    B, S = case["batch"], case["seq"]
    s = torch.arange(S, device="cuda").expand(B, S)
    if case["start"] == "each":  # sequences that are some way along
        return s + torch.randint(0, 4096, (B, 1), generator=gen, device="cuda")
    cut = torch.randint(0, S, (B, 1), generator=gen, device="cuda")  # two documents to a row
    return torch.where(s < cut, s, s - cut)


def _qkv(case, gen):
    """Queries and keys as slices of one projection's output."""
    B, S, H, K, D = (case[k] for k in ("batch", "seq", "heads", "kv_heads", "dim"))
    x = torch.randn(B, S, H + 2 * K, D, generator=gen, device="cuda")
    x *= 0.3 + 2.0 * torch.rand(H + 2 * K, 1, generator=gen, device="cuda")
    x = x.to(TYPES[case["dtype"]])
    return x[:, :, :H], x[:, :, H:H + K]


def _upstream(case, heads, gen):
    B, S, D = case["batch"], case["seq"], case["dim"]
    if case["layout"] == "heads":
        return (0.01 * torch.randn(B, heads, S, D, generator=gen, device="cuda")).to(TYPES[case["dtype"]]).transpose(1, 2)
    return (0.01 * torch.randn(B, S, heads, D, generator=gen, device="cuda")).to(TYPES[case["dtype"]])


def _pow2(e):
    """2 ** e in 32 bits, exactly."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _quantise(x):
    """8-bit floats (e4m3) of x [T, C], 32 tokens of a column to a shared power of two: the
    codes [T / 32, C, 32] and the exponents' bytes [T / 32, C], T rounded up."""
    T, C = x.shape
    nb = -(-T // GROUP)
    x = torch.nn.functional.pad(x.float(), (0, 0, 0, nb * GROUP - T)).view(nb, GROUP, C).transpose(1, 2)
    m, k = torch.frexp(x.abs().amax(2))
    e = (k - 9 + (m > 0.875).int()).clamp(-100, 119)  # the least e with max |x| <= 448 2^e
    q = (x * _pow2(-e)[:, :, None]).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)
    return q.view(torch.uint8).contiguous(), (e + 127).to(torch.uint8)


def _restore(q, exps, T):
    """The values [T, C], in 32 bits, that 8-bit codes and exponents stand for."""
    x = q.view(torch.float8_e4m3fn).float() * _pow2(exps.int() - 127)[:, :, None]
    return x.transpose(1, 2).reshape(-1, q.shape[1])[:T]


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1000003 * seed + 29)
    op, dt = case["op"], TYPES[case["dtype"]]
    st = {"case": case}
    if op in ("embed", "embed_grad"):
        st["tokens"] = _tokens(case, gen)
        if op == "embed":
            st["table"] = (0.02 * torch.randn(case["vocab"], case["dim"], generator=gen, device="cuda")).to(dt)
        else:
            st["grad"] = (0.01 * torch.randn(case["tokens"], case["dim"], generator=gen, device="cuda")).to(dt)
    elif op in ("qk", "qk_grad"):
        st["q"], st["k"] = _qkv(case, gen)
        st["wq"], st["wk"] = ((1.0 + 0.2 * torch.randn(case["dim"], generator=gen, device="cuda")).to(TYPES[case["gains"]])
                              for _ in range(2))
        st["pos"] = _positions(case, gen)
        half = case["rot"] // 2
        rate = 1e6 ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)
        angle = torch.arange(8192, dtype=torch.float64, device="cuda")[:, None] * rate
        st["cos"], st["sin"] = angle.cos().float(), angle.sin().float()
        if op == "qk_grad":
            st["gq"], st["gk"] = (_upstream(case, case[h], gen) for h in ("heads", "kv_heads"))
    else:
        x = _activation(case["tokens"], case["cols"], case["data"], case["dtype"], gen)
        if op == "pack":
            st["x"] = x
        else:
            st["q8"], st["exps"] = _quantise(x)
            st["grad"] = (1e-3 * torch.randn(case["tokens"], case["rows"], generator=gen, device="cuda")).to(dt)
    return st


def _rotate(x, cos, sin, neighbours):
    """The first 2 cos.shape[-1] elements of each head turned by the angles of its position."""
    R = 2 * cos.shape[-1]
    c, s = cos[:, :, None], sin[:, :, None]
    a, b = (x[..., 0:R:2], x[..., 1:R:2]) if neighbours else (x[..., :R // 2], x[..., R // 2:R])
    u, v = a * c - b * s, b * c + a * s
    y = torch.stack([u, v], -1).flatten(-2) if neighbours else torch.cat([u, v], -1)
    return torch.cat([y, x[..., R:]], -1)


def _norm_rope(x, w, cos, sin, neighbours):
    x = x.float()
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    return _rotate(x * r * w.float(), cos, sin, neighbours)


def _norm_rope_grad(g, x, w, cos, sin, neighbours):
    x = x.float()
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    n = x * r
    dz = _rotate(g.float(), cos, -sin, neighbours)
    dn = dz * w.float()
    return r * (dn - n * (dn * n).mean(-1, keepdim=True)), (dz * n).sum((0, 1, 2))


def _plain(st):
    case = st["case"]
    op, dt = case["op"], TYPES[case["dtype"]]
    if op in ("embed", "embed_grad"):
        t = st["tokens"]
        ok = (t >= 0) & (t < case["vocab"])
        if op == "embed":
            return ((st["table"][t.clamp(0)].float() * case["scale"]) * ok[:, None]).to(dt)
        out = torch.zeros(case["vocab"], case["dim"], device=t.device)
        out.index_add_(0, t.clamp(0), st["grad"].float() * ok[:, None])
        return (out * case["scale"]).to(TYPES[case["out"]])
    if op in ("qk", "qk_grad"):
        cos, sin, nb = st["cos"][st["pos"]], st["sin"][st["pos"]], case["pairs"] == "neighbours"
        if op == "qk":
            return [_norm_rope(st[x], st["w" + x], cos, sin, nb).to(dt) for x in "qk"]
        (dq, dwq), (dk, dwk) = (_norm_rope_grad(st["g" + x], st[x], st["w" + x], cos, sin, nb) for x in "qk")
        gains = TYPES[case["gains"]]
        return [dq.to(dt), dk.to(dt), dwq.to(gains), dwk.to(gains)]
    if op == "pack":
        return _restore(*_quantise(st["x"]), case["tokens"]).to(dt)
    x = _restore(st["q8"], st["exps"], case["tokens"])
    return (st["grad"].float().t() @ x).to(TYPES[case["out"]])


def run(st):
    if not own:
        return _plain(st)
    import paper_2606_27216_amd as hm

    case = st["case"]
    op = case["op"]
    if op == "embed":
        return hm.embed(st["tokens"], st["table"], scale=case["scale"])
    if op == "embed_grad":
        return hm.embed_grad(st["tokens"], st["grad"], case["vocab"], scale=case["scale"], dtype=TYPES[case["out"]])
    if op in ("qk", "qk_grad"):
        args = (st["q"], st["k"], st["wq"], st["wk"], st["cos"], st["sin"])
        kw = {"positions": st["pos"], "eps": EPS, "interleaved": case["pairs"] == "neighbours"}
        if op == "qk":
            return hm.qk_norm_rope(*args, **kw)
        return hm.qk_norm_rope_grad(st["gq"], st["gk"], *args, **kw)
    if op == "pack":
        q8, exps = hm.act_pack(st["x"])
        return hm.act_unpack(q8, exps, case["tokens"], dtype=TYPES[case["dtype"]])
    return hm.weight_grad(st["grad"], st["q8"], st["exps"], dtype=TYPES[case["out"]])


def work(case):
    op, es = case["op"], SIZE[case["dtype"]]
    if op in ("embed", "embed_grad"):
        N, D = case["tokens"], case["dim"]
        if op == "embed_grad":
            return {"bytes": 8 * N + N * D * es + case["vocab"] * D * SIZE[case["out"]], "flops": 2 * N * D}
        # distinct rows that the drawn tokens are expected to name
        rows = 1.0 if case["ids"] == "one" else float((1.0 - (1.0 - _probabilities(case)) ** N).sum())
        return {"bytes": 8 * N + int(rows * D * es) + N * D * es, "flops": N * D}
    if op in ("qk", "qk_grad"):
        T = case["batch"] * case["seq"]
        n = T * (case["heads"] + case["kv_heads"]) * case["dim"]
        table = min(T, 8192) * case["rot"] * 4
        return {"bytes": n * es * (2 if op == "qk" else 3) + table + 8 * T, "flops": n * (10 if op == "qk" else 20)}
    T, C = case["tokens"], case["cols"]
    held = -(-T // GROUP) * C * (GROUP + 1)
    if op == "pack":
        return {"bytes": 2 * T * C * es + 2 * held, "flops": 6 * T * C}
    O = case["rows"]
    return {"bytes": T * O * es + held + O * C * SIZE[case["out"]], "flops": 2 * T * O * C}


def _exact_norm_rope(x, w, angle_cos, angle_sin, neighbours):
    """The rotation as a product of complex numbers, the norm from its definition."""
    z = x / (x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + EPS).sqrt() * w
    h = angle_cos.shape[-1]
    turn = torch.complex(angle_cos, angle_sin).unsqueeze(2)
    if neighbours:
        t = torch.view_as_real(torch.view_as_complex(z[..., :2 * h].reshape(*z.shape[:-1], h, 2).contiguous()) * turn)
        t = t.reshape(*z.shape[:-1], 2 * h)
    else:
        t = torch.complex(z[..., :h], z[..., h:2 * h]) * turn
        t = torch.cat([t.real, t.imag], -1)
    return torch.cat([t, z[..., 2 * h:]], -1)


def _exp2(n):
    """2 ** n in 64 bits, exactly, for whole numbers n."""
    return ((n.long() + 1023) << 52).view(torch.float64)


def _exact_values(x):
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


def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    if op in ("embed", "embed_grad"):
        t = st["tokens"]
        ok = (t >= 0) & (t < case["vocab"])
        if op == "embed":
            out = torch.zeros(case["tokens"], case["dim"], dtype=torch.float64, device=t.device)
            out[ok] = st["table"][t[ok]].double() * case["scale"]
            return out
        out = torch.zeros(case["vocab"], case["dim"], dtype=torch.float64, device=t.device)
        return out.index_put_((t[ok],), st["grad"][ok].double() * case["scale"], accumulate=True)
    if op in ("qk", "qk_grad"):
        nb = case["pairs"] == "neighbours"
        c, s = st["cos"].double()[st["pos"]], st["sin"].double()[st["pos"]]
        outs, gains = [], []
        for x in "qk":
            v, w = st[x].double(), st["w" + x].double()
            if op == "qk":
                outs.append(_exact_norm_rope(v, w, c, s, nb))
                continue
            v, w = v.clone().requires_grad_(), w.requires_grad_()
            dv, dw = torch.autograd.grad(_exact_norm_rope(v, w, c, s, nb), (v, w), st["g" + x].double())
            outs.append(dv)
            gains.append(dw)
        return outs + gains
    if op == "pack":
        return _exact_values(st["x"].double())
    x = st["q8"].view(torch.float8_e4m3fn).double() * _exp2(st["exps"].long() - 127)[:, :, None]
    x = x.permute(0, 2, 1).reshape(-1, case["cols"])[:case["tokens"]]
    return torch.mm(st["grad"].double().t(), x)
