"""The entry points of a decoder block's operators on a machine without a GPU: refusals before
anything is enqueued, workspaces, and the binding's view of the header."""
import os
import re
import shutil
import subprocess

import pytest

import paper_2606_27216_amd as hm
from paper_2606_27216_amd import block_ops as ops
from paper_2606_27216_amd import train_ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x10000  # a pointer that no call may follow
BIG = 1 << 40
NAN, INF = float("nan"), float("inf")


def _call(name, good, **bad):
    args = dict(good, **bad)
    assert list(args) == list(good)
    return getattr(hm.lib(), "himuon_" + name)(*args.values())


NORM = dict(n=4, width=8, x=P, ld_x=8, res=2 * P, ld_res=8, gain=P, gain_dtype=hm.F32, h=3 * P, ld_h=8, y=4 * P, ld_y=8, codes=None,
            exps=None, eps=1e-6, dtype=hm.BF16, stream=None)
NORM_GRAD = dict(n=4, width=8, g_y=P, ld_g_y=8, g_h=P, ld_g_h=8, h=P, ld_h=8, gain=P, gain_dtype=hm.F32, dh=P, ld_dh=8, dgain=P,
                 eps=1e-6, dtype=hm.BF16, ws=P, ws_bytes=BIG, stream=None)
LOGPROB = dict(n=4, vocab=100, logits=P, ld=100, dtype=hm.BF16, tokens=P, index=train_ops.I64, scale=1.0, top=5, logprob=P, entropy=P,
               lse=P, top_logprob=P, top_index=P, stream=None)
LOGPROB_GRAD = dict(n=4, vocab=100, g_logprob=P, g_entropy=P, logits=P, ld=100, dtype=hm.BF16, tokens=P, index=train_ops.I64, lse=P,
                    entropy=P, scale=1.0, d=P, ld_d=100, stream=None)


@pytest.mark.parametrize("name,good,bad", [
    *[("add_norm", NORM, b) for b in (dict(n=-1), dict(width=0), dict(x=None), dict(ld_x=7), dict(ld_res=7), dict(gain=None),
                                      dict(gain_dtype=2), dict(h=None), dict(ld_h=7), dict(y=None), dict(ld_y=7), dict(y=3 * P),
                                      dict(codes=P), dict(exps=P), dict(codes=P + 8, exps=P), dict(eps=-1.0), dict(eps=NAN),
                                      dict(eps=INF), dict(dtype=2), dict(ld_x=1 << 61))],
    *[("add_norm_grad", NORM_GRAD, b) for b in (dict(n=-1), dict(width=0), dict(g_y=None), dict(ld_g_y=7), dict(ld_g_h=7), dict(h=None),
                                                dict(ld_h=7), dict(gain=None), dict(gain_dtype=-1), dict(dh=None), dict(ld_dh=7),
                                                dict(dgain=None), dict(eps=-1.0), dict(eps=NAN), dict(dtype=5))],
    *[("token_logprob", LOGPROB, b) for b in (dict(n=-1), dict(vocab=0, top=0), dict(logits=None), dict(ld=99), dict(dtype=2),
                                              dict(tokens=None), dict(index=2), dict(scale=0.0), dict(scale=-1.0), dict(scale=NAN),
                                              dict(scale=INF), dict(top=-1), dict(top=65), dict(vocab=4, ld=4), dict(logprob=None),
                                              dict(entropy=None), dict(lse=None), dict(top_logprob=None), dict(top_index=None),
                                              dict(ld=1 << 61))],
    *[("token_logprob_grad", LOGPROB_GRAD, b) for b in (dict(n=-1), dict(vocab=0), dict(logits=None), dict(ld=99), dict(dtype=-1),
                                                        dict(tokens=None), dict(index=-1), dict(lse=None), dict(entropy=None),
                                                        dict(scale=0.0), dict(d=None), dict(ld_d=99))],
])
def test_invalid_arguments(name, good, bad):
    assert _call(name, good, **bad) == hm.ERR_INVALID_ARG


@pytest.mark.parametrize("name,good,bad", [
    ("add_norm", NORM, dict(n=1 << 31)), ("add_norm", NORM, dict(width=1 << 27, ld_x=1 << 27, ld_res=1 << 27, ld_h=1 << 27, ld_y=1 << 27)),
    ("add_norm", NORM, dict(n=1 << 30, codes=P, exps=P)),
    ("add_norm_grad", NORM_GRAD, dict(n=1 << 31)),
    ("token_logprob", LOGPROB, dict(n=1 << 31)), ("token_logprob", LOGPROB, dict(vocab=(1 << 31) - 1, ld=1 << 31)),
    ("token_logprob", LOGPROB, dict(n=1 << 30)), ("token_logprob", LOGPROB, dict(n=1 << 25, vocab=5000, ld=5000)),
    ("token_logprob_grad", LOGPROB_GRAD, dict(n=1 << 25)), ("token_logprob_grad", LOGPROB_GRAD, dict(n=1 << 20, vocab=1 << 20, ld=1 << 20, ld_d=1 << 20)),
])
def test_sizes_beyond_the_kernels(name, good, bad):
    assert _call(name, good, **bad) == hm.ERR_UNSUPPORTED


def test_empty_calls_enqueue_nothing():
    assert _call("add_norm", NORM, n=0, x=None, res=None, h=None, y=None) == hm.OK
    assert _call("token_logprob", LOGPROB, n=0, logits=None, tokens=None, logprob=None, entropy=None, lse=None) == hm.OK
    assert _call("token_logprob_grad", LOGPROB_GRAD, n=0, logits=None, tokens=None, d=None) == hm.OK


def _attn(**bad):
    f = dict(batch=2, q_len=10, k_len=12, hq=4, hk=2, dim=64, causal=1, dtype=hm.BF16, index=train_ops.I32, qs=0, ks=0, ql=0, kl=0,
             scale=0.125)
    assert set(bad) <= set(f)
    f.update(bad)
    return ops._ATTN.pack(*f.values())


HEADS = train_ops._HEADS.pack(P, 64 * 4 * 12, 64 * 4, 64)
OUT = train_ops._HEADS.pack(2 * P, 64 * 4 * 12, 64 * 4, 64)
NONE = train_ops._HEADS.pack(0, 64 * 4 * 12, 64 * 4, 64)


def _forward(args, heads=(HEADS,) * 3 + (OUT,), lse=P, ws=None, ws_bytes=0):
    return hm.lib().himuon_attention(args, *heads, lse, ws, ws_bytes, None)


def _backward(args, heads=(HEADS,) * 5 + (OUT,) * 3, lse=P, ws=P, ws_bytes=BIG):
    return hm.lib().himuon_attention_grad(args, *heads[:5], lse, *heads[5:], ws, ws_bytes, None)


@pytest.mark.parametrize("bad", [dict(batch=-1), dict(q_len=-1), dict(k_len=-1), dict(hq=0), dict(hk=0), dict(hq=3), dict(dim=0),
                                 dict(dtype=2), dict(index=2), dict(qs=P), dict(ks=P), dict(scale=0.0), dict(scale=-1.0), dict(scale=NAN),
                                 dict(scale=INF)])
def test_attention_invalid_arguments(bad):
    assert _forward(_attn(**bad)) == hm.ERR_INVALID_ARG
    assert _backward(_attn(**bad)) == hm.ERR_INVALID_ARG
    assert hm.lib().himuon_attention_workspace_size(_attn(**bad)) == 0
    assert hm.lib().himuon_attention_grad_workspace_size(_attn(**bad)) == 0


@pytest.mark.parametrize("bad", [dict(dim=257), dict(batch=1 << 31), dict(q_len=1 << 30), dict(k_len=1 << 31), dict(batch=1 << 24, q_len=1 << 10),
                                 dict(qs=P, ks=P, q_len=1 << 30)])
def test_attention_sizes_beyond_the_kernels(bad):
    assert _forward(_attn(**bad)) == hm.ERR_UNSUPPORTED
    assert _backward(_attn(**bad)) == hm.ERR_UNSUPPORTED


def test_attention_pointers_strides_and_workspaces():
    for good, call in (([HEADS] * 3 + [OUT], _forward), ([HEADS] * 5 + [OUT] * 3, _backward)):
        assert call(None) == hm.ERR_INVALID_ARG
        for i in range(len(good)):
            for bad in (NONE, None, train_ops._HEADS.pack(5 * P, 1 << 50, 64 * 4, 64)):
                assert call(_attn(), [bad if i == j else h for j, h in enumerate(good)]) == hm.ERR_INVALID_ARG
            if good[i] is OUT:  # a result in an input's place
                assert call(_attn(), [HEADS if i == j else h for j, h in enumerate(good)]) == hm.ERR_INVALID_ARG
        assert call(_attn(), lse=None) == hm.ERR_INVALID_ARG
    for flat in (train_ops._HEADS.pack(5 * P, 0, 256, 64), train_ops._HEADS.pack(5 * P, 4096, 0, 64), train_ops._HEADS.pack(5 * P, 4096, 256, 0)):
        assert _forward(_attn(), [HEADS] * 3 + [flat]) == hm.ERR_INVALID_ARG  # rows of a result must not fall on each other
        for i in range(5, 8):
            assert _backward(_attn(), [flat if i == j else HEADS if j < 5 else OUT for j in range(8)]) == hm.ERR_INVALID_ARG
    L = hm.lib()
    assert L.himuon_attention_grad_workspace_size(_attn()) >= 2 * 10 * 4 * 8
    for bad in (dict(ws=None), dict(ws=P + 8), dict(ws_bytes=2 * 10 * 4 * 8 - 1)):
        assert _backward(_attn(), **bad) == hm.ERR_WORKSPACE
    # one query against many keys: the keys are shared out over blocks, whose results meet in a workspace
    one = _attn(q_len=1, k_len=4096)
    need = L.himuon_attention_workspace_size(one)
    assert need > 0 and L.himuon_attention_workspace_size(_attn(q_len=100, k_len=4096)) == 0
    assert L.himuon_attention_workspace_size(_attn(batch=1 << 12, q_len=1, k_len=4096)) == 0  # (blocks enough)
    for bad in (dict(ws=None, ws_bytes=need), dict(ws=P + 8, ws_bytes=need), dict(ws=P, ws_bytes=need - 1)):
        assert _forward(one, **bad) == hm.ERR_WORKSPACE


def test_attention_empty_calls():
    assert _forward(_attn(batch=0), [NONE] * 4, lse=None) == hm.OK
    assert _forward(_attn(q_len=0), [NONE] * 4, lse=None) == hm.OK
    assert _backward(_attn(batch=0), [NONE] * 8, lse=None, ws=None, ws_bytes=0) == hm.OK
    assert _backward(_attn(q_len=0, k_len=0), [NONE] * 8, lse=None, ws=None, ws_bytes=0) == hm.OK


def test_norm_workspace():
    size = hm.lib().himuon_add_norm_grad_workspace_size
    assert size(100, 64) > 0 and size(0, 64) > 0 and size(-1, 64) == 0 and size(4, 0) == 0 and size(1 << 31, 8) == 0
    assert size(1 << 20, 4096) <= 4096 * 4 * 2048
    for bad in (dict(ws=None), dict(ws=P + 8), dict(ws_bytes=31)):
        assert _call("add_norm_grad", NORM_GRAD, **bad) == hm.ERR_WORKSPACE


def test_tensors_of_the_wrong_kind():
    torch = pytest.importorskip("torch")
    x, w, t, q = torch.zeros(4, 8), torch.ones(8), torch.zeros(4, dtype=torch.int64), torch.zeros(2, 4, 2, 8)
    lse = torch.zeros(2, 4, 2)
    for f in (lambda: hm.add_norm(x, x, w), lambda: hm.add_norm_grad(x, x, w), lambda: hm.token_logprob(x, t),
              lambda: hm.token_logprob_grad(None, None, x, t, torch.zeros(4), torch.zeros(4)), lambda: hm.attention(q, q, q),
              lambda: hm.attention_grad(q, q, q, q, q, lse)):
        with pytest.raises(ValueError):
            f()


def test_the_bindings_constants_and_layouts_are_the_headers(tmp_path):
    src = open(os.path.join(ROOT, "include", "himuon.h")).read()
    assert int(re.search(r"#define HIMUON_MAX_ATTN_DIM (\d+)", src)[1]) == ops.MAX_ATTN_DIM
    assert int(re.search(r"#define HIMUON_MAX_TOP (\d+)", src)[1]) == ops.MAX_TOP
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    prog = tmp_path / "layout.c"
    prog.write_text('#include "himuon.h"\n#include <stdio.h>\n#include <string.h>\nint main(void) { himuon_attn_t a; memset(&a, 0, sizeof a);\n'
                    'a.batch = 1; a.q_len = 2; a.k_len = 3; a.q_heads = 4; a.k_heads = 5; a.head_dim = 6; a.causal = 1; a.dtype = 7; a.index = 8;\n'
                    'a.q_starts = (void*)9; a.k_starts = (void*)10; a.q_lengths = (void*)11; a.k_lengths = (void*)12; a.scale = 0.5f;\n'
                    'fwrite(&a, sizeof a, 1, stdout); return 0; }\n')
    exe = tmp_path / "layout"
    subprocess.run([cc, "-I", os.path.join(ROOT, "include"), str(prog), "-o", str(exe)], check=True)
    got = subprocess.run([str(exe)], check=True, capture_output=True).stdout
    assert got == ops._ATTN.pack(1, 2, 3, 4, 5, 6, 1, 7, 8, 9, 10, 11, 12, 0.5)
