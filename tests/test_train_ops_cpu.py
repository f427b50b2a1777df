"""The entry points of the training-step operators on a machine without a GPU: sizes,
refusals before anything is enqueued, and the binding's view of the header."""
import os
import re
import shutil
import struct
import subprocess

import pytest

import paper_2606_27216_amd as hm
from paper_2606_27216_amd import train_ops as ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x10000  # a pointer that no call may follow
BIG = 1 << 40


def _call(name, good, **bad):
    args = dict(good, **bad)
    return getattr(hm.lib(), "himuon_" + name)(*args.values())


EMBED = dict(n=4, tokens=P, index=ops.I64, rows=10, dim=8, table=P, ld_table=8, out=2 * P, ld_out=8, scale=1.0, dtype=hm.F32,
             stream=None)
GRAD = dict(n=4, tokens=P, index=ops.I64, rows=10, dim=8, grad=P, ld_grad=8, dtype=hm.F32, out=2 * P, ld_out=8, out_dtype=hm.F32,
            scale=1.0, accumulate=0, ws=P, ws_bytes=BIG, stream=None)
PACK = dict(n=64, cols=8, x=P, ld=8, dtype=hm.BF16, codes=P, exps=P, stream=None)
UNPACK = dict(n=64, cols=8, codes=P, exps=P, x=P, ld=8, dtype=hm.BF16, stream=None)
WGRAD = dict(n=64, out=16, cols=8, grad=P, ld_grad=16, dtype=hm.BF16, codes=P, exps=P, dw=P, ld_dw=8, out_dtype=hm.F32,
             accumulate=0, ws=P, ws_bytes=BIG, stream=None)


@pytest.mark.parametrize("name,good,bad", [
    ("embed", EMBED, dict(n=-1)), ("embed", EMBED, dict(rows=0)), ("embed", EMBED, dict(dim=0)), ("embed", EMBED, dict(ld_table=7)),
    ("embed", EMBED, dict(ld_out=7)), ("embed", EMBED, dict(tokens=None)), ("embed", EMBED, dict(table=None)),
    ("embed", EMBED, dict(out=None)), ("embed", EMBED, dict(out=P)), ("embed", EMBED, dict(dtype=2)), ("embed", EMBED, dict(index=2)),
    ("embed", EMBED, dict(ld_table=1 << 61)),
    ("embed_grad", GRAD, dict(n=-1)), ("embed_grad", GRAD, dict(rows=0)), ("embed_grad", GRAD, dict(dim=0)),
    ("embed_grad", GRAD, dict(ld_grad=7)), ("embed_grad", GRAD, dict(ld_out=7)), ("embed_grad", GRAD, dict(tokens=None)),
    ("embed_grad", GRAD, dict(grad=None)), ("embed_grad", GRAD, dict(out=None)), ("embed_grad", GRAD, dict(out=P)),
    ("embed_grad", GRAD, dict(dtype=-1)), ("embed_grad", GRAD, dict(out_dtype=5)), ("embed_grad", GRAD, dict(index=-1)),
    ("act_pack", PACK, dict(n=-1)), ("act_pack", PACK, dict(cols=0)), ("act_pack", PACK, dict(x=None)), ("act_pack", PACK, dict(ld=7)),
    ("act_pack", PACK, dict(dtype=3)), ("act_pack", PACK, dict(codes=None)), ("act_pack", PACK, dict(codes=P + 8)),
    ("act_pack", PACK, dict(exps=None)),
    ("act_unpack", UNPACK, dict(n=-1)), ("act_unpack", UNPACK, dict(codes=P + 4)), ("act_unpack", UNPACK, dict(ld=7)),
    ("act_unpack", UNPACK, dict(x=None)), ("act_unpack", UNPACK, dict(exps=None)), ("act_unpack", UNPACK, dict(dtype=9)),
    ("weight_grad", WGRAD, dict(n=-1)), ("weight_grad", WGRAD, dict(out=0)), ("weight_grad", WGRAD, dict(cols=0)),
    ("weight_grad", WGRAD, dict(grad=None)), ("weight_grad", WGRAD, dict(ld_grad=15)), ("weight_grad", WGRAD, dict(ld_dw=7)),
    ("weight_grad", WGRAD, dict(codes=None)), ("weight_grad", WGRAD, dict(codes=P + 8)), ("weight_grad", WGRAD, dict(exps=None)),
    ("weight_grad", WGRAD, dict(dw=None)), ("weight_grad", WGRAD, dict(dtype=2)), ("weight_grad", WGRAD, dict(out_dtype=2)),
])
def test_invalid_arguments(name, good, bad):
    assert _call(name, good, **bad) == hm.ERR_INVALID_ARG


@pytest.mark.parametrize("name,good,bad", [
    ("embed", EMBED, dict(n=1 << 31)), ("embed", EMBED, dict(rows=1 << 31)), ("embed_grad", GRAD, dict(n=1 << 31)),
    ("embed_grad", GRAD, dict(rows=1 << 31)), ("act_pack", PACK, dict(n=1 << 31)), ("act_unpack", UNPACK, dict(n=1 << 31)),
    ("weight_grad", WGRAD, dict(n=1 << 31)), ("weight_grad", WGRAD, dict(out=1 << 27, ld_grad=1 << 27)),
    ("weight_grad", WGRAD, dict(cols=1 << 27, ld_dw=1 << 27)),
])
def test_sizes_beyond_the_kernels(name, good, bad):
    assert _call(name, good, **bad) == hm.ERR_UNSUPPORTED


def test_workspaces():
    L = hm.lib()
    need = L.himuon_embed_grad_workspace_size(100000, 10, 8)
    assert need > 0 and L.himuon_embed_grad_workspace_size(-1, 10, 8) == 0 and L.himuon_embed_grad_workspace_size(4, 0, 8) == 0
    assert L.himuon_embed_grad_workspace_size(4, 10, 8) == 0  # a short batch needs none
    for bad in (dict(ws=None), dict(ws=P + 8), dict(ws_bytes=need - 1)):
        assert _call("embed_grad", GRAD, n=100000, **bad) == hm.ERR_WORKSPACE
    # keys and positions twice, and two partial rows a chunk of 32 tokens
    assert L.himuon_embed_grad_workspace_size(65536, 32000, 4096) < 65536 * 16 + 65536 // 32 * 2 * 4096 * 4 + (1 << 20)
    # the gradient is read in place if it can be: an odd address or fp32 needs room for its terms
    size = L.himuon_weight_grad_workspace_size
    T, O, C = 8192, 11008, 4096
    small = size(T, O, C, P, O, hm.BF16)
    assert 0 < small < 8 << 20 and size(64, 16, 8, P, 16, hm.BF16) == 0
    assert size(T, O, C, P + 2, O, hm.BF16) >= T * O * 2 and size(T, O, C, P, O + 1, hm.BF16) >= T * O * 2
    assert size(T, O, C, P, O, hm.F32) >= 3 * T * O * 2
    assert size(T, O, C, P, O - 1, hm.BF16) == 0 and size(T, 0, C, P, O, hm.BF16) == 0 and size(T, O, C, P, O, 7) == 0
    need = size(9000, 700, 1000, P, 700, hm.BF16)
    for bad in (dict(ws=None), dict(ws=P + 16), dict(ws_bytes=need - 1)):
        assert _call("weight_grad", WGRAD, n=9000, out=700, cols=1000, ld_grad=700, ld_dw=1000, **bad) == hm.ERR_WORKSPACE
    size = L.himuon_qk_norm_rope_grad_workspace_size
    assert size(2, 3, 64) > 0 and size(2, 3, 0) == 0 and size(2, 3, 514) == 0 and size(-1, 3, 64) == 0
    assert size(1 << 20, 1 << 20, 64) == 0


def _qk(**bad):
    f = dict(batch=2, seq=4, hq=2, hk=1, dim=64, rot=64, inter=0, dtype=hm.F32, gain=hm.F32, index=ops.I64, wq=P, wk=P, cos=P, sin=P,
             rows=100, pos=P, eps=1e-6)
    f.update(bad)
    return ops._QK.pack(*f.values())


HEADS = ops._HEADS.pack(P, 512, 128, 64)
NONE = ops._HEADS.pack(0, 512, 128, 64)


@pytest.mark.parametrize("bad", [dict(batch=-1), dict(seq=-1), dict(hq=0), dict(hk=0), dict(dim=0), dict(dim=63), dict(rot=66),
                                 dict(rot=63), dict(rot=-2), dict(dtype=2), dict(gain=-1), dict(index=2), dict(wq=0), dict(wk=0),
                                 dict(cos=0), dict(sin=0), dict(rows=-1), dict(eps=-1.0), dict(eps=float("nan")),
                                 dict(eps=float("inf"))])
def test_qk_invalid_arguments(bad):
    L = hm.lib()
    assert L.himuon_qk_norm_rope(_qk(**bad), HEADS, HEADS, HEADS, HEADS, None) == hm.ERR_INVALID_ARG
    assert L.himuon_qk_norm_rope_grad(_qk(**bad), HEADS, HEADS, HEADS, HEADS, HEADS, HEADS, P, P, P, BIG, None) == hm.ERR_INVALID_ARG


def test_qk_pointers_and_limits():
    L = hm.lib()
    for i in range(4):
        heads = [NONE if i == j else HEADS for j in range(4)]
        assert L.himuon_qk_norm_rope(_qk(), *heads, None) == hm.ERR_INVALID_ARG
    assert L.himuon_qk_norm_rope(None, HEADS, HEADS, HEADS, HEADS, None) == hm.ERR_INVALID_ARG
    assert L.himuon_qk_norm_rope(_qk(), None, HEADS, HEADS, HEADS, None) == hm.ERR_INVALID_ARG
    for i in range(6):
        heads = [NONE if i == j else HEADS for j in range(6)]
        assert L.himuon_qk_norm_rope_grad(_qk(), *heads, P, P, P, BIG, None) == hm.ERR_INVALID_ARG
    six = [HEADS] * 6
    assert L.himuon_qk_norm_rope_grad(_qk(), *six, None, P, P, BIG, None) == hm.ERR_INVALID_ARG
    assert L.himuon_qk_norm_rope_grad(_qk(), *six, P, P, None, BIG, None) == hm.ERR_WORKSPACE
    assert L.himuon_qk_norm_rope_grad(_qk(), *six, P, P, P, 16, None) == hm.ERR_WORKSPACE
    assert L.himuon_qk_norm_rope(_qk(dim=514), HEADS, HEADS, HEADS, HEADS, None) == hm.ERR_UNSUPPORTED
    assert L.himuon_qk_norm_rope(_qk(batch=1 << 20, seq=1 << 20), HEADS, HEADS, HEADS, HEADS, None) == hm.ERR_UNSUPPORTED


def test_empty_calls_enqueue_nothing():
    L = hm.lib()
    assert _call("embed", EMBED, n=0, tokens=None, out=None) == hm.OK
    assert _call("embed_grad", GRAD, n=0, tokens=None, grad=None, accumulate=1) == hm.OK
    assert _call("act_pack", PACK, n=0, x=None, codes=None, exps=None) == hm.OK
    assert _call("act_unpack", UNPACK, n=0, x=None, codes=None, exps=None) == hm.OK
    assert _call("weight_grad", WGRAD, n=0, grad=None, codes=None, exps=None, accumulate=1) == hm.OK
    assert L.himuon_qk_norm_rope(_qk(seq=0), NONE, NONE, NONE, NONE, None) == hm.OK


def test_tensors_of_the_wrong_kind():
    torch = pytest.importorskip("torch")
    t, x = torch.zeros(4, dtype=torch.int64), torch.zeros(4, 8)
    for f in (lambda: hm.embed(t, x), lambda: hm.embed_grad(t, x, 10), lambda: hm.act_pack(x),
              lambda: hm.act_unpack(torch.zeros(1, 8, 32, dtype=torch.uint8), torch.zeros(1, 8, dtype=torch.uint8), 4),
              lambda: hm.weight_grad(x, torch.zeros(1, 8, 32, dtype=torch.uint8), torch.zeros(1, 8, dtype=torch.uint8)),
              lambda: hm.qk_norm_rope(x[None], x[None], x[0], x[0], x, x)):
        with pytest.raises(ValueError):
            f()


def test_the_bindings_constants_and_layouts_are_the_headers(tmp_path):
    src = open(os.path.join(ROOT, "include", "himuon.h")).read()
    assert int(re.search(r"#define HIMUON_MAX_HEAD_DIM (\d+)", src)[1]) == ops.MAX_HEAD_DIM
    assert int(re.search(r"#define HIMUON_ACT_GROUP (\d+)", src)[1]) == ops.ACT_GROUP
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    prog = tmp_path / "layout.c"
    prog.write_text('#include "himuon.h"\n#include <stdio.h>\nint main(void) { himuon_qk_t q = {2, 4, 2, 1, 64, 32, 1, 0, 1, 1, '
                    '(void*)1, (void*)2, (float*)3, (float*)4, 100, (void*)5, 0.5f}; himuon_heads_t h = {(void*)6, 7, 8, 9};\n'
                    'fwrite(&q, sizeof q, 1, stdout); fwrite(&h, sizeof h, 1, stdout); return 0; }\n')
    exe = tmp_path / "layout"
    subprocess.run([cc, "-I", os.path.join(ROOT, "include"), str(prog), "-o", str(exe)], check=True)
    got = subprocess.run([str(exe)], check=True, capture_output=True).stdout
    want = ops._QK.pack(2, 4, 2, 1, 64, 32, 1, 0, 1, 1, 1, 2, 3, 4, 100, 5, 0.5) + ops._HEADS.pack(6, 7, 8, 9)
    assert len(got) == len(want) == ops._QK.size + ops._HEADS.size
    pad = struct.calcsize("@2q8i4PqPf")  # (what follows eps is padding)
    assert got[:pad] == want[:pad] and got[ops._QK.size:] == want[ops._QK.size:]
