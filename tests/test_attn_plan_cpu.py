"""Which kernels of attention and its gradient the GPU tests' sizes run on: a change of the rule must not
leave one of them without a test."""
import os
import shutil
import subprocess

import pytest
import test_gpu_attention_tiles as tiles

import paper_2606_27216_amd as hm
from paper_2606_27216_amd import block_ops, train_ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x10000
PROGRAM = r"""
#include "attn_plan.h"
#include <cstdio>
int main()
{
    himuon_attn_t a{};
    long long batch, q_len, k_len;
    int packed;
    while (scanf("%lld %lld %lld %d %d %d %d %d", &batch, &q_len, &k_len, &a.q_heads, &a.k_heads, &a.head_dim, &a.dtype, &packed) == 8) {
        using namespace himuon::attn;
        a.batch = batch;
        a.q_len = q_len;
        a.k_len = k_len;
        a.q_starts = a.k_starts = packed ? &a : nullptr;
        const int group = a.q_heads / a.k_heads;
        const auto q = attn_tiles<false>(packed, batch, q_len, group, a.k_heads, kTileRows), k = attn_tiles<true>(packed, batch, k_len, group, a.k_heads, kTileRows);
        const GradPlan g = plan_grad(a.dtype == HIMUON_F32, q_len > 0 ? q.blocks : 0, k_len > 0 ? k.blocks : 0);
        printf("%d %lld %d %d\n", (int)plan_forward(a), few_rows(a) ? (long long)few_splits(a) : 0, (int)g.q_shared, (int)g.k_shared);
    }
}
"""
FORMS = ["few rows", "few tiles", "long"]


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    """(form of the forward pass, splits, queries' side shared, keys' side shared) of
    (batch, queries, keys, heads, key heads, head, type, packed)."""
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    d = tmp_path_factory.mktemp("plan")
    (d / "plan.cpp").write_text(PROGRAM)
    subprocess.run([cxx, "-std=c++17", "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2606_27216_amd", "csrc"),
                    str(d / "plan.cpp"), "-o", str(d / "plan")], check=True)

    def ask(cases):
        lines = "".join(f"{b} {n} {m} {h} {k} {c} {hm.BF16 if t == 'bf16' else hm.F32} {int(p)}\n" for b, n, m, h, k, c, t, p in cases)
        out = subprocess.run([str(d / "plan")], input=lines, check=True, capture_output=True, text=True).stdout.split("\n")
        return [(FORMS[int(f)], int(s), q == "1", k == "1") for f, s, q, k in (line.split() for line in out if line)]

    return ask


def _cases():
    return [(*c[:7], False) for c in tiles.BATCHES] + [(len(s) - 1, n, n, h, k, c, t, True) for s, n, h, k, c, t in tiles.PACKED]


def test_the_long_kernels_run(plan):
    cases = _cases()
    assert all(p == ("long", 0, False, False) for p in plan(cases))


def test_every_form_of_the_long_kernels_has_a_test():
    """Each width of the products in both types: whole heads that are aligned, cut ones, unaligned rows; with
    more than eight tiles of 32 on the side that is walked over, which is more than a ring of LDS buffers holds twice."""
    seen = set()
    for batch, nq, nk, hq, hk, dim, dtype, layout in tiles.BATCHES:
        width = 64 if dim <= 64 else 128 if dim <= 128 else 256
        kind = "unaligned" if layout == "odd" else "whole" if dim == width else "cut"
        assert dim % (8 if dtype == "bf16" else 4) == 0  # (else a row would not be whole chunks)
        if nk > 256 and nq * (hq // hk) > 256:
            seen.add((width, dtype, kind))
    for dtype in ("bf16", "f32"):
        for width in (64, 128, 256):
            assert (width, dtype, "whole") in seen and (width, dtype, "unaligned") in seen
        for width in (128, 256):
            assert (width, dtype, "cut") in seen
        assert {dim for *_, dim, t in tiles.PACKED if t == dtype} == {64, 128, 256}
        # one, two, three heads to a group and (bf16) more than 32
        groups = {hq // hk for _, _, _, hq, hk, _, t, _ in tiles.BATCHES if t == dtype}
        assert {1, 2, 3} <= groups and (dtype == "f32" or max(groups) > 32)


def test_the_librarys_splits_are_these(plan):
    cases = [(b, n, m, h, k, c, t, False) for b in (1, 3, 40, 300) for n, h, k in ((1, 8, 2), (4, 16, 2), (32, 1, 1), (33, 1, 1), (1, 64, 1))
             for m in (64, 65, 1000, 40000) for c in (64, 72, 256) for t in ("bf16", "f32")]
    for (b, n, m, h, k, c, t, _), (form, splits, *_) in zip(cases, plan(cases)):
        args = block_ops._ATTN.pack(b, n, m, h, k, c, 1, hm.BF16 if t == "bf16" else hm.F32, train_ops.I32, 0, 0, 0, 0, 0.1)
        width = 64 if c <= 64 else 128 if c <= 128 else 256
        need = b * k * splits * 32 * (width + 4) * 4 if splits > 1 else 0
        assert hm.lib().himuon_attention_workspace_size(args) == need
        assert (form == "few rows") == (n * (h // k) <= 32 and m > 64)
