"""Which kernel of the weight gradient each size of the GPU tests runs on: a change of the
rule must not leave one of them without a test."""
import os
import shutil
import subprocess

import pytest
import test_gpu_act8 as act8
import test_gpu_wgrad_tiles as tiles

import paper_2606_27216_amd as hm

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
TILES = ["direct", "128 pair", "128", "256"]
PROGRAM = r"""
#include "wgrad_plan.h"
#include <cstdio>
int main()
{
    long long t, o, c, ld, at;
    int dtype;
    while (scanf("%lld %lld %lld %lld %lld %d", &t, &o, &c, &ld, &at, &dtype) == 6) {
        const himuon::WgradPlan g = himuon::plan_wgrad(t, o, c, reinterpret_cast<const void*>((uintptr_t)at), ld, dtype);
        printf("%d %d %d %zu\n", (int)g.tile, g.splits, (int)g.stage, g.total);
    }
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    """(tile, splits, laid out, workspace) of (tokens, rows, columns, type), rows side by side."""
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    d = tmp_path_factory.mktemp("plan")
    (d / "plan.cpp").write_text(PROGRAM)
    subprocess.run([cxx, "-std=c++17", "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2606_27216_amd", "csrc"),
                    str(d / "plan.cpp"), "-o", str(d / "plan")], check=True)

    def ask(cases):
        lines = "".join(f"{t} {o} {c} {o} 4096 {hm.BF16 if dtype == 'bf16' else hm.F32}\n" for t, o, c, dtype in cases)
        out = subprocess.run([str(d / "plan")], input=lines, check=True, capture_output=True, text=True).stdout.split("\n")
        return [(TILES[int(tile)], int(splits), bool(int(stage)), int(total)) for tile, splits, stage, total in
                (line.split() for line in out if line)]

    return ask


def _both(shapes):
    return [(*s, dtype) for s in shapes for dtype in ("bf16", "f32")]


def test_the_librarys_plan_is_this_one(plan):
    cases = _both(act8.WSIZES + act8.LARGE + tiles.WHOLE + tiles.SPLIT)
    for (t, o, c, dtype), (*_, total) in zip(cases, plan(cases)):
        code = hm.BF16 if dtype == "bf16" else hm.F32
        assert hm.lib().himuon_weight_grad_workspace_size(t, o, c, 4096, o, code) == total


def test_sizes_of_256_tiles(plan):
    assert all((tile, splits) == ("256", 1) for tile, splits, *_ in plan(_both(tiles.WHOLE)))
    assert all((tile, splits) == ("256", 2) for tile, splits, *_ in plan(_both(tiles.SPLIT)))
    # the last group of tokens is cut, and bf16 gradients are read in place and laid out
    assert all(t % 32 for t, _, _ in tiles.WHOLE + tiles.SPLIT)
    for shapes in (tiles.WHOLE, tiles.SPLIT):
        assert {stage for _, _, stage, _ in plan([(*s, "bf16") for s in shapes])} == {False, True}
    rows, cols = tiles.WHOLE[2][1:]
    assert -(-rows // 256) * -(-cols // 256) > 512  # three rounds over 256 CUs


def test_every_kernel_has_a_test(plan):
    """Each tile with and without partial sums (128-tiles are never split), gradients in place and laid out
    (the direct kernel lays none out), fp32 and bf16."""
    cases = _both(act8.WSIZES + act8.LARGE + tiles.WHOLE + tiles.SPLIT)
    seen = {(tile, splits > 1, stage, dtype) for (*_, dtype), (tile, splits, stage, _) in zip(cases, plan(cases))}
    for tile in TILES:
        for split in (False, True):
            if (tile, split) == ("128", True):
                continue
            assert (tile, split, tile != "direct", "f32") in seen, (tile, split)
            for stage in (False, True):
                if not (tile == "direct" and stage):
                    assert (tile, split, stage, "bf16") in seen, (tile, split, stage)
