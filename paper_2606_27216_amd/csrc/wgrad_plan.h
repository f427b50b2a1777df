// Which kernel a weight gradient runs on (act8_ops.hip), and the workspace that it takes: plain
// C++, so that the rule can be asked without a GPU.
#pragma once

#include "himuon.h"
#include "sizes.h"

#include <algorithm>

namespace himuon {

// Which kernel a call runs on.
enum class Tile : int { DIRECT, B128_PAIR, B128, B256 };

struct WgradPlan {
    Tile tile;
    bool stage;
    int terms, splits;
    int64_t pitch, exp_pitch, groups, part_pitch;
    size_t exps_at, part_at, total;
};

// The rule goes by the workgroups that each tile gives the 256 CUs and by the slices that
// each of them walks over. Measured, us a call, bf16 / fp32 gradients, tokens x rows x columns:
//   - DIRECT while two rounds of 64-tiles serve and a workgroup has at most 128 groups to
//     share out over its waves. Against B128_PAIR: 1024^3 9.3 / 12.0 (15.2 / 26.8), 4096 x
//     1024^2 20.0 / 35.4 (23.6 / 41.6), 512 x 1536 x 1280 10.0 / 15.4 (9.9 / 26.3); beyond:
//     8192 x 1024^2 34.7 / 72.9 (26.8 / 68.3), 512 x 2048^2 17.3 / 30.0 (10.5 / 24.5).
//   - B128_PAIR (two groups of waves to a tile) while there are no more tiles than CUs:
//     512 x 2048^2 10.5 / 24.5 (B128, split in two, 24.9 / 34.6); 512 tiles of 4096 x 2048
//     at 1024 tokens 25.0 / 63.5 (B128 23.0 / 59.7).
//   - B256 or B128 by their rounds over the chip, in slices of a 256-tile (about 0.62 us): a
//     round of 256-tiles takes its slices and 8 for its ends, each split 15 for the join; a
//     CU works 128-tiles off at 0.345 a slice, three of them at a time. Measured, B256 and
//     B128: 4096^2 (256 tiles) at 256, 1024, 8192 tokens 21.0 and 18.9, 39.3 and 39.3, 202 and
//     244; 4928 x 3264 (260 tiles, two rounds) at 2681 tokens 141 and 88; 11008 x 4096 (688
//     tiles) at 256, 2048 55 and 38, 171 and 171; 2048 x 4096 (128 tiles, two splits) at 4096,
//     16384 75 and 67, 214 and 249.
inline WgradPlan plan_wgrad(int64_t tokens, int64_t out, int64_t cols, const void* grad, int64_t ld, int dtype)
{
    WgradPlan g;
    g.groups = ceil_div(tokens, HIMUON_ACT_GROUP);
    g.terms = dtype == HIMUON_F32 ? 3 : 1;
    const int64_t slices = g.groups * g.terms;
    const int64_t t64 = ceil_div(out, 64) * ceil_div(cols, 64);
    const int64_t t128 = ceil_div(out, 128) * ceil_div(cols, 128);
    const int64_t t256 = ceil_div(out, 256) * ceil_div(cols, 256);
    auto split = [](int64_t workgroups, int64_t tiles, int64_t parts) {
        return std::max<int64_t>(1, std::min<int64_t>(workgroups / tiles, parts));
    };
    const int64_t direct = split(256, t64, g.groups / 32);
    int64_t splits;
    if (t64 <= 512 && ceil_div(t64, 256) * g.groups <= 128 * direct && ld < (INT64_C(1) << 24)) {
        g.tile = Tile::DIRECT;
        splits = direct;
    } else if (t128 <= 256) {
        g.tile = Tile::B128_PAIR;
        splits = split(256, t128, slices / 16);
    } else {
        splits = split(256, t256, slices / 8);
        const double by256 = (double)ceil_div(t256 * splits, 256) * ((double)slices / (double)splits + 8) + 4 +
                             (splits > 1 ? 15. * (double)splits : 0.);
        const double by128 = 0.345 * (double)ceil_div(t128, 256) * (double)slices + 8;
        g.tile = by256 <= by128 ? Tile::B256 : Tile::B128;
        if (g.tile == Tile::B128) splits = 1;
    }
    g.splits = (int)splits;
    g.stage = g.tile != Tile::DIRECT &&
              (dtype == HIMUON_F32 || out % 8 || ld % 8 || ((uintptr_t)grad & 15) || ld >= (INT64_C(1) << 26));
    g.pitch = (int64_t)round_up((size_t)out, 8);
    g.exp_pitch = (int64_t)round_up((size_t)cols, 4);
    g.part_pitch = g.exp_pitch;
    size_t at = g.stage ? round_up((size_t)slices * HIMUON_ACT_GROUP * (size_t)g.pitch * 2, 256) : 0;
    g.exps_at = at;
    // (the exponents of whole rows of 4 bytes at an aligned address are read in place)
    if (g.tile != Tile::DIRECT) at += round_up((size_t)g.groups * (size_t)g.exp_pitch, 256);
    g.part_at = at;
    if (g.splits > 1) at += round_up((size_t)g.splits * (size_t)out * (size_t)g.part_pitch * 4, 256);
    g.total = at;
    return g;
}

// Whether the plan's workgroups are a launch that can be made.
inline bool tiles_launchable(const WgradPlan& g, int64_t out, int64_t cols)
{
    const int64_t edge = g.tile == Tile::DIRECT ? 64 : g.tile == Tile::B256 ? 256 : 128;
    return launchable(ceil_div(out, edge) * ceil_div(cols, edge) * g.splits, g.tile == Tile::B128 ? 256 : 512);
}

}  // namespace himuon
