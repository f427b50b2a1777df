// Which kernels a call of attention and of its gradient runs on (attention.hip, attention_grad.hip):
// plain C++, so that the rule can be asked without a GPU. Arguments have been checked.
#pragma once

#include "himuon.h"
#include "sizes.h"

#include <algorithm>

namespace himuon {
namespace attn {

constexpr int kRows = 32;          // of a wave: rows or columns of a product's tile
constexpr int kTileRows = 4 * kRows;  // of a block of four waves with rows of their own
constexpr int kFewLds = 128 << 10;

// Columns that a head's products run over.
inline int padded_dim(int64_t dim) { return dim <= 64 ? 64 : dim <= 128 ? 128 : 256; }

// Blocks of one tile of `tile` rows and one key head (KEYS: keys, else pairs of a query and a head of the group).
struct AttnTiles {
    int64_t slots, blocks;  // slots: tiles of a sequence, or of the packed array; blocks: -1 past 2^62
};
template <bool KEYS> AttnTiles attn_tiles(bool packed, int64_t batch, int64_t len, int64_t group, int64_t k_heads, int tile)
{
    const int64_t rows = KEYS ? len : len * group;
    AttnTiles t;
    t.slots = packed ? rows / tile + batch + 2 : ceil_div(rows, tile);
    const int64_t items = packed ? t.slots : t.slots * batch;
    t.blocks = small_product(items, k_heads) ? items * k_heads : -1;
    return t;
}

// A token or some of each sequence against many keys: the waves of a block share the 32 rows that a group of heads
// has, and take the keys in pieces. One query a sequence, 32 + 8 heads of 128, bf16, us in this form / in the others:
// 1 x 4096 keys to each of 4 sequences 23 / 71, 512 16 / 14, 128 11.7 / 12.1; 64 sequences with 48 keys 14.9 / 12.2, 128
// 14.9 / 12.2, 512 28 / 23, 2048 96 / 86 (heads of sequences enough to fill the chip: the others are faster).
inline bool few_rows(const himuon_attn_t& a) { return !a.q_starts && a.q_len * (a.q_heads / a.k_heads) <= kRows && a.k_len > 64; }

// Blocks that share the keys of a group of heads: as many as fill the chip, one to a CU. The same calls with 128 / 256 / 512
// blocks, us: 1 x 32768 keys 45 / 44 / 63, 4 x 4096 27 / 23 / 30, 8 x 4096 42 / 30 / 36, 16 x 4096 84 / 56 / 57, 4 x 32768 159 / 100 / 101,
// 1 x 8192 23 / 28 / 28. One, two or four tiles to a wave at least: 1 x 2048 19.1 / 16.5 / 16.3, 1 x 8192 28 / 28 / 23.
inline int64_t few_splits(const himuon_attn_t& a)
{
    const int64_t es = a.dtype == HIMUON_BF16 ? 2 : 4;
    const int64_t waves = std::min<int64_t>(4, kFewLds / (4 * kRows * padded_dim(a.head_dim) * es));
    const int64_t most = ceil_div(a.k_len, kRows * waves * 2);  // two tiles to a wave
    return std::max<int64_t>(1, std::min<int64_t>(most, ceil_div(256, a.batch * a.k_heads)));
}

// The forward pass: the keys of 32 rows shared out over waves (few rows: over blocks too), or 32 rows to a wave.
enum class Forward : int { FEW_ROWS, FEW_TILES, LONG };

// Blocks of four times 32 rows below which the waves of a block share 32 of them. Heads of 128, 16 + 8 of
// them, causal, first form / second, us: 1 x 128 tokens (16 blocks) bf16 11.4 / 11.2, fp32 28 / 20; 1 x 512
// (64) 17 / 14 and 81 / 62; 2 x 512 (128) 18 / 25 and 83 / 109.
constexpr int64_t kSharedBelow = 96;

inline Forward plan_forward(const himuon_attn_t& a)
{
    if (few_rows(a)) return Forward::FEW_ROWS;
    const int64_t blocks = attn_tiles<false>(a.q_starts != nullptr, a.batch, a.q_len, a.q_heads / a.k_heads, a.k_heads, kTileRows).blocks;
    return blocks >= 0 && blocks < kSharedBelow ? Forward::FEW_TILES : Forward::LONG;
}

// The gradient: which sides' tiles are shared by the waves of a block (a side without tokens has no blocks).
struct GradPlan {
    bool q_shared, k_shared;
};

// Blocks of four times 32 keys (rows) below which the waves of a block share 32 of them: where the
// first kind leaves the chip idle, with one wave on the long way over the other side's tiles. Heads of 128,
// 16 + 8 of them, causal, first form / second, us: fp32 1 x 128 tokens 111 / 38 (8 blocks of keys, 16 of
// rows), 1 x 512 382 / 109 (32, 64), 2 x 1024 747 / 386 (128, 256), 4 x 1024 774 / 771 (256, 512; keys in the second
// and rows in the first 660), 8 x 1024 1093 / 1551; bf16 1 x 128 29 / 20, 1 x 512 57 / 35, 2 x 512 59 / 46 (64, 128;
// keys in the second and rows in the first 50), 4 x 512 61 / 79 (128, 256).
inline GradPlan plan_grad(bool f32, int64_t q_blocks, int64_t k_blocks)
{
    GradPlan g;
    g.k_shared = k_blocks > 0 && k_blocks < (f32 ? 512 : 96);
    g.q_shared = q_blocks > 0 && q_blocks < (f32 ? 512 : g.k_shared ? 192 : 96);
    return g;
}

}  // namespace attn
}  // namespace himuon
