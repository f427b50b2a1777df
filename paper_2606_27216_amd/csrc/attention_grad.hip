// The backward pass of attention (himuon_attention_grad).
//
//     p = exp(c q k^T - lse),  D = rowsum(g o),  ds = p (g v^T - D)
//     dv = p^T g,  dk = c ds^T q,  dq = c ds k
// from the forward pass's inputs, o and lse. Two kernels: one whose waves hold 32 rows of queries
// and walk over the keys (dq; it also leaves every row's lse and D behind for the other one), and
// one whose waves hold 32 keys and walk over the rows of the head's whole group (dk, dv). (Few
// tiles: both in one launch, behind one that computes lse and D.) Scores
// are computed in both: seven products instead of five, but no sum is shared between blocks, so
// that results have one order of summation and there are no atomics. As in the forward pass p and
// ds are a product's second operand as they stand.
//
// What bounds it: the issue of instructions, and in the keys' kernel one wave to a SIMD, as its
// registers hold two operands and two sums of 32 keys (causal bf16, 16 x 1024 tokens, 16 + 8 heads of 128:
// queries' side 145 us, keys' 200, the matrix cores busy in 38% and 36% of their cycles and LDS read in 19% and 22% of a
// CU's; 2 x 4096 with 32 + 8 heads 890 both, 0.77 PFLOP/s of the five products that the mathematics asks for); in
// fp32 the products (8 x 1024 tokens 1090 us). Heads of more than 128 columns in fp32: each of a result's parts forms the
// scores and g v^T for itself, 27 products for 5 (8 x 1024 tokens, 16 + 8 heads of 256: 8.2 ms).
//
// bf16 p and ds are rounded to bf16 for their products, as in the forward pass: gradients are off by 0.0024 to 0.0027 of
// their size, 0.0017 to 0.0022 if only they are rounded. fp32 arrays keep them in fp32.
#include "attn_device.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

namespace himuon {
namespace attn {
namespace {

constexpr int kThreads = 256;
static_assert(kTileRows == kRows * kThreads / 64, "");

// Tiles of 32 rows lie in a ring of LDS buffers. A tile's g v^T goes out beside its exponentials, and
// in bf16 the next tile's scores beside its ds, as long as registers hold both; fp32 products take
// sixteen times as long, and ds does not weigh.
template <GemmStore ST, int DP> constexpr bool ahead() { return ST == GemmStore::BF16 && DP <= 128; }
template <GemmStore ST, int DP> constexpr int ring() { return ahead<ST, DP>() ? 4 : 2; }

// x = rows of a tile in LDS times 32 rows held as fragments; `work(i)` goes out beside the products,
// i = 0 .. NS - 1.
template <GemmStore ST, int DP, class Work>
HM_DEV void row_product(f32x16& x, const uint8_t* tile, const Frag<ST> (&f)[DP / 16], int lane, Work work)
{
    using L = Lay<ST, DP>;
    auto read = [=](int i) __attribute__((always_inline)) { return L::row_frag(tile, lane & 31, i, lane >> 5); };
    Ahead<Frag<ST>, DP / 16, kDepth<ST, DP>> r;
    x = f32x16{};
    r.fill(read);
    r.run(read, [&](int i, const Frag<ST>& a) {
        mma<ST>(x, a, f[i]);
        work(i);
    });
}

// The same, of the first `steps` parts of 16 columns alone.
template <GemmStore ST, int DP> HM_DEV void row_product_of(int steps, f32x16& x, const uint8_t* tile, const Frag<ST> (&f)[DP / 16], int lane)
{
    auto read = [=](int i) __attribute__((always_inline)) { return Lay<ST, DP>::row_frag(tile, lane & 31, i, lane >> 5); };
    Ahead<Frag<ST>, DP / 16, kDepth<ST, DP>> r;
    x = f32x16{};
    r.fill(read);
    r.run(read, [&](int i, const Frag<ST>& a) {
        if (i < steps) mma<ST>(x, a, f[i]);
    });
}

// acc[t] += columns 32 (t0 + t) .. of a tile times an operand, t below `cols`.
template <GemmStore ST, int DP, int DT>
HM_DEV void col_product(f32x16 (&acc)[DT], const uint8_t* tile, const Frag<ST> (&f)[2], int t0, int cols, int lane)
{
    auto read = [=](int i) __attribute__((always_inline)) { return Lay<ST, DP>::col_frag(tile, 16 * (i & 1), 32 * (t0 + (i >> 1)), lane); };
    Ahead<Frag<ST>, 2 * DT, kDepth<ST, DP>> r;
    r.fill(read);
    r.run(read, [&](int i, const Frag<ST>& a) {
        if (i >> 1 < cols) mma<ST>(acc[i >> 1], a, f[i & 1]);
    });
}

// A row in memory times one held as fragments.
template <bool VEC, GemmStore ST, int DP> HM_DEV float row_dot(const Frag<ST> (&g)[DP / 16], const uint8_t* row, bool on, int dim, int h)
{
    float d = 0.f;
#pragma unroll
    for (int i = 0; i < DP / 16; i += 4) {
        Frag<ST> o[4];
        load_row<VEC, ST, 64>(o, row + 16 * i * Lay<ST, DP>::ES, on, dim - 16 * i, h);
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) d = fmaf(frag_value<ST>(g[i + j], e), frag_value<ST>(o[j], e), d);
        __builtin_amdgcn_sched_barrier(0);
    }
    return add_halves(d);
}

// The part of 16 elements, in pairs, that step i of N does.
template <int N> HM_DEV constexpr int share_of(int i) { return (16 * i / N) & ~1; }

// Row of a group's heads in `stats`.
HM_DEV int64_t stat_row(const AttnArgs& p, const Seq& s, int kh, int64_t r)
{
    const int64_t tokens = p.packed ? p.q_len : p.q_len * p.batch;
    return ((int64_t)kh * tokens + (int64_t)s.batch * p.q_len + s.q0) * p.group + r;
}

// Columns of a result are cut into this many parts, each a block's, where registers hold no more.
template <GemmStore ST, int DP> constexpr int q_parts() { return ST == GemmStore::F32 && DP == 256 ? 4 : 1; }
template <GemmStore ST, int DP> constexpr int kv_parts() { return DP < 256 ? 1 : ST == GemmStore::F32 ? 8 : 2; }

template <GemmStore ST, int DP, bool DMA> __global__ void __launch_bounds__(kThreads, (ahead<ST, DP>() ? 2 : 1)) attn_grad_q(const AttnArgs p)
{
    using L = Lay<ST, DP>;
    constexpr int R = ring<ST, DP>(), TILE = kRows * L::PITCH, PARTS = q_parts<ST, DP>(), DT = L::DT / PARTS, VALUES = R * TILE;
    __shared__ __attribute__((aligned(16))) uint8_t lds[2 * R * TILE];  // [R] keys, [R] values
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x) >> 6, h = lane >> 5;
    const int G = p.group;

    const Item item = find_item<PARTS, true>(p, blockIdx.x, gridDim.x);
    const int kh = item.kh, t0 = item.part * DT;  // the first of this block's tiles of 32 columns
    const Seq s = find_seq<false, kTileRows>(p, item.item, G);
    const int rows = s.q_cap * G, r0 = s.tile * kTileRows;  // (a sequence's rows are counted in 32 bits)
    if (r0 >= rows) return;

    const int r = r0 + wave * kRows + (lane & 31);
    const int query = (int)((uint32_t)r / (uint32_t)G);
    const int head = kh * G + (int)((uint32_t)r - (uint32_t)query * (uint32_t)G);
    const bool exists = r < rows;
    const int n_lane = query < s.nq ? visible(p, s, query) : 0;
    const bool on = n_lane > 0;  // (a row that sees nothing has no gradient)
    Frag<ST> q[L::NS], g[L::NS];
    load_row<DMA, ST, DP>(q, at(p.q, s.batch, s.q0 + query, head), on, p.dim, h);
    load_row<DMA, ST, DP>(g, at(p.g, s.batch, s.q0 + query, head), on, p.dim, h);
    const float d = row_dot<DMA, ST, DP>(g, at(p.o, s.batch, s.q0 + query, head), on, p.dim, h);
    const float c = p.scale * kLog2e;
    // (infinity: whatever the row's scores are, its p are zero)
    const float lse = on ? p.lse[((int64_t)s.batch * p.q_len + s.q0 + query) * ((int64_t)p.hk * G) + head] * kLog2e : INFINITY;
    if (exists && h == 0 && t0 == 0) p.stats[stat_row(p, s, kh, r)] = float2{lse, d};

    // tiles of keys that the block's and the wave's rows see; keys seen by all of the wave's rows
    const int w0 = r0 + wave * kRows, in_use = s.nq * G;
    auto seen = [&](int row) { return row < in_use ? visible(p, s, (int)((uint32_t)row / (uint32_t)G)) : 0; };
    const int tiles = (seen(min(r0 + kTileRows, in_use) - 1) + kRows - 1) / kRows * (r0 < in_use);
    const int mine = (seen(min(w0 + kRows, in_use) - 1) + kRows - 1) / kRows * (w0 < in_use);
    const int n_all = seen(w0), whole = min(tiles, s.nk / kRows);

    f32x16 dq[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t) dq[t] = f32x16{};
    const int row_bytes = p.dim * L::ES;
    const uint8_t *kp = at(p.k, s.batch, s.k0, kh), *vp = at(p.v, s.batch, s.k0, kh);
    const Share<ST, DP, kRows, kThreads> share{(int)threadIdx.x};
    constexpr int NI = Share<ST, DP, kRows, kThreads>::NI;
    const bool exact = DMA && row_bytes == L::PITCH;
    uint32_t k_off[NI], v_off[NI];
#pragma unroll
    for (int i = 0; i < NI; ++i) {
        k_off[i] = share.offset(i, p.k.ss);
        v_off[i] = share.offset(i, p.v.ss);
    }
    auto load = [&](int t, int place) __attribute__((always_inline)) {
        if (t >= tiles) return;
        auto in = [&](int i) { return t * kRows + share.row(i) < s.nk; };
        share.template stage<DMA>(lds + place * TILE, kp + t * (kRows * p.k.ss), row_bytes, t < whole, [&](int i) { return share.row(i) * p.k.ss; }, in);
        share.template stage<DMA>(lds + VALUES + place * TILE, vp + t * (kRows * p.v.ss), row_bytes, t < whole,
                                  [&](int i) { return share.row(i) * p.v.ss; }, in);
    };
    // hides the keys that this lane's row does not see
    auto hide = [&](f32x16& x, int t, float with) __attribute__((always_inline)) {
        if ((t + 1) * kRows <= n_all) return;
        const int left = n_lane - t * kRows - 4 * h;
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = result_row(i, 0) < left ? x[i] : with;
    };
    // (x: the tile's scores, next: those of the tile behind it)
    auto step = [&](int t, auto place, f32x16& x, f32x16& next) __attribute__((always_inline)) {
        const int S = place;
        if (exact && t + R - 1 < whole) {
            dev::dma_wait_barrier<(R > 3 ? R - 3 : 0) * 2 * NI>();
            share.copy(lds + (S + R - 1) % R * TILE, kp + (t + R - 1) * (kRows * p.k.ss), k_off);
            share.copy(lds + VALUES + (S + R - 1) % R * TILE, vp + (t + R - 1) * (kRows * p.v.ss), v_off);
        } else {
            dev::dma_wait_barrier<0>();
            load(t + R - 1, (S + R - 1) % R);
        }
        if (t >= mine) return;
        auto tile = [&](int u) { return lds + u % R * TILE; };
        if (!ahead<ST, DP>() || t == 0) {
            row_product<ST, DP>(x, tile(S), q, lane, [](int) {});
            hide(x, t, -INFINITY);
        }
        f32x16 y;
        row_product<ST, DP>(y, tile(S) + VALUES, g, lane, [&](int j) {
#pragma unroll
            for (int i = share_of<L::NS>(j); i < share_of<L::NS>(j + 1); ++i) {
                x[i] = __builtin_amdgcn_exp2f(fmaf(x[i], c, -lse));
                settle(x, i);
            }
        });
        hide(y, t, d);
        auto read = [&](int i) __attribute__((always_inline)) { return L::col_frag(tile(S), 16 * (i / DT), 32 * (t0 + i % DT), lane); };
        Ahead<Frag<ST>, 2 * DT, kDepth<ST, DP>> cols;
        Frag<ST> ds[2];
        auto work = [&](int from, int to) __attribute__((always_inline)) {
#pragma unroll
            for (int i = from; i < to; i += 2) {
                set_pair<ST>(ds, i / 2, x[i] * (y[i] - d), x[i + 1] * (y[i + 1] - d));
                settle_pair<ST>(ds, i / 2);
            }
        };
        if constexpr (ahead<ST, DP>()) {  // (behind the wave's last tile the next scores are nothing's, and not used)
            row_product<ST, DP>(next, tile(S + 1), q, lane, [&](int j) { work(share_of<L::NS>(j), share_of<L::NS>(j + 1)); });
            cols.fill(read);
            hide(next, t + 1, -INFINITY);
        } else {
            cols.fill(read);
            work(0, 16);
        }
        cols.run(read, [&](int i, const Frag<ST>& f) { mma<ST>(dq[i % DT], f, ds[i / DT]); });
    };
    if (tiles > 0) {
        if (DMA && p.dim < DP) {
            clear_lds<kThreads>(lds, 2 * R * TILE);
            __syncthreads();
        }
#pragma unroll
        for (int t = 0; t < R - 1; ++t) load(t, t);
        dev::dma_wait_barrier<0>();
        f32x16 x, x2;
        if constexpr (ahead<ST, DP>()) {
            for (int t = 0; t < tiles; t += R) {
                step(t, std::integral_constant<int, 0>{}, x, x2);
                if (t + 1 < tiles) step(t + 1, std::integral_constant<int, 1>{}, x2, x);
                if (t + 2 < tiles) step(t + 2, std::integral_constant<int, 2>{}, x, x2);
                if (t + 3 < tiles) step(t + 3, std::integral_constant<int, 3>{}, x2, x);
            }
        } else {
            for (int t = 0; t < tiles; ++t) step(t, t % R, x, x2);
        }
    }
    if (!exists) return;
    store_row<DMA, ST>(at(p.dq, s.batch, s.q0 + query, head) + 32 * t0 * L::ES, dq, on, p.scale, p.dim - 32 * t0, h);
}

template <GemmStore ST, int DP, bool DMA> __global__ void __launch_bounds__(kThreads) attn_grad_kv(const AttnArgs p)
{
    using L = Lay<ST, DP>;
    constexpr int R = ring<ST, DP>(), BR = kRows, TILE = BR * L::PITCH, PARTS = kv_parts<ST, DP>(), DT = L::DT / PARTS, BUF = 2 * TILE + BR * 8;
    __shared__ __attribute__((aligned(16))) uint8_t lds[R * BUF];  // [R][rows of q, of g, their lse, their D]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x) >> 6, h = lane >> 5;
    const int G = p.group;

    const Item item = find_item<PARTS, false>(p, blockIdx.x, gridDim.x);
    const int kh = item.kh, t0 = item.part * DT;
    const Seq s = find_seq<true, kTileRows>(p, item.item, 1);
    const int j0 = s.tile * kTileRows;  // (a sequence's first keys, which most queries see, first)
    if (j0 >= s.k_cap) return;
    const int key = j0 + wave * kRows + (lane & 31);
    const bool exists = key < s.k_cap, on = key < s.nk;
    Frag<ST> k[L::NS], v[L::NS];
    load_row<DMA, ST, DP>(k, at(p.k, s.batch, s.k0 + key, kh), on, p.dim, h);
    load_row<DMA, ST, DP>(v, at(p.v, s.batch, s.k0 + key, kh), on, p.dim, h);

    // rows that see keys of the block, of the wave, this lane's and all of the wave's (a
    // sequence's rows are counted in 32 bits)
    const int off = s.nk - s.nq, wj = j0 + wave * kRows;
    auto first_row = [&](int j) { return p.causal ? max(0, j - off) * G : 0; };
    // (keys behind those in use have none, and their rows no place in 32 bits)
    const int end = j0 < s.nk ? s.nq * G : 0, begin = j0 < s.nk ? first_row(j0) / BR * BR : 0;
    const bool w_whole = wj + kRows <= s.nk;
    const int w_begin = wj < s.nk ? first_row(wj) : INT32_MAX, w_all = w_whole ? first_row(wj + kRows - 1) : INT32_MAX;
    const int mine = on ? first_row(key) : INT32_MAX;

    f32x16 dk[DT], dv[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t) dk[t] = dv[t] = f32x16{};
    const float c = p.scale * kLog2e;
    const int row_bytes = p.dim * L::ES;
    // Where this thread's rows of the next tile lie: their place in the group and offsets (with
    // copy()'s own part), moved back by a tile's rows each time. (Without DMA each is worked out.)
    // The rows are walked over from the last one, which all keys' blocks read, so that blocks that
    // run together read the same rows together.
    const Share<ST, DP, BR, kThreads> share{(int)threadIdx.x};
    constexpr int NI = Share<ST, DP, BR, kThreads>::NI;
    const uint8_t *const qp = at(p.q, s.batch, s.q0, kh * G), *const gp = at(p.g, s.batch, s.q0, kh * G);
    const int step_q = BR / G, step_g = BR - step_q * G;
    const uint32_t q_step = (uint32_t)(step_q * p.q.ss + step_g * p.q.sh), g_step = (uint32_t)(step_q * p.g.ss + step_g * p.g.sh);
    const uint32_t q_wrap = (uint32_t)(p.q.ss - G * p.q.sh), g_wrap = (uint32_t)(p.g.ss - G * p.g.sh);
    auto offset = [&](int r, const Heads& x) {
        const uint32_t token = (uint32_t)r / (uint32_t)G;
        return token * x.ss + (int64_t)((uint32_t)r - token * (uint32_t)G) * x.sh;
    };
    const int tiles = end > begin ? (end - begin + BR - 1) / BR : 0;
    int place[NI];
    uint32_t q_off[NI], g_off[NI];
    if constexpr (DMA) {
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int r = begin + max(0, tiles - 1) * BR + share.row(i);
            place[i] = r % G;
            q_off[i] = (uint32_t)offset(r, p.q) + share.rest(i);
            g_off[i] = (uint32_t)offset(r, p.g) + share.rest(i);
        }
    }
    auto advance = [&]() __attribute__((always_inline)) {
        if constexpr (DMA) {
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                place[i] -= step_g;
                const bool wrap = place[i] < 0;
                place[i] += wrap ? G : 0;
                q_off[i] -= q_step + (wrap ? q_wrap : 0);
                g_off[i] -= g_step + (wrap ? g_wrap : 0);
            }
        }
    };
    const float2* const stats = p.stats + stat_row(p, s, kh, 0);
    const bool exact = DMA && row_bytes == L::PITCH;
    auto load_stats = [&](uint8_t* to, int r0) __attribute__((always_inline)) {  // (by every wave, so that all count the same)
        dev::dma4((uint32_t)__builtin_amdgcn_readfirstlane((int)dev::lds_offset(to)), 8 * (lane & 31) + 4 * h, dev::uniform_address(stats + r0));
    };
    // First row of the tile that is the u-th; all but the first one are whole.
    auto row_of = [&](int u) { return begin + (tiles - 1 - u) * BR; };
    auto load = [&](int u, int slot) __attribute__((always_inline)) {
        if (u >= tiles) return;
        uint8_t* const to = lds + slot * BUF;
        const int r0 = row_of(u);
        const bool whole = r0 + BR <= end;
        auto in = [&](int i) { return r0 + share.row(i) < end; };
        share.template stage<DMA>(to, qp, row_bytes, whole, [&](int i) {
            if constexpr (DMA) return q_off[i] - share.rest(i);
            else return offset(r0 + share.row(i), p.q);
        }, in);
        share.template stage<DMA>(to + TILE, gp, row_bytes, whole, [&](int i) {
            if constexpr (DMA) return g_off[i] - share.rest(i);
            else return offset(r0 + share.row(i), p.g);
        }, in);
        if (whole) {
            load_stats(to + 2 * TILE, r0);
        } else if (threadIdx.x < BR) {
            const float2 st = r0 + (int)threadIdx.x < end ? stats[r0 + threadIdx.x] : float2{INFINITY, 0.f};
            reinterpret_cast<float*>(to + 2 * TILE)[threadIdx.x] = st.x;
            reinterpret_cast<float*>(to + 2 * TILE)[BR + threadIdx.x] = st.y;
        }
        advance();
    };
    // hides the rows that do not see this lane's key
    auto hide = [&](f32x16& x, int u, float with) __attribute__((always_inline)) {
        const int r0 = row_of(u);
        if (r0 >= w_all) return;
        const int hidden = min(mine - r0, BR) - 4 * h;
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = result_row(i, 0) < hidden ? with : x[i];
    };
    const int own = w_begin == INT32_MAX ? 0 : tiles - max(0, w_begin - begin) / BR;  // the wave's tiles
    Ahead<Frag<ST>, L::NS, kDepth<ST, DP>> ry;
    // (x: the tile's scores, next: those of the tile behind it)
    auto step = [&](int u, auto slot, f32x16& x, f32x16& next) __attribute__((always_inline)) {
        const int S = slot;
        if (exact && u + R - 1 < tiles) {
            dev::dma_wait_barrier<(R > 3 ? R - 3 : 0) * (2 * NI + 1)>();
            uint8_t* const to = lds + (S + R - 1) % R * BUF;
            if constexpr (DMA) {
                share.copy(to, qp, q_off);
                share.copy(to + TILE, gp, g_off);
            }
            load_stats(to + 2 * TILE, row_of(u + R - 1));
            advance();
        } else {
            dev::dma_wait_barrier<0>();
            load(u + R - 1, (S + R - 1) % R);
        }
        if (u >= own) return;
        // Every product's first reads go out beside the product before (a lone wave has nothing else
        // to wait with): `ry` those of g v^T, for the next step too.
        auto tile = [&](int i) { return lds + i % R * BUF; };
        auto read_rows = [&](const uint8_t* from) { return [=](int i) __attribute__((always_inline)) { return L::row_frag(from, lane & 31, i, h); }; };
        auto read_cols = [&](const uint8_t* from) {
            return [=](int i) __attribute__((always_inline)) { return L::col_frag(from, 16 * (i / DT), 32 * (t0 + i % DT), lane); };
        };
        const auto read_y = read_rows(tile(S) + TILE), read_next = read_rows(tile(S + 1)), read_y2 = read_rows(tile(S + 1) + TILE);
        const auto read_g = read_cols(tile(S) + TILE), read_q = read_cols(tile(S));
        Ahead<Frag<ST>, L::NS, kDepth<ST, DP>> rn;
        Ahead<Frag<ST>, 2 * DT, kDepth<ST, DP>> cols_g, cols_q;
        if (!ahead<ST, DP>() || u == 0) {
            row_product<ST, DP>(x, tile(S), k, lane, [](int) {});
            ry.fill(read_y);
            hide(x, u, -INFINITY);
        }
        const float* const st = reinterpret_cast<const float*>(tile(S) + 2 * TILE) + 4 * h;
        f32x4 row[4];
        auto rows_of = [&](const float* from) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < 4; ++i) row[i] = *reinterpret_cast<const f32x4*>(from + 8 * i);
        };
        f32x16 y{};
        Frag<ST> pr[2], ds[2];
        rows_of(st);
        if constexpr (ahead<ST, DP>()) rn.fill(read_next);
        ry.run(read_y, [&](int j, const Frag<ST>& f) {
            mma<ST>(y, f, v[j]);
#pragma unroll
            for (int i = share_of<L::NS>(j); i < share_of<L::NS>(j + 1); i += 2) {
                x[i] = __builtin_amdgcn_exp2f(fmaf(x[i], c, -row[i >> 2][i & 3]));
                x[i + 1] = __builtin_amdgcn_exp2f(fmaf(x[i + 1], c, -row[i >> 2][(i & 3) + 1]));
                settle(x, i);
                settle(x, i + 1);
                set_pair<ST>(pr, i / 2, x[i], x[i + 1]);
                settle_pair<ST>(pr, i / 2);
            }
        });
        rows_of(st + BR);
        hide(y, u, 0.f);
        if constexpr (ahead<ST, DP>()) cols_g.fill(read_g);
        auto work = [&](int from, int to) __attribute__((always_inline)) {
#pragma unroll
            for (int i = from; i < to; i += 2) {
                set_pair<ST>(ds, i / 2, x[i] * (y[i] - row[i >> 2][i & 3]), x[i + 1] * (y[i + 1] - row[i >> 2][(i & 3) + 1]));
                settle_pair<ST>(ds, i / 2);
            }
        };
        if constexpr (ahead<ST, DP>()) {  // (behind the last tile the next scores are nothing's, and not used)
            next = f32x16{};
            rn.run(read_next, [&](int j, const Frag<ST>& f) {
                mma<ST>(next, f, k[j]);
                work(share_of<L::NS>(j), share_of<L::NS>(j + 1));
            });
            cols_q.fill(read_q);
            hide(next, u + 1, -INFINITY);
        } else {
            work(0, 16);
            cols_g.fill(read_g);
        }
        cols_g.run(read_g, [&](int i, const Frag<ST>& f) { mma<ST>(dv[i % DT], f, pr[i / DT]); });
        if constexpr (ahead<ST, DP>()) ry.fill(read_y2);
        else cols_q.fill(read_q);
        cols_q.run(read_q, [&](int i, const Frag<ST>& f) { mma<ST>(dk[i % DT], f, ds[i / DT]); });
    };
    if (tiles > 0) {
        if (DMA && p.dim < DP) {
            clear_lds<kThreads>(lds, R * BUF);
            __syncthreads();
        }
#pragma unroll
        for (int t = 0; t < R - 1; ++t) load(t, t);
        dev::dma_wait_barrier<0>();
        f32x16 x, x2;
        if constexpr (ahead<ST, DP>()) {
            for (int t = 0; t < tiles; t += R) {
                step(t, std::integral_constant<int, 0>{}, x, x2);
                if (t + 1 < tiles) step(t + 1, std::integral_constant<int, 1>{}, x2, x);
                if (t + 2 < tiles) step(t + 2, std::integral_constant<int, 2>{}, x, x2);
                if (t + 3 < tiles) step(t + 3, std::integral_constant<int, 3>{}, x2, x);
            }
        } else {
            for (int t = 0; t < tiles; ++t) step(t, t % R, x, x2);
        }
    }
    if (!exists) return;
    const int dim = p.dim - 32 * t0;
    store_row<DMA, ST>(at(p.dk, s.batch, s.k0 + key, kh) + 32 * t0 * L::ES, dk, on, p.scale, dim, h);
    store_row<DMA, ST>(at(p.dv, s.batch, s.k0 + key, kh) + 32 * t0 * L::ES, dv, on, 1.f, dim, h);
}

// Where tiles are few, the waves of a block share 32 rows (keys) and take the other side's tiles in
// turn, each through LDS of its own and without a barrier; their sums meet there in the end. (fp32, 901
// packed tokens in documents, 12 + 4 heads of 80: 78 us both sides, 112 in a launch of each with the same cuts; 1 x 512 tokens, 16 + 8
// heads of 128 109, of which the products' cycles on the longest block's way are 55. Copying a tile's rows in
// an order that hid them behind products changed nothing.)
constexpr int kSharedLds = 128 << 10;
template <int W, int TILE, int DT> constexpr int shared_lds() { return W * std::max(2 * TILE, kRows * (32 * DT + 4) * (int)sizeof(float)); }
template <GemmStore ST, int DP> constexpr int shared_waves() { return std::min(4, kSharedLds / (2 * kRows * Lay<ST, DP>::PITCH)); }

// The waves' sums (N of them, mul[n] times each) added in their order and stored as rows of
// `dim` elements; row r of sum n at out(n, r), zeros if it is not on(r). `lds`: the waves' own, no longer in use.
template <GemmStore ST, int W, int DT, int N, class Out, class On>
HM_DEV void join_waves(uint8_t* lds, const f32x16 (&acc)[N][DT], const float (&mul)[N], int rows, int dim, Out out, On on)
{
    constexpr int DS = 32 * DT + 4, LR = 2 * W;  // LR: lanes to a row (shared_lds() has the room)
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = lane >> 5;
    float* const sums = reinterpret_cast<float*>(lds);
#pragma unroll
    for (int n = 0; n < N; ++n) {
        __syncthreads();
        float* const own = sums + (wave * kRows + (lane & 31)) * DS;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int i = 0; i < 16; i += 4)
                *reinterpret_cast<f32x4*>(own + 32 * t + result_row(i, h)) = f32x4{acc[n][t][i], acc[n][t][i + 1], acc[n][t][i + 2], acc[n][t][i + 3]};
        __syncthreads();
        const int row = threadIdx.x / LR, x = threadIdx.x % LR;
        if (row < rows) {
            uint8_t* const to = out(n, row);
            const bool live = on(row);
            for (int d = 4 * x; d < dim && d < 32 * DT; d += 4 * LR) {
                f32x4 v = {};
#pragma unroll
                for (int u = 0; u < W; ++u) v += *reinterpret_cast<const f32x4*>(sums + (u * kRows + row) * DS + d);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (d + e < dim) put1<ST>(to, d + e, live ? v[e] * mul[n] : 0.f);
            }
        }
    }
}

// Block `id` of `n` of queries. lds: of each wave keys and values, then [waves] sums.
template <GemmStore ST, int DP, bool DMA> HM_DEV void grad_q_shared(const AttnArgs& p, uint8_t* lds, uint32_t id, uint32_t n_blocks)
{
    using L = Lay<ST, DP>;
    constexpr int W = shared_waves<ST, DP>(), TILE = kRows * L::PITCH, PARTS = q_parts<ST, DP>(), DT = L::DT / PARTS;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x) >> 6, h = lane >> 5;
    const int G = p.group;

    const Item item = find_item<PARTS, true>(p, id, n_blocks);
    const int kh = item.kh, t0 = item.part * DT;
    const Seq s = find_seq<false, kRows>(p, item.item, G);
    const int rows = s.q_cap * G, r0 = s.tile * kRows;
    if (r0 >= rows) return;

    const int r = r0 + (lane & 31);
    const int query = (int)((uint32_t)r / (uint32_t)G);
    const int head = kh * G + (int)((uint32_t)r - (uint32_t)query * (uint32_t)G);
    const int n_lane = r < rows && query < s.nq ? visible(p, s, query) : 0;
    const bool on = n_lane > 0;
    Frag<ST> q[L::NS], g[L::NS];
    load_row<DMA, ST, DP>(q, at(p.q, s.batch, s.q0 + query, head), on, p.dim, h);
    load_row<DMA, ST, DP>(g, at(p.g, s.batch, s.q0 + query, head), on, p.dim, h);
    const float2 st = r < rows ? p.stats[stat_row(p, s, kh, r)] : float2{INFINITY, 0.f};
    const float c = p.scale * kLog2e, lse = st.x, d = st.y;

    const int in_use = s.nq * G;
    auto seen = [&](int row) { return row < in_use ? visible(p, s, (int)((uint32_t)row / (uint32_t)G)) : 0; };
    const int n = r0 < in_use ? seen(min(r0 + kRows, in_use) - 1) : 0, tiles = (n + kRows - 1) / kRows, n_all = seen(r0);

    f32x16 dq[1][DT];
#pragma unroll
    for (int t = 0; t < DT; ++t) dq[0][t] = f32x16{};
    const int row_bytes = p.dim * L::ES, steps = (p.dim + 15) / 16, cols = min(DT, (p.dim + 31) / 32 - t0);
    const uint8_t *kp = at(p.k, s.batch, s.k0, kh), *vp = at(p.v, s.batch, s.k0, kh);
    uint8_t *const kt = lds + wave * 2 * TILE, *const vt = kt + TILE;
    const Share<ST, DP, kRows, 64> share{lane};
    auto load = [&](uint8_t* to, const uint8_t* from, int64_t stride, int t) __attribute__((always_inline)) {
        share.template stage<DMA>(to, from + t * (kRows * stride), row_bytes, false, [&](int i) { return share.row(i) * stride; },
                                  [&](int i) { return t * kRows + share.row(i) < s.nk; });
    };
    if (wave < tiles) {
        load(kt, kp, p.k.ss, wave);
        load(vt, vp, p.v.ss, wave);
    }
#pragma unroll 1
    for (int t = wave; t < tiles; t += W) {
        wave_wait<0>();
        const bool cut = (t + 1) * kRows > n_all;
        const int left = n_lane - t * kRows - 4 * h;
        f32x16 x, y;
        Frag<ST> ds[2];
        row_product_of<ST, DP>(steps, x, kt, q, lane);
        row_product_of<ST, DP>(steps, y, vt, g, lane);
        wave_wait<-1>();
        if (t + W < tiles) load(vt, vp, p.v.ss, t + W);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float e = __builtin_amdgcn_exp2f(fmaf(x[i], c, -lse)) * (y[i] - d);
            y[i] = cut && result_row(i, 0) >= left ? 0.f : e;
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) ds[u] = as_operand<ST>(y, u);
        col_product<ST, DP>(dq[0], kt, ds, t0, cols, lane);
        wave_wait<-1>();
        if (t + W < tiles) load(kt, kp, p.k.ss, t + W);
    }
    const float mul[1] = {p.scale};
    join_waves<ST, W, DT, 1>(lds, dq, mul, min(kRows, rows - r0), p.dim - 32 * t0, [&](int, int row) {
        const int token = (int)((uint32_t)(r0 + row) / (uint32_t)G);
        return at(p.dq, s.batch, s.q0 + token, kh * G + r0 + row - token * G) + 32 * t0 * L::ES;
    }, [&](int row) { return seen(r0 + row) > 0; });
}

// Block `id` of `n` of keys. lds: of each wave rows of q and of g, then [waves] sums.
template <GemmStore ST, int DP, bool DMA> HM_DEV void grad_kv_shared(const AttnArgs& p, uint8_t* lds, float* stats_lds, uint32_t id, uint32_t n_blocks)
{
    using L = Lay<ST, DP>;
    constexpr int W = shared_waves<ST, DP>(), TILE = kRows * L::PITCH, PARTS = kv_parts<ST, DP>(), DT = L::DT / PARTS;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x) >> 6, h = lane >> 5;
    const int G = p.group;

    const Item item = find_item<PARTS, false>(p, id, n_blocks);
    const int kh = item.kh, t0 = item.part * DT;
    const Seq s = find_seq<true, kRows>(p, item.item, 1);
    const int j0 = s.tile * kRows;
    if (j0 >= s.k_cap) return;
    const int key = j0 + (lane & 31);
    const bool on = key < s.nk;
    Frag<ST> k[L::NS], v[L::NS];
    load_row<DMA, ST, DP>(k, at(p.k, s.batch, s.k0 + key, kh), on, p.dim, h);
    load_row<DMA, ST, DP>(v, at(p.v, s.batch, s.k0 + key, kh), on, p.dim, h);

    // rows that see keys of the block, all of them, and this lane's
    const int off = s.nk - s.nq;
    auto first_row = [&](int j) { return p.causal ? max(0, j - off) * G : 0; };
    // (keys behind those in use have none, and their rows no place in 32 bits)
    const int end = j0 < s.nk ? s.nq * G : 0, begin = j0 < s.nk ? first_row(j0) / kRows * kRows : 0;
    const int all = j0 + kRows <= s.nk ? first_row(j0 + kRows - 1) : INT32_MAX, mine = on ? first_row(key) : INT32_MAX;
    const int tiles = end > begin ? (end - begin + kRows - 1) / kRows : 0;

    f32x16 acc[2][DT];  // dk, dv
#pragma unroll
    for (int t = 0; t < DT; ++t) acc[0][t] = acc[1][t] = f32x16{};
    const float c = p.scale * kLog2e;
    const int row_bytes = p.dim * L::ES, steps = (p.dim + 15) / 16, cols = min(DT, (p.dim + 31) / 32 - t0);
    const uint8_t *const qp = at(p.q, s.batch, s.q0, kh * G), *const gp = at(p.g, s.batch, s.q0, kh * G);
    uint8_t *const qt = lds + wave * 2 * TILE, *const gt = qt + TILE;
    float* const st = stats_lds + wave * 2 * kRows;  // a tile's lse, then its D
    const float2* const stats = p.stats + stat_row(p, s, kh, 0);
    const Share<ST, DP, kRows, 64> share{lane};
    const uint32_t over_g = (65535u + (uint32_t)G) / (uint32_t)G;
    auto load = [&](uint8_t* to, const uint8_t* from, const Heads& x, int t) __attribute__((always_inline)) {
        // A row lies less than G + 32 behind its tile's first token: the tokens in between without a
        // division (below 32 times 2^16 / G, rounded up, is exact to 2^16).
        const int r0 = begin + t * kRows, token0 = (int)((uint32_t)r0 / (uint32_t)G), place0 = r0 - token0 * G;
        share.template stage<DMA>(to, from + token0 * x.ss, row_bytes, false, [&](int i) {
            const int place = place0 + share.row(i);
            const int tokens = G < kRows ? (int)((uint32_t)place * over_g >> 16) : place >= G;
            return tokens * x.ss + (int64_t)(place - tokens * G) * x.sh;
        }, [&](int i) { return r0 + share.row(i) < end; });
    };
    if (wave < tiles) {
        load(qt, qp, p.q, wave);
        load(gt, gp, p.g, wave);
    }
#pragma unroll 1
    for (int t = wave; t < tiles; t += W) {
        const int r0 = begin + t * kRows;
        const float2 mine_st = r0 + (lane & 31) < end ? stats[r0 + (lane & 31)] : float2{INFINITY, 0.f};
        wave_wait<0>();
        st[lane] = h ? mine_st.y : mine_st.x;
        f32x16 x, y;
        Frag<ST> pr[2], ds[2];
        row_product_of<ST, DP>(steps, x, qt, k, lane);
        row_product_of<ST, DP>(steps, y, gt, v, lane);
        wave_wait<-1>();
        const int hidden = r0 < all ? min(mine - r0, kRows) - 4 * h : INT32_MIN;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float lse = st[result_row(i, h)], d = st[kRows + result_row(i, h)];
            x[i] = result_row(i, 0) < hidden ? 0.f : __builtin_amdgcn_exp2f(fmaf(x[i], c, -lse));
            y[i] = result_row(i, 0) < hidden ? 0.f : x[i] * (y[i] - d);
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) pr[u] = as_operand<ST>(x, u);
        col_product<ST, DP>(acc[1], gt, pr, t0, cols, lane);
        wave_wait<-1>();
        if (t + W < tiles) load(gt, gp, p.g, t + W);
#pragma unroll
        for (int u = 0; u < 2; ++u) ds[u] = as_operand<ST>(y, u);
        col_product<ST, DP>(acc[0], qt, ds, t0, cols, lane);
        wave_wait<-1>();
        if (t + W < tiles) load(qt, qp, p.q, t + W);
    }
    const float mul[2] = {p.scale, 1.f};
    join_waves<ST, W, DT, 2>(lds, acc, mul, min(kRows, s.k_cap - j0), p.dim - 32 * t0, [&](int n, int row) {
        return at(n == 0 ? p.dk : p.dv, s.batch, s.k0 + j0 + row, kh) + 32 * t0 * L::ES;
    }, [&](int row) { return j0 + row < s.nk; });
}

// Both in one launch, keys first: a block of either has a CU to itself, and where blocks are few the
// queries' run on the CUs that the keys' leave. Every row's lse and D have to be there before.
template <GemmStore ST, int DP, bool DMA> __global__ void __launch_bounds__((64 * shared_waves<ST, DP>())) attn_grad_shared(const AttnArgs p)
{
    constexpr int W = shared_waves<ST, DP>(), TILE = kRows * Lay<ST, DP>::PITCH, DT = Lay<ST, DP>::DT;
    constexpr int Q = shared_lds<W, TILE, DT / q_parts<ST, DP>()>(), KV = shared_lds<W, TILE, DT / kv_parts<ST, DP>()>();
    __shared__ __attribute__((aligned(16))) uint8_t lds[std::max(Q, KV)];
    __shared__ __attribute__((aligned(16))) float stats[W * 2 * kRows];
    const uint32_t of_keys = (uint32_t)p.k_blocks;
    if (blockIdx.x < of_keys) {
        AttnArgs k = p;
        k.slots = p.k_slots;
        grad_kv_shared<ST, DP, DMA>(k, lds, stats, blockIdx.x, of_keys);
    } else {
        grad_q_shared<ST, DP, DMA>(p, lds, blockIdx.x - of_keys, gridDim.x - of_keys);
    }
}

// lse and D of every row.
template <GemmStore ST, int DP, bool DMA> __global__ void __launch_bounds__(kThreads) attn_grad_rows(const AttnArgs p)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x) >> 6, h = lane >> 5, G = p.group;
    const Item item = find_item<1, true>(p, blockIdx.x, gridDim.x);
    const Seq s = find_seq<false, kTileRows>(p, item.item, G);
    const int r = s.tile * kTileRows + wave * kRows + (lane & 31);
    const int query = (int)((uint32_t)r / (uint32_t)G), head = item.kh * G + (int)((uint32_t)r - (uint32_t)query * (uint32_t)G);
    const bool exists = r < s.q_cap * G, on = exists && query < s.nq && visible(p, s, query) > 0;
    Frag<ST> g[DP / 16];
    load_row<DMA, ST, DP>(g, at(p.g, s.batch, s.q0 + query, head), on, p.dim, h);
    const float d = row_dot<DMA, ST, DP>(g, at(p.o, s.batch, s.q0 + query, head), on, p.dim, h);
    if (!exists || h != 0) return;
    const float lse = on ? p.lse[((int64_t)s.batch * p.q_len + s.q0 + query) * ((int64_t)p.hk * G) + head] * kLog2e : INFINITY;
    p.stats[stat_row(p, s, item.kh, r)] = float2{lse, d};
}

// ---------------------------------------------------------------- host side

template <GemmStore ST, bool DMA, int DP> int launch_grad(AttnArgs p, hipStream_t stream)
{
    int64_t q_blocks = 0, k_blocks = 0;
    AttnArgs pk = p;
    // Blocks of four waves with 32 rows each, or with 32 rows that they share.
    if (!set_grid<false>(p, kTileRows, kThreads * q_parts<ST, DP>(), &q_blocks) ||
        !set_grid<true>(pk, kTileRows, kThreads * kv_parts<ST, DP>(), &k_blocks))
        return HIMUON_ERR_UNSUPPORTED;
    constexpr int T = 64 * shared_waves<ST, DP>();
    const GradPlan plan = plan_grad(ST == GemmStore::F32, p.q_len > 0 ? q_blocks : 0, p.k_len > 0 ? k_blocks : 0);
    const bool k_shared = plan.k_shared, q_shared = plan.q_shared;
    AttnArgs ps = p;
    int64_t qs_blocks = 0, ks_blocks = 0;
    if ((q_shared && !set_grid<false>(ps, kRows, T * q_parts<ST, DP>(), &qs_blocks)) ||
        (k_shared && !set_grid<true>(pk, kRows, T * kv_parts<ST, DP>(), &ks_blocks)))
        return HIMUON_ERR_UNSUPPORTED;
    ps.k_slots = pk.slots;
    ps.k_blocks = (int32_t)(ks_blocks * kv_parts<ST, DP>());
    const int64_t blocks = qs_blocks * q_parts<ST, DP>() + ps.k_blocks;
    if (blocks > 0 && !launchable(blocks, T)) return HIMUON_ERR_UNSUPPORTED;
    if ((p.dq.ptr && (p.dq.ptr == p.dk.ptr || p.dq.ptr == p.dv.ptr)) || (p.dk.ptr && p.dk.ptr == p.dv.ptr)) return HIMUON_ERR_INVALID_ARG;
    StreamDevice on(stream);
    if (on.status != HIMUON_OK) return on.status;
    if (q_shared) hipLaunchKernelGGL((attn_grad_rows<ST, DP, DMA>), dim3((unsigned)q_blocks), dim3(kThreads), 0, stream, p);
    else if (p.q_len > 0)
        hipLaunchKernelGGL((attn_grad_q<ST, DP, DMA>), dim3((unsigned)(q_blocks * q_parts<ST, DP>())), dim3(kThreads), 0, stream, p);
    if (blocks > 0) hipLaunchKernelGGL((attn_grad_shared<ST, DP, DMA>), dim3((unsigned)blocks), dim3(T), 0, stream, ps);
    if (p.k_len > 0 && !k_shared)
        hipLaunchKernelGGL((attn_grad_kv<ST, DP, DMA>), dim3((unsigned)(k_blocks * kv_parts<ST, DP>())), dim3(kThreads), 0, stream, pk);
    return launch_status();
}

template <GemmStore ST, bool DMA> int launch_dim(const AttnArgs& p, hipStream_t stream)
{
    if (p.dim <= 64) return launch_grad<ST, DMA, 64>(p, stream);
    if (p.dim <= 128) return launch_grad<ST, DMA, 128>(p, stream);
    return launch_grad<ST, DMA, 256>(p, stream);
}

}  // namespace
}  // namespace attn
}  // namespace himuon

extern "C" size_t himuon_attention_grad_workspace_size(const himuon_attn_t* args)
{
    using namespace himuon;
    if (attn::check_attn(args) != HIMUON_OK) return 0;
    const int64_t tokens = args->q_starts ? args->q_len : args->batch * args->q_len;
    return round_up((size_t)(tokens * args->q_heads) * sizeof(float2), 256);
}

extern "C" int himuon_attention_grad(const himuon_attn_t* args, const himuon_heads_t* g, const himuon_heads_t* q, const himuon_heads_t* k,
                                     const himuon_heads_t* v, const himuon_heads_t* out, const float* lse, const himuon_heads_t* dq,
                                     const himuon_heads_t* dk, const himuon_heads_t* dv, void* workspace, size_t workspace_bytes,
                                     void* stream)
{
    using namespace himuon;
    using namespace himuon::attn;
    const int st = check_attn(args);
    if (st != HIMUON_OK) return st;
    if (empty_batch(args) || (args->q_len == 0 && args->k_len == 0)) return HIMUON_OK;
    AttnArgs p = attn_args(args);
    bool dma = true;
    const int64_t nq = args->q_len, nk = args->k_len;
    if (!set_heads(p.g, g, args, nq, args->q_heads, false, &dma) || !set_heads(p.q, q, args, nq, args->q_heads, false, &dma) ||
        !set_heads(p.k, k, args, nk, args->k_heads, false, &dma) || !set_heads(p.v, v, args, nk, args->k_heads, false, &dma) ||
        !set_heads(p.o, out, args, nq, args->q_heads, false, &dma) || !set_heads(p.dq, dq, args, nq, args->q_heads, true, &dma) ||
        !set_heads(p.dk, dk, args, nk, args->k_heads, true, &dma) || !set_heads(p.dv, dv, args, nk, args->k_heads, true, &dma) ||
        (nq > 0 && !lse))
        return HIMUON_ERR_INVALID_ARG;
    for (const Heads* o : {&p.dq, &p.dk, &p.dv})
        for (const Heads* i : {&p.g, &p.q, &p.k, &p.v, &p.o})
            if (o->ptr && o->ptr == i->ptr) return HIMUON_ERR_INVALID_ARG;
    p.lse = const_cast<float*>(lse);
    const size_t need = himuon_attention_grad_workspace_size(args);
    if (need > 0 && (!workspace || ((uintptr_t)workspace & 15) || workspace_bytes < need)) return HIMUON_ERR_WORKSPACE;
    p.stats = static_cast<float2*>(workspace);
    const hipStream_t hs = static_cast<hipStream_t>(stream);
    if (args->dtype == HIMUON_BF16) return dma ? launch_dim<GemmStore::BF16, true>(p, hs) : launch_dim<GemmStore::BF16, false>(p, hs);
    return dma ? launch_dim<GemmStore::F32, true>(p, hs) : launch_dim<GemmStore::F32, false>(p, hs);
}
