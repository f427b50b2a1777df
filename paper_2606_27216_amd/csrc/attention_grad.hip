// The backward pass of attention (himuon_attention_grad).
//
//     p = exp(c q k^T - lse),  D = rowsum(g o),  ds = p (g v^T - D)
//     dv = p^T g,  dk = c ds^T q,  dq = c ds k
// from the forward pass's inputs, o and lse. Two kernels: one whose waves hold 32 rows of queries
// and walk over the keys (dq; it also leaves every row's lse and D behind for the other one), and
// one whose waves hold 32 keys and walk over the rows of the head's whole group (dk, dv). Scores
// are computed in both: seven products instead of five, but no sum is shared between blocks, so
// that results have one order of summation and there are no atomics. As in the forward pass p and
// ds are a product's second operand as they stand.
#include "attn_device.h"

#include <algorithm>
#include <cmath>

namespace himuon {
namespace attn {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64, kTileRows = kRows * kWaves;

// Keys of a tile that all waves read.
template <GemmStore ST, int DP> constexpr int tile_keys() { return DP * (ST == GemmStore::BF16 ? 2 : 4) <= 256 ? 64 : 32; }

// Row of a group's heads in `stats`.
HM_DEV int64_t stat_row(const AttnArgs& p, const Seq& s, int kh, int64_t r)
{
    const int64_t tokens = p.packed ? p.q_len : p.q_len * p.batch;
    return ((int64_t)kh * tokens + (int64_t)s.batch * p.q_len + s.q0) * p.group + r;
}

// Columns of a result are cut into this many parts, each a block's, where registers hold no more.
template <GemmStore ST, int DP> constexpr int q_parts() { return ST == GemmStore::F32 && DP == 256 ? 4 : 1; }
template <GemmStore ST, int DP> constexpr int kv_parts() { return DP < 256 ? 1 : ST == GemmStore::F32 ? 4 : 2; }

template <GemmStore ST, int DP, bool DMA> __global__ void __launch_bounds__(kThreads) attn_grad_q(const AttnArgs p)
{
    using L = Lay<ST, DP>;
    constexpr int BN = tile_keys<ST, DP>(), TILE = BN * L::PITCH, PARTS = q_parts<ST, DP>(), DT = L::DT / PARTS;
    __shared__ __attribute__((aligned(16))) uint8_t lds[4 * TILE];  // [2][keys, values]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x) >> 6, h = lane >> 5;
    const int G = p.group;

    int64_t w = xcd_order(blockIdx.x, gridDim.x);
    const int t0 = PARTS == 1 ? 0 : (int)(w % PARTS) * DT;  // the first of this block's tiles of 32 columns
    w /= PARTS;
    const int64_t items = p.packed ? p.slots : (int64_t)p.slots * p.batch;
    const int kh = (int)(w / items);
    const int64_t at_item = w - kh * items;
    const int64_t tile = p.packed ? items - 1 - at_item : at_item / p.slots * p.slots + (p.slots - 1 - at_item % p.slots);
    const Seq s = find_seq<false, kTileRows>(p, tile, G);
    const int64_t rows = (int64_t)s.q_cap * G, r0 = (int64_t)s.tile * kTileRows;
    if (r0 >= rows) return;

    const int64_t r = r0 + wave * kRows + (lane & 31);
    const int query = (int)((uint32_t)r / (uint32_t)G);
    const int head = kh * G + (int)((uint32_t)r - (uint32_t)query * (uint32_t)G);
    const bool exists = r < rows;
    const int n_lane = query < s.nq ? visible(p, s, query) : 0;
    const bool on = n_lane > 0;  // (a row that sees nothing has no gradient)
    Frag<ST> q[L::NS], g[L::NS];
    load_row<ST, DP>(q, at(p.q, s.batch, s.q0 + query, head), on, p.dim, h);
    load_row<ST, DP>(g, at(p.g, s.batch, s.q0 + query, head), on, p.dim, h);
    float d = 0.f;
    const uint8_t* const o_row = at(p.o, s.batch, s.q0 + query, head);
#pragma unroll
    for (int i = 0; i < L::NS; i += 4) {
        Frag<ST> o[4];
        load_row<ST, 64>(o, o_row + 16 * i * L::ES, on, p.dim - 16 * i, h);
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) d = fmaf(frag_value<ST>(g[i + j], e), frag_value<ST>(o[j], e), d);
        __builtin_amdgcn_sched_barrier(0);
    }
    d = add_halves(d);
    const float c = p.scale * kLog2e;
    // (infinity: whatever the row's scores are, its p are zero)
    const float lse = on ? p.lse[((int64_t)s.batch * p.q_len + s.q0 + query) * ((int64_t)p.hk * G) + head] * kLog2e : INFINITY;
    if (exists && h == 0 && t0 == 0) p.stats[stat_row(p, s, kh, r)] = float2{lse, d};

    const int last = min((int)((r0 + kTileRows - 1) / G), s.nq - 1);
    const int n_block = s.nq > 0 && r0 < (int64_t)s.nq * G ? visible(p, s, last) : 0;
    const int64_t w0 = r0 + wave * kRows;
    const int n_wave = w0 < (int64_t)s.nq * G ? visible(p, s, min((int)((w0 + kRows - 1) / G), s.nq - 1)) : 0;
    const int n_all = visible(p, s, (int)(w0 / G));

    f32x16 dq[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t) dq[t] = f32x16{};
    const int row_bytes = p.dim * L::ES;
    const uint8_t *kp = at(p.k, s.batch, s.k0, kh), *vp = at(p.v, s.batch, s.k0, kh);
    const Share<ST, DP, BN, kThreads> share{(int)threadIdx.x};
    auto load = [&](int buf, int j0) __attribute__((always_inline)) {
        uint8_t* const t = lds + buf * 2 * TILE;
        const bool whole = j0 + BN <= s.nk;
        auto in = [&](int i) { return j0 + share.row(i) < s.nk; };
        share.template stage<DMA>(t, kp + j0 * p.k.ss, row_bytes, whole, [&](int i) { return share.row(i) * p.k.ss; }, in);
        share.template stage<DMA>(t + TILE, vp + j0 * p.v.ss, row_bytes, whole, [&](int i) { return share.row(i) * p.v.ss; }, in);
    };
    auto keys = [&](const uint8_t* kt, const uint8_t* vt, bool masked, int left) __attribute__((always_inline)) {
        f32x16 x{}, y{};
        ahead<L::NS>([&](int i) { return Pair<ST>{L::row_frag(kt, lane & 31, i, h), L::row_frag(vt, lane & 31, i, h)}; },
                     [&](int i, const Pair<ST>& f) {
                         mma<ST>(x, f.a, q[i]);
                         mma<ST>(y, f.b, g[i]);
                     });
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float pr = __builtin_amdgcn_exp2f(fmaf(x[i], c, -lse));
            y[i] = pr * (y[i] - d);
        }
        if (masked) {
#pragma unroll
            for (int i = 0; i < 16; ++i) y[i] = result_row(i, h) < left ? y[i] : 0.f;
        }
        const Frag<ST> ds[2] = {as_operand<ST>(y, 0), as_operand<ST>(y, 1)};
        ahead<2 * DT>([&](int i) { return L::col_frag(kt, 16 * (i / DT), 32 * (t0 + i % DT), lane); },
                      [&](int i, const Frag<ST>& a) { mma<ST>(dq[i % DT], a, ds[i / DT]); });
    };
    if (n_block > 0) {
        if (DMA && p.dim < DP) {
            clear_lds<kThreads>(lds, 4 * TILE);
            __syncthreads();
        }
        load(0, 0);
        int buf = 0;
        for (int j0 = 0; j0 < n_block; j0 += BN, buf ^= 1) {
            dev::dma_wait_barrier<0>();
            if (j0 + BN < n_block) load(buf ^ 1, j0 + BN);
            const uint8_t* const t = lds + buf * 2 * TILE;
#pragma unroll 1
            for (int j = 0; j < BN; j += kRows) {
                if (j0 + j >= n_wave) break;
                const uint8_t* const kt = t + j * L::PITCH;
                keys(kt, kt + TILE, j0 + j + kRows > n_all, n_lane - j0 - j);
            }
        }
    }
    if (!exists) return;
    store_row<DMA, ST>(at(p.dq, s.batch, s.q0 + query, head) + 32 * t0 * L::ES, dq, on, p.scale, p.dim - 32 * t0, h);
}

template <GemmStore ST, int DP, bool DMA> __global__ void __launch_bounds__(kThreads) attn_grad_kv(const AttnArgs p)
{
    using L = Lay<ST, DP>;
    constexpr int BR = kRows, TILE = BR * L::PITCH, PARTS = kv_parts<ST, DP>(), DT = L::DT / PARTS, BUF = 2 * TILE + BR * 8;
    __shared__ __attribute__((aligned(16))) uint8_t lds[2 * BUF];  // [2][rows of q, of g, {lse, D}]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x) >> 6, h = lane >> 5;
    const int G = p.group;

    int64_t w = xcd_order(blockIdx.x, gridDim.x);
    const int t0 = PARTS == 1 ? 0 : (int)(w % PARTS) * DT;
    w /= PARTS;
    const int64_t items = p.packed ? p.slots : (int64_t)p.slots * p.batch;
    const int kh = (int)(w / items);
    const Seq s = find_seq<true, kTileRows>(p, w - kh * items, 1);
    const int j0 = s.tile * kTileRows;  // (a sequence's first keys, which most queries see, first)
    if (j0 >= s.k_cap) return;
    const int key = j0 + wave * kRows + (lane & 31);
    const bool exists = key < s.k_cap, on = key < s.nk;
    Frag<ST> k[L::NS], v[L::NS];
    load_row<ST, DP>(k, at(p.k, s.batch, s.k0 + key, kh), on, p.dim, h);
    load_row<ST, DP>(v, at(p.v, s.batch, s.k0 + key, kh), on, p.dim, h);

    // rows that see keys of the block, of the wave, this lane's and all of the wave's
    const int off = s.nk - s.nq;
    auto first_row = [&](int j) { return p.causal ? (int64_t)max(0, j - off) * G : (int64_t)0; };
    const int64_t end = j0 < s.nk ? (int64_t)s.nq * G : 0;
    const int64_t begin = first_row(j0) / BR * BR, w_begin = first_row(j0 + wave * kRows);
    const int64_t w_all = first_row(j0 + wave * kRows + kRows - 1), mine = on ? first_row(key) : INT64_MAX;
    const bool w_on = j0 + wave * kRows < s.nk, w_whole = j0 + wave * kRows + kRows <= s.nk;

    f32x16 dk[DT], dv[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t) dk[t] = dv[t] = f32x16{};
    const float c = p.scale * kLog2e;
    const int row_bytes = p.dim * L::ES;
    const Share<ST, DP, BR, kThreads> share{(int)threadIdx.x};
    const float2* const stats = p.stats + stat_row(p, s, kh, 0);
    auto load = [&](int buf, int64_t r0) __attribute__((always_inline)) {
        uint8_t* const t = lds + buf * BUF;
        const bool whole = r0 + BR <= end;
        const int q0 = (int)(r0 / G), g0 = (int)(r0 - (int64_t)q0 * G);
        const uint8_t *qp = at(p.q, s.batch, s.q0 + q0, kh * G), *gp = at(p.g, s.batch, s.q0 + q0, kh * G);
        auto in = [&](int i) { return r0 + share.row(i) < end; };
        auto place = [&](int i, const Heads& x) {
            const int r = g0 + share.row(i), dq = (int)((uint32_t)r / (uint32_t)G);
            return dq * x.ss + (r - dq * G) * x.sh;
        };
        share.template stage<DMA>(t, qp, row_bytes, whole, [&](int i) { return place(i, p.q); }, in);
        share.template stage<DMA>(t + TILE, gp, row_bytes, whole, [&](int i) { return place(i, p.g); }, in);
        if (whole) {
            if (wave == 0) dev::dma4((uint32_t)__builtin_amdgcn_readfirstlane((int)dev::lds_offset(t + 2 * TILE)), 4 * lane, dev::uniform_address(stats + r0));
        } else if (threadIdx.x < BR)
            reinterpret_cast<float2*>(t + 2 * TILE)[threadIdx.x] = r0 + threadIdx.x < end ? stats[r0 + threadIdx.x] : float2{INFINITY, 0.f};
    };
    auto rows = [&](const uint8_t* qt, const float2* st, int64_t r0, bool masked) __attribute__((always_inline)) {
        const uint8_t* const gt = qt + TILE;
        f32x16 x{}, y{};
        ahead<L::NS>([&](int i) { return Pair<ST>{L::row_frag(qt, lane & 31, i, h), L::row_frag(gt, lane & 31, i, h)}; },
                     [&](int i, const Pair<ST>& f) {
                         mma<ST>(x, f.a, k[i]);
                         mma<ST>(y, f.b, v[i]);
                     });
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float2 a = st[result_row(i, h)];
            x[i] = __builtin_amdgcn_exp2f(fmaf(x[i], c, -a.x));
            y[i] = x[i] * (y[i] - a.y);
        }
        if (masked) {
            const int hidden = (int)min(mine - r0, (int64_t)BR);  // rows that do not see this lane's key
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                x[i] = result_row(i, h) < hidden ? 0.f : x[i];
                y[i] = result_row(i, h) < hidden ? 0.f : y[i];
            }
        }
        const Frag<ST> pr[2] = {as_operand<ST>(x, 0), as_operand<ST>(x, 1)}, ds[2] = {as_operand<ST>(y, 0), as_operand<ST>(y, 1)};
        ahead<2 * DT>(
            [&](int i) {
                return Pair<ST>{L::col_frag(gt, 16 * (i / DT), 32 * (t0 + i % DT), lane), L::col_frag(qt, 16 * (i / DT), 32 * (t0 + i % DT), lane)};
            },
            [&](int i, const Pair<ST>& f) {
                mma<ST>(dv[i % DT], f.a, pr[i / DT]);
                mma<ST>(dk[i % DT], f.b, ds[i / DT]);
            });
    };
    if (begin < end) {
        if (DMA && p.dim < DP) {
            clear_lds<kThreads>(lds, 2 * BUF);
            __syncthreads();
        }
        load(0, begin);
        int buf = 0;
        for (int64_t r0 = begin; r0 < end; r0 += BR, buf ^= 1) {
            dev::dma_wait_barrier<0>();
            if (r0 + BR < end) load(buf ^ 1, r0 + BR);
            if (!w_on || r0 + BR <= w_begin) continue;
            const uint8_t* const t = lds + buf * BUF;
            const float2* const st = reinterpret_cast<const float2*>(t + 2 * TILE);
            rows(t, st, r0, r0 < w_all || !w_whole);
        }
    }
    if (!exists) return;
    const int dim = p.dim - 32 * t0;
    store_row<DMA, ST>(at(p.dk, s.batch, s.k0 + key, kh) + 32 * t0 * L::ES, dk, on, p.scale, dim, h);
    store_row<DMA, ST>(at(p.dv, s.batch, s.k0 + key, kh) + 32 * t0 * L::ES, dv, on, 1.f, dim, h);
}

// ---------------------------------------------------------------- host side

template <GemmStore ST, bool DMA, int DP> int launch_grad(AttnArgs p, hipStream_t stream)
{
    int64_t q_blocks = 0, k_blocks = 0;
    AttnArgs pk = p;
    if (!set_grid(p, p.q_len * p.group, kTileRows, kThreads * q_parts<ST, DP>(), &q_blocks) ||
        !set_grid(pk, pk.k_len, kTileRows, kThreads * kv_parts<ST, DP>(), &k_blocks))
        return HIMUON_ERR_UNSUPPORTED;
    StreamDevice on(stream);
    if (on.status != HIMUON_OK) return on.status;
    if (p.q_len > 0) hipLaunchKernelGGL((attn_grad_q<ST, DP, DMA>), dim3((unsigned)(q_blocks * q_parts<ST, DP>())), dim3(kThreads), 0, stream, p);
    if (p.k_len > 0)
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
    p.lse = const_cast<float*>(lse);
    const size_t need = himuon_attention_grad_workspace_size(args);
    if (need > 0 && (!workspace || ((uintptr_t)workspace & 15) || workspace_bytes < need)) return HIMUON_ERR_WORKSPACE;
    p.stats = static_cast<float2*>(workspace);
    const hipStream_t hs = static_cast<hipStream_t>(stream);
    if (args->dtype == HIMUON_BF16) return dma ? launch_dim<GemmStore::BF16, true>(p, hs) : launch_dim<GemmStore::BF16, false>(p, hs);
    return dma ? launch_dim<GemmStore::F32, true>(p, hs) : launch_dim<GemmStore::F32, false>(p, hs);
}
