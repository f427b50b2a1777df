// Attention over whole sequences (himuon_attention).
//
// For the queries of a sequence and the group of heads that share a key head:
//     s = c q k^T over the keys that a query sees,  o = softmax(s) v,  lse = log sum exp s
// in one pass over the keys with a running maximum m and sum l, o held unnormalised. The rows
// of a tile are (query, head of the group) pairs, so that a group's heads share the keys they
// read and short sequences fill their tiles. A wave holds 32 rows as columns of s^T = k q^T:
// a row's statistics are one lane's, and p^T is the second operand of o^T = v^T p^T as it
// stands.
#include "attn_device.h"

#include <algorithm>
#include <cmath>

namespace himuon {
namespace attn {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64, kTileRows = kRows * kWaves;

// Keys of a tile: two buffers of keys and values leave room for two blocks to a CU where rows are short.
template <GemmStore ST, int DP> constexpr int tile_keys() { return DP * (ST == GemmStore::BF16 ? 2 : 4) <= 256 ? 64 : 32; }

template <GemmStore ST, int DP> struct Running {
    using L = Lay<ST, DP>;
    f32x16 o[L::DT];
    float m, l;  // l: of this half's keys

    HM_DEV void clear()
    {
#pragma unroll
        for (int t = 0; t < L::DT; ++t) o[t] = f32x16{};
        m = -INFINITY;
        l = 0.f;
    }

    // KT tiles of 32 keys at `kt`, `vt`; `masked` (the same in all lanes): this lane's row sees the first `left` of them.
    template <int KT> HM_DEV void keys(const uint8_t* kt, const uint8_t* vt, const Frag<ST> (&q)[L::NS], float c, bool masked, int left, int lane)
    {
        const int h = lane >> 5;
        f32x16 s[KT];
#pragma unroll
        for (int k = 0; k < KT; ++k) s[k] = f32x16{};
        ahead<KT * L::NS>([&](int i) { return L::row_frag(kt, 32 * (i / L::NS) + (lane & 31), i % L::NS, h); },
                          [&](int i, const Frag<ST>& a) { mma<ST>(s[i / L::NS], a, q[i % L::NS]); });
        if (masked) {
#pragma unroll
            for (int k = 0; k < KT; ++k)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[k][i] = 32 * k + result_row(i, h) < left ? s[k][i] : -INFINITY;
        }
        float top = s[0][0];
#pragma unroll
        for (int k = 0; k < KT; ++k)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, s[k][i]);
        top = max_halves(top);
        // The maximum follows once it is left behind by 2^8: any value near it serves, and most
        // tiles then leave o as it is.
        if (__any(top * c > m * c + 8.f)) {
            const float now = fmaxf(m, top);
            const float f = now == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m - now) * c);
            m = now;
            l *= f;
#pragma unroll
            for (int t = 0; t < L::DT; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[t][i] *= f;
        }
        const float mc = m == -INFINITY ? 0.f : m * c;
        float sum[2] = {};
#pragma unroll
        for (int k = 0; k < KT; ++k)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                s[k][i] = __builtin_amdgcn_exp2f(fmaf(s[k][i], c, -mc));
                sum[i & 1] += s[k][i];
            }
        l += sum[0] + sum[1];
        Frag<ST> pr[2 * KT];
#pragma unroll
        for (int k = 0; k < 2 * KT; ++k) pr[k] = as_operand<ST>(s[k / 2], k % 2);
        ahead<2 * KT * L::DT>([&](int i) { return L::col_frag(vt, 16 * (i / L::DT), 32 * (i % L::DT), lane); },
                              [&](int i, const Frag<ST>& a) { mma<ST>(o[i % L::DT], a, pr[i / L::DT]); });
    }
};

template <GemmStore ST, int DP, bool DMA> __global__ void __launch_bounds__(kThreads, (DP * (ST == GemmStore::BF16 ? 2 : 4) <= 256 ? 2 : 1)) attn_forward(const AttnArgs p)
{
    using L = Lay<ST, DP>;
    constexpr int BN = tile_keys<ST, DP>(), TILE = BN * L::PITCH;
    __shared__ __attribute__((aligned(16))) uint8_t lds[4 * TILE];  // [2][keys, values]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x) >> 6, h = lane >> 5;
    const int G = p.group;

    const int64_t w = xcd_order(blockIdx.x, gridDim.x);
    const int64_t items = p.packed ? p.slots : (int64_t)p.slots * p.batch;  // of a key head
    const int kh = (int)(w / items);
    const int64_t at_item = w - kh * items;
    // (a sequence's last tiles, which see the most keys, first)
    const int64_t tile = p.packed ? items - 1 - at_item : at_item / p.slots * p.slots + (p.slots - 1 - at_item % p.slots);
    const Seq s = find_seq<false, kTileRows>(p, tile, G);
    const int64_t rows = (int64_t)s.q_cap * G, r0 = (int64_t)s.tile * kTileRows;
    if (r0 >= rows) return;

    const int64_t r = r0 + wave * kRows + (lane & 31);
    const int query = (int)((uint32_t)r / (uint32_t)G);
    const int head = kh * G + (int)((uint32_t)r - (uint32_t)query * (uint32_t)G);
    const bool exists = r < rows, on = query < s.nq;
    Frag<ST> q[L::NS];
    load_row<ST, DP>(q, at(p.q, s.batch, s.q0 + query, head), on, p.dim, h);

    // keys that the block's, the wave's and the lane's rows see
    const int last = min((int)((r0 + kTileRows - 1) / G), s.nq - 1);
    const int n_block = s.nq > 0 && r0 < (int64_t)s.nq * G ? visible(p, s, last) : 0;
    const int64_t w0 = r0 + wave * kRows;
    const int n_wave = w0 < (int64_t)s.nq * G ? visible(p, s, min((int)((w0 + kRows - 1) / G), s.nq - 1)) : 0;
    const int n_all = visible(p, s, (int)(w0 / G));  // seen by all of the wave's rows
    const int n_lane = on ? visible(p, s, query) : 0;

    Running<ST, DP> run;
    run.clear();
    const float c = p.scale * kLog2e;
    const int row_bytes = p.dim * L::ES;
    const uint8_t *kp = at(p.k, s.batch, s.k0, kh), *vp = at(p.v, s.batch, s.k0, kh);
    const Share<ST, DP, BN, kThreads> share{(int)threadIdx.x};
    auto load = [&](int buf, int j0) __attribute__((always_inline)) {
        uint8_t* const t = lds + buf * 2 * TILE;
        const bool whole = j0 + BN <= s.nk;
        auto on = [&](int i) { return j0 + share.row(i) < s.nk; };
        share.template stage<DMA>(t, kp + j0 * p.k.ss, row_bytes, whole, [&](int i) { return share.row(i) * p.k.ss; }, on);
        share.template stage<DMA>(t + TILE, vp + j0 * p.v.ss, row_bytes, whole, [&](int i) { return share.row(i) * p.v.ss; }, on);
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
            if (j0 >= n_wave) continue;
            const uint8_t* const t = lds + buf * 2 * TILE;
            run.template keys<BN / 32>(t, t + TILE, q, c, j0 + BN > n_all, n_lane - j0, lane);
        }
    }
    if (!exists) return;
    const float l = add_halves(run.l);
    store_row<DMA, ST>(at(p.o, s.batch, s.q0 + query, head), run.o, on && l != 0.f, 1.f / l, p.dim, h);
    if (h == 0)
        p.lse[((int64_t)s.batch * p.q_len + s.q0 + query) * ((int64_t)p.hk * G) + head] =
            !on || l == 0.f ? -INFINITY : fmaf(run.m, p.scale, __logf(l));
}

// Few rows in all (a token or some of each sequence against many keys): a tile's 32 rows are
// all that a group of heads has, and the keys are shared out over the waves of a block and over
// `splits` blocks. Each wave keeps two tiles of 32 keys of its own on the way, without a
// barrier; the waves' results meet in LDS, the blocks' in `part`: [splits] rows of DP sums and
// of {m, l}.
constexpr int kFewLds = 128 << 10;
template <GemmStore ST, int DP> constexpr int few_waves() { return std::min(4, kFewLds / (4 * kRows * Lay<ST, DP>::PITCH)); }
template <GemmStore ST, int DP> constexpr int few_lds()
{
    return few_waves<ST, DP>() * kRows * std::max(4 * Lay<ST, DP>::PITCH, (DP + 4) * 4);
}
constexpr int kStat = 4;  // floats behind a row of partial sums

template <GemmStore ST, int DP, bool DMA> __global__ void __launch_bounds__((64 * few_waves<ST, DP>())) attn_few(const AttnArgs p)
{
    using L = Lay<ST, DP>;
    constexpr int W = few_waves<ST, DP>(), TILE = kRows * L::PITCH, DS = DP + kStat;
    __shared__ __attribute__((aligned(16))) uint8_t lds[few_lds<ST, DP>()];  // of each wave: [2][keys, values]; then [waves][32][DS] floats
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x) >> 6, h = lane >> 5;
    const int G = p.group, split = (int)(blockIdx.x % (uint32_t)p.splits);
    const int64_t w = blockIdx.x / (uint32_t)p.splits;
    const int kh = (int)(w % (uint32_t)p.hk);
    const Seq s = find_seq<false, kRows>(p, w / (uint32_t)p.hk, G);  // (one tile to a sequence)
    const int rows = s.q_cap * G;
    const int query = (lane & 31) / G, head = kh * G + (lane & 31) - query * G;
    const bool exists = (lane & 31) < rows, on = query < s.nq;
    Frag<ST> q[L::NS];
    load_row<ST, DP>(q, at(p.q, s.batch, s.q0 + query, head), on && exists, p.dim, h);

    const int n = s.nq > 0 ? visible(p, s, s.nq - 1) : 0, n_all = visible(p, s, 0), n_lane = on && exists ? visible(p, s, query) : 0;
    const int tiles = (n + kRows - 1) / kRows, turns = (tiles + p.splits * W - 1) / (p.splits * W);
    const int first = (split * W + wave) * turns, end = min(tiles, first + turns);
    Running<ST, DP> run;
    run.clear();
    const float c = p.scale * kLog2e;
    const int row_bytes = p.dim * L::ES;
    const uint8_t *kp = at(p.k, s.batch, s.k0, kh), *vp = at(p.v, s.batch, s.k0, kh);
    uint8_t* const mine = lds + wave * 4 * TILE;
    const Share<ST, DP, kRows, 64> share{lane};
    auto load = [&](int buf, int t) __attribute__((always_inline)) {
        const int j0 = t * kRows;
        uint8_t* const to = mine + buf * 2 * TILE;
        const bool whole = j0 + kRows <= s.nk;
        auto in = [&](int i) { return j0 + share.row(i) < s.nk; };
        share.template stage<DMA>(to, kp + j0 * p.k.ss, row_bytes, whole, [&](int i) { return share.row(i) * p.k.ss; }, in);
        share.template stage<DMA>(to + TILE, vp + j0 * p.v.ss, row_bytes, whole, [&](int i) { return share.row(i) * p.v.ss; }, in);
    };
    if (first < end) {
        if (DMA && p.dim < DP) {
            for (int i = 16 * lane; i < 4 * TILE; i += 16 * 64) *reinterpret_cast<u32x4*>(mine + i) = u32x4{};
            wave_wait<0>();
        }
        load(0, first);
        int buf = 0;
        for (int t = first; t < end; ++t, buf ^= 1) {
            // (the reads of the buffer that is filled next have returned; with the next tile on its
            // way, what is waited for is the one before)
            if (t + 1 < end) {
                wave_wait<-1>();
                load(buf ^ 1, t + 1);
                if ((t + 2) * kRows <= s.nk) wave_wait<2 * Share<ST, DP, kRows, 64>::NI>();
                else wave_wait<0>();
            } else {
                wave_wait<0>();
            }
            const uint8_t* const at_k = mine + buf * 2 * TILE;
            run.template keys<1>(at_k, at_k + TILE, q, c, (t + 1) * kRows > n_all, n_lane - t * kRows, lane);
        }
    }
    run.l = add_halves(run.l);
    __syncthreads();
    float* const sums = reinterpret_cast<float*>(lds);
    float* const own = sums + (wave * kRows + (lane & 31)) * DS;
#pragma unroll
    for (int t = 0; t < L::DT; ++t)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
            *reinterpret_cast<f32x4*>(own + 32 * t + result_row(i, h)) = f32x4{run.o[t][i], run.o[t][i + 1], run.o[t][i + 2], run.o[t][i + 3]};
    if (h == 0) {
        own[DP] = run.m;
        own[DP + 1] = run.l;
    }
    __syncthreads();
    constexpr int LR = 2 * W;  // lanes to a row
    const int row = threadIdx.x / LR, x = threadIdx.x % LR;
    if (row >= rows) return;
    float m = -INFINITY, l = 0.f, f[W];
#pragma unroll
    for (int v = 0; v < W; ++v) m = fmaxf(m, sums[(v * kRows + row) * DS + DP]);
#pragma unroll
    for (int v = 0; v < W; ++v) {
        const float* const from = sums + (v * kRows + row) * DS + DP;
        f[v] = from[0] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((from[0] - m) * c);
        l += from[0] == -INFINITY ? from[1] : f[v] * from[1];
    }
    const int token = row / G, hd = kh * G + row - token * G;
    const bool used = token < s.nq;
    float* const part = p.splits > 1 ? p.part + (((w * p.splits) + split) * kRows + row) * DS : nullptr;
    uint8_t* const out = at(p.o, s.batch, s.q0 + token, hd);
    const float mul = 1.f / l;
    const bool some = used && l != 0.f;
    for (int d = 4 * x; d < p.dim; d += 4 * LR) {
        f32x4 v = {};
#pragma unroll
        for (int u = 0; u < W; ++u) {
            const f32x4 a = *reinterpret_cast<const f32x4*>(sums + (u * kRows + row) * DS + d);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = fmaf(f[u], a[e], v[e]);
        }
        if (part) {
            *reinterpret_cast<f32x4*>(part + d) = v;
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (d + e < p.dim) put1<ST>(out, d + e, some ? v[e] * mul : 0.f);
        }
    }
    if (x == 0) {
        if (part) {
            part[DP] = m;
            part[DP + 1] = l;
        } else {
            p.lse[((int64_t)s.batch * p.q_len + s.q0 + token) * ((int64_t)p.hk * G) + hd] =
                !used || l == 0.f ? -INFINITY : fmaf(m, p.scale, __logf(l));
        }
    }
}

// The blocks' partial results of a row joined, in their order: a wave to a row.
template <GemmStore ST, int DP> __global__ void __launch_bounds__(kThreads) attn_join(const AttnArgs p)
{
    constexpr int DS = DP + kStat, E = DP / 64;
    const int lane = threadIdx.x & 63, G = p.group, rows = (int)p.q_len * G;
    const int64_t id = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6);
    const int64_t w = id / rows;
    const int row = (int)(id - w * rows), kh = (int)(w % (uint32_t)p.hk);
    if (w >= (int64_t)p.batch * p.hk) return;
    const Seq s = find_seq<false, kRows>(p, w / (uint32_t)p.hk, G);
    const float* const part = p.part + (w * p.splits * kRows + row) * DS;
    const float c = p.scale * kLog2e;
    float m = -INFINITY;
    for (int i = 0; i < p.splits; ++i) m = fmaxf(m, part[(int64_t)i * kRows * DS + DP]);
    float l = 0.f, v[E] = {};
    for (int i = 0; i < p.splits; ++i) {
        const float* const from = part + (int64_t)i * kRows * DS;
        const float mi = from[DP], f = mi == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((mi - m) * c);
        l += mi == -INFINITY ? from[DP + 1] : f * from[DP + 1];
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = fmaf(f, lane + 64 * e < p.dim ? from[lane + 64 * e] : 0.f, v[e]);
    }
    const int token = row / G, hd = kh * G + row - token * G;
    const bool used = token < s.nq;
    uint8_t* const out = at(p.o, s.batch, token, hd);
    const float mul = 1.f / l;
#pragma unroll
    for (int e = 0; e < E; ++e)
        if (lane + 64 * e < p.dim) put1<ST>(out, lane + 64 * e, used && l != 0.f ? v[e] * mul : 0.f);
    if (lane == 0)
        p.lse[((int64_t)s.batch * p.q_len + token) * ((int64_t)p.hk * G) + hd] = !used || l == 0.f ? -INFINITY : fmaf(m, p.scale, __logf(l));
}

// ---------------------------------------------------------------- host side

// Blocks that share the keys of a short call (one at a time on each CU: 256 of them).
template <class F> int by_dim(const AttnArgs& p, F f)
{
    if (p.dim <= 64) return f(std::integral_constant<int, 64>{});
    if (p.dim <= 128) return f(std::integral_constant<int, 128>{});
    return f(std::integral_constant<int, 256>{});
}

int padded_dim(int64_t dim) { return dim <= 64 ? 64 : dim <= 128 ? 128 : 256; }

bool few_rows(const himuon_attn_t* a) { return !a->q_starts && a->q_len * (a->q_heads / a->k_heads) <= kRows && a->k_len > 64; }

int64_t few_splits(const himuon_attn_t* a)
{
    const int64_t waves = std::min<int64_t>(4, kFewLds / (4 * kRows * padded_dim(a->head_dim) * dtype_size(a->dtype)));
    const int64_t most = ceil_div(a->k_len, kRows * waves * 2);  // two tiles to a wave
    return std::max<int64_t>(1, std::min<int64_t>(most, ceil_div(256, a->batch * a->k_heads)));
}

template <GemmStore ST, bool DMA> int launch_forward(AttnArgs p, bool few, hipStream_t stream)
{
    return by_dim(p, [&](auto dim) {
        constexpr int DP = decltype(dim)::value;
        if (few) {
            const int64_t blocks = (int64_t)p.batch * p.hk * p.splits;
            constexpr int T = 64 * few_waves<ST, DP>();
            if (!launchable(blocks, T)) return (int)HIMUON_ERR_UNSUPPORTED;
            StreamDevice on(stream);
            if (on.status != HIMUON_OK) return on.status;
            p.slots = 1;
            hipLaunchKernelGGL((attn_few<ST, DP, DMA>), dim3((unsigned)blocks), dim3(T), 0, stream, p);
            if (p.splits > 1) {
                const int64_t joins = ceil_div((int64_t)p.batch * p.hk * p.q_len * p.group, kWaves);
                hipLaunchKernelGGL((attn_join<ST, DP>), dim3((unsigned)joins), dim3(kThreads), 0, stream, p);
            }
            return launch_status();
        }
        int64_t blocks;
        if (!set_grid(p, p.q_len * p.group, kTileRows, kThreads, &blocks)) return (int)HIMUON_ERR_UNSUPPORTED;
        StreamDevice on(stream);
        if (on.status != HIMUON_OK) return on.status;
        hipLaunchKernelGGL((attn_forward<ST, DP, DMA>), dim3((unsigned)blocks), dim3(kThreads), 0, stream, p);
        return launch_status();
    });
}

}  // namespace

int check_attn(const himuon_attn_t* a)
{
    if (!a || a->batch < 0 || a->q_len < 0 || a->k_len < 0 || a->q_heads < 1 || a->k_heads < 1 || a->head_dim < 1)
        return HIMUON_ERR_INVALID_ARG;
    if (a->q_heads % a->k_heads || !known_dtype(a->dtype) || !known_index(a->index)) return HIMUON_ERR_INVALID_ARG;
    if (!(a->scale > 0.f) || !std::isfinite(a->scale) || !a->q_starts != !a->k_starts) return HIMUON_ERR_INVALID_ARG;
    if (a->head_dim > HIMUON_MAX_ATTN_DIM) return HIMUON_ERR_UNSUPPORTED;
    constexpr int64_t most = INT64_C(1) << 30;
    const int64_t group = a->q_heads / a->k_heads;
    if (a->batch > most || a->q_len > most / group || a->k_len > most) return HIMUON_ERR_UNSUPPORTED;
    // (rows of statistics; a batch's index)
    if (!small_product(a->batch * (a->q_starts ? 1 : a->q_len), a->q_heads * 8) || !small_product(a->batch, a->k_len))
        return HIMUON_ERR_UNSUPPORTED;
    return HIMUON_OK;
}

AttnArgs attn_args(const himuon_attn_t* a)
{
    AttnArgs p{};
    p.qs = a->q_starts;
    p.ks = a->k_starts;
    p.ql = a->q_lengths;
    p.kl = a->k_lengths;
    p.q_len = a->q_len;
    p.k_len = a->k_len;
    p.batch = (int32_t)a->batch;
    p.hk = a->k_heads;
    p.group = a->q_heads / a->k_heads;
    p.dim = a->head_dim;
    p.causal = a->causal != 0;
    p.wide = a->index == HIMUON_I64;
    p.packed = a->q_starts != nullptr;
    p.splits = 1;
    p.scale = a->scale;
    return p;
}

// Strides in bytes. `given`: whether there is an element at all; `dma`: cleared if rows are not
// 16-byte aligned, or a tile's rows lie too far apart for 32-bit offsets.
bool set_heads(Heads& t, const himuon_heads_t* h, const himuon_attn_t* a, int64_t tokens, int heads, bool output, bool* dma)
{
    t = Heads{};
    if (tokens == 0 || empty_batch(a)) return true;
    if (!h || !h->ptr) return false;
    const bool packed = a->q_starts != nullptr;
    if (output && ((!packed && a->batch > 1 && !h->stride_batch) || (tokens > 1 && !h->stride_seq) || (heads > 1 && !h->stride_head)))
        return false;
    const int64_t es = dtype_size(a->dtype);
    constexpr int64_t most = INT64_C(1) << 40;  // elements between neighbours
    for (const int64_t s : {h->stride_batch, h->stride_seq, h->stride_head})
        if (s > most || s < -most) return false;
    t.ptr = static_cast<uint8_t*>(h->ptr);
    t.sb = packed ? 0 : h->stride_batch * es;
    t.ss = h->stride_seq * es;
    t.sh = h->stride_head * es;
    const int64_t group = a->q_heads / a->k_heads;
    if (((uintptr_t)t.ptr | (uintptr_t)t.sb | (uintptr_t)t.ss | (uintptr_t)t.sh | (uintptr_t)(a->head_dim * es)) & 15) *dma = false;
    if (t.ss < 0 || t.sh < 0 || t.ss > INT64_C(1) << 24 || t.sh * group > INT64_C(1) << 31) *dma = false;
    return true;
}

bool set_grid(AttnArgs& p, int64_t rows, int tile, int threads, int64_t* blocks)
{
    const int64_t slots = p.packed ? rows / tile + p.batch + 2 : ceil_div(rows, tile);
    const int64_t items = p.packed ? slots : slots * p.batch;
    if (slots > INT32_MAX || !small_product(items, p.hk) || !launchable(items * p.hk, threads)) return false;
    p.slots = (int32_t)slots;
    *blocks = items * p.hk;
    return true;
}

}  // namespace attn
}  // namespace himuon

extern "C" size_t himuon_attention_workspace_size(const himuon_attn_t* args)
{
    using namespace himuon;
    using namespace himuon::attn;
    if (check_attn(args) != HIMUON_OK || empty_batch(args) || args->q_len == 0 || !few_rows(args)) return 0;
    const int64_t splits = few_splits(args);
    if (splits == 1) return 0;
    return (size_t)(args->batch * args->k_heads * splits) * kRows * (size_t)(padded_dim(args->head_dim) + kStat) * sizeof(float);
}

extern "C" int himuon_attention(const himuon_attn_t* args, const himuon_heads_t* q, const himuon_heads_t* k, const himuon_heads_t* v,
                                const himuon_heads_t* out, float* lse, void* workspace, size_t workspace_bytes, void* stream)
{
    using namespace himuon;
    using namespace himuon::attn;
    const int st = check_attn(args);
    if (st != HIMUON_OK) return st;
    if (empty_batch(args) || args->q_len == 0) return HIMUON_OK;
    AttnArgs p = attn_args(args);
    bool dma = true;
    if (!set_heads(p.q, q, args, args->q_len, args->q_heads, false, &dma) || !set_heads(p.k, k, args, args->k_len, args->k_heads, false, &dma) ||
        !set_heads(p.v, v, args, args->k_len, args->k_heads, false, &dma) || !set_heads(p.o, out, args, args->q_len, args->q_heads, true, &dma) || !lse)
        return HIMUON_ERR_INVALID_ARG;
    p.lse = lse;
    const bool few = few_rows(args);
    if (few) p.splits = (int32_t)few_splits(args);
    const size_t need = himuon_attention_workspace_size(args);
    if (need > 0 && (!workspace || ((uintptr_t)workspace & 15) || workspace_bytes < need)) return HIMUON_ERR_WORKSPACE;
    p.part = static_cast<float*>(workspace);
    const hipStream_t hs = static_cast<hipStream_t>(stream);
    if (args->dtype == HIMUON_BF16)
        return dma ? launch_forward<GemmStore::BF16, true>(p, few, hs) : launch_forward<GemmStore::BF16, false>(p, few, hs);
    return dma ? launch_forward<GemmStore::F32, true>(p, few, hs) : launch_forward<GemmStore::F32, false>(p, few, hs);
}
