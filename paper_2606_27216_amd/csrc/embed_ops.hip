// Token table lookup and its gradient (himuon_embed, himuon_embed_grad).
//
//     out[i, :] = scale E[t_i, :]          dE[v, :] = scale sum_{i: t_i = v} g[i, :]
//
// Both are bound by memory. The lookup is a gather: a row (or a part of one) per
// group of lanes, four 16-byte chunks in flight per lane.
//
// The gradient sorts the tokens (stable radix sort of (token, position), two or
// three digits, ranks by ballots within a wave), so that a row's terms are
// adjacent and its sum has one order. The sorted list is cut into chunks of S
// entries, whatever rows they name: a wave sums the runs of equal tokens of its
// chunk over 512 columns. Runs that lie inside a chunk go to the table at once; a run
// that crosses chunks leaves one fp32 partial sum per chunk, and a last launch
// adds these up in order. So a token that makes up much of a batch is spread over the
// chip like any other. Rows that no token names are set to zero beside the sums.
#include "elementwise8.h"
#include "train_ops.h"

#include <algorithm>

namespace himuon {
namespace {

constexpr int kThreads = 256;
constexpr int kWave = 64;

// ------------------------------------------------------------------- lookup

struct EmbedArgs {
    const void* tokens;
    const void* table;
    void* out;
    int64_t n, rows, ld_table, ld_out, units;
    int32_t dim, wide, segs;
    float scale;
};

// A wave takes 64 / LPR rows (LPR lanes to a row) and U chunks of eight columns
// per lane of them; a row is cut into `segs` such parts.
template <GemmStore ST, int LPR, int U> __global__ void __launch_bounds__(kThreads) embed_rows(const EmbedArgs p)
{
    const int64_t unit = (int64_t)blockIdx.x * (kThreads / kWave) + (threadIdx.x >> 6);
    if (unit >= p.units) return;
    const int lane = threadIdx.x & 63;
    const int64_t group = unit / p.segs;
    const int seg = (int)(unit - group * p.segs);
    const int64_t row = group * (kWave / LPR) + lane / LPR;
    if (row >= p.n) return;
    const int64_t t = load_index(p.tokens, row, p.wide != 0);
    const bool in = t >= 0 && t < p.rows;
    const int64_t src = (in ? t : 0) * p.ld_table, dst = row * p.ld_out;
    const int c0 = seg * (LPR * U * 8) + (lane % LPR) * 8;
    float v[U][8];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int c = c0 + u * LPR * 8;
        if (c < p.dim && in) {
            load8<ST>(p.table, src + c, min(8, p.dim - c), false, v[u]);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[u][e] *= p.scale;
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[u][e] = 0.f;
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int c = c0 + u * LPR * 8;
        if (c < p.dim) store8<ST>(p.out, dst + c, min(8, p.dim - c), false, v[u]);
    }
}

template <GemmStore ST, int LPR, int U> int launch_embed(EmbedArgs p, hipStream_t stream)
{
    p.segs = (int)ceil_div(p.dim, LPR * U * 8);
    p.units = ceil_div(p.n, kWave / LPR) * p.segs;
    const int64_t blocks = ceil_div(p.units, kThreads / kWave);
    if (blocks > INT32_MAX) return HIMUON_ERR_UNSUPPORTED;
    hipLaunchKernelGGL((embed_rows<ST, LPR, U>), dim3((unsigned)blocks), dim3(kThreads), 0, stream, p);
    return launch_status();
}

template <GemmStore ST> int launch_embed_st(const EmbedArgs& p, hipStream_t stream)
{
    // lanes to a row: as many as it has chunks
    if (p.dim <= 64) return launch_embed<ST, 8, 1>(p, stream);
    if (p.dim <= 256) return launch_embed<ST, 32, 1>(p, stream);
    // few rows: one chunk per lane, so that they spread over the chip
    if (p.n * ceil_div(p.dim, 512) < 4096) return launch_embed<ST, 64, 1>(p, stream);
    return launch_embed<ST, 64, 4>(p, stream);
}

// ------------------------------------------------------------------ sorting

// Digits of at most 10 bits; a key is the token, n_rows for one outside the table.
constexpr int kMaxBins = 1024;
constexpr int kIpt = 4;                      // keys per thread and tile
constexpr int kTile = kThreads * kIpt;       // keys of a tile

struct SortArgs {
    const void* tokens;          // first digit: the caller's tokens
    const uint32_t *key_in, *pos_in;
    uint32_t *key_out, *pos_out;
    uint32_t* hist;              // [tiles][bins]
    uint8_t* named;              // rows that some token names, whole 16 bytes (cleared and marked by the first digit)
    int64_t rows;
    int32_t n, wide, tiles, shift, bits, first;
};

__device__ __forceinline__ uint32_t sort_key(const SortArgs& p, int i)
{
    if (!p.first) return p.key_in[i];
    const int64_t t = load_index(p.tokens, i, p.wide != 0);
    return t >= 0 && t < p.rows ? (uint32_t)t : (uint32_t)p.rows;
}

// Counts of each digit in every tile.
__global__ void __launch_bounds__(kThreads) sort_count(const SortArgs p)
{
    __shared__ uint32_t h[kMaxBins];
    const int bins = 1 << p.bits;
    for (int b = threadIdx.x; b < bins; b += kThreads) h[b] = 0;
    if (p.first) {
        for (int64_t r = (int64_t)blockIdx.x * kThreads + threadIdx.x; r < (p.rows + 15) / 16; r += (int64_t)gridDim.x * kThreads)
            reinterpret_cast<uint4*>(p.named)[r] = uint4{};
    }
    __syncthreads();
    if ((int)blockIdx.x >= p.tiles) return;
#pragma unroll
    for (int k = 0; k < kIpt; ++k) {
        const int i = blockIdx.x * kTile + k * kThreads + threadIdx.x;
        if (i < p.n) atomicAdd(&h[(sort_key(p, i) >> p.shift) & (bins - 1)], 1u);
    }
    __syncthreads();
    for (int b = threadIdx.x; b < bins; b += kThreads) p.hist[(int64_t)blockIdx.x * bins + b] = h[b];
}

// Moves a tile's keys to their places by this digit. A wave ranks 64 keys at a time:
// lanes of equal digit find each other by one ballot per bit, the first of them
// takes the digit's count on. So equal digits keep their order.
__global__ void __launch_bounds__(kThreads) sort_scatter(const SortArgs p)
{
    constexpr int W = kThreads / kWave;
    constexpr int BPT = kMaxBins / kThreads;  // bins per thread
    __shared__ uint32_t cnt[W][kMaxBins];
    __shared__ uint32_t wsum[W];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int bins = 1 << p.bits;
    for (int b = tid; b < W * kMaxBins; b += kThreads) (&cnt[0][0])[b] = 0;
    __syncthreads();
    uint32_t key[kIpt], rank[kIpt];
    const int base = blockIdx.x * kTile + wave * (kWave * kIpt);
#pragma unroll
    for (int k = 0; k < kIpt; ++k) {
        const int i = base + k * kWave + lane;
        key[k] = i < p.n ? sort_key(p, i) : 0u;
        if (p.first && i < p.n && key[k] < (uint32_t)p.rows) p.named[key[k]] = 1;
    }
    volatile uint32_t* const mine = cnt[wave];
#pragma unroll
    for (int k = 0; k < kIpt; ++k) {
        const bool valid = base + k * kWave + lane < p.n;
        const uint32_t d = (key[k] >> p.shift) & (uint32_t)(bins - 1);
        uint64_t peers = __ballot(valid);
        for (int b = 0; b < p.bits; ++b) {
            const bool one = (d >> b) & 1;
            const uint64_t m = __ballot(one);
            peers &= one ? m : ~m;
        }
        const uint32_t below = (uint32_t)__popcll(peers & ((UINT64_C(1) << lane) - 1));
        const uint32_t start = mine[d];
        __builtin_amdgcn_wave_barrier();
        rank[k] = start + below;
        if (valid && below == 0) mine[d] = start + (uint32_t)__popcll(peers);
        __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    // Where each digit of this tile starts: all smaller digits, then the same digit
    // in earlier tiles, then in earlier waves.
    uint32_t total[BPT], before[BPT], sum = 0;
#pragma unroll
    for (int j = 0; j < BPT; ++j) total[j] = before[j] = 0;
    const int b0 = tid * BPT;
    if (b0 < bins) {
        const uint4* const row = reinterpret_cast<const uint4*>(p.hist) + tid;
        const int step = bins / BPT;  // (eight rows at a time, all loads in flight)
        for (int t0 = 0; t0 < p.tiles; t0 += 8) {
            uint4 h[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) h[k] = row[(int64_t)min(t0 + k, p.tiles - 1) * step];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const uint32_t on = t0 + k < p.tiles ? ~0u : 0u, earlier = t0 + k < (int)blockIdx.x ? ~0u : 0u;
                const uint32_t v[BPT] = {h[k].x, h[k].y, h[k].z, h[k].w};
#pragma unroll
                for (int j = 0; j < BPT; ++j) {
                    total[j] += v[j] & on;
                    before[j] += v[j] & earlier;
                }
            }
        }
    }
#pragma unroll
    for (int j = 0; j < BPT; ++j) sum += total[j];
    uint32_t scan = sum;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        const uint32_t v = __shfl_up(scan, o);
        if (lane >= o) scan += v;
    }
    if (lane == 63) wsum[wave] = scan;
    __syncthreads();
    uint32_t start = scan - sum;
    for (int w = 0; w < wave; ++w) start += wsum[w];
#pragma unroll
    for (int j = 0; j < BPT; ++j) {
        uint32_t at = start + before[j];
        start += total[j];
        if (b0 + j < bins) {
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const uint32_t c = cnt[w][b0 + j];
                cnt[w][b0 + j] = at;
                at += c;
            }
        }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kIpt; ++k) {
        const int i = base + k * kWave + lane;
        if (i >= p.n) continue;
        const uint32_t at = cnt[wave][(key[k] >> p.shift) & (uint32_t)(bins - 1)] + rank[k];
        p.key_out[at] = key[k];
        p.pos_out[at] = p.first ? (uint32_t)i : p.pos_in[i];
    }
}

// All digits of a short list in one launch: a block of 1024 threads keeps keys and
// positions in LDS (up to kSmall of them).
constexpr int kSmallThreads = 1024;
constexpr int kSmall = kSmallThreads * kIpt;

__global__ void __launch_bounds__(kSmallThreads) sort_small(const SortArgs p, int digits)
{
    constexpr int W = kSmallThreads / kWave;
    __shared__ uint32_t keys[kSmall], poss[kSmall];
    __shared__ uint16_t cnt[W][kMaxBins];
    __shared__ uint32_t wsum[W];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int bins = 1 << p.bits;
    uint32_t key[kIpt], pos[kIpt], rank[kIpt];
    const int base = wave * (kWave * kIpt);
    if (p.named) {
        for (int64_t r = tid; r < (p.rows + 15) / 16; r += kSmallThreads) reinterpret_cast<uint4*>(p.named)[r] = uint4{};
    }
#pragma unroll
    for (int k = 0; k < kIpt; ++k) {
        const int i = base + k * kWave + lane;
        key[k] = i < p.n ? sort_key(p, i) : 0u;
        pos[k] = (uint32_t)i;
    }
    volatile uint16_t* const mine = cnt[wave];
    for (int d = 0; d < digits; ++d) {
        const int shift = d * p.bits;
        for (int b = tid; b < W * kMaxBins / 2; b += kSmallThreads) reinterpret_cast<uint32_t*>(&cnt[0][0])[b] = 0;
        __syncthreads();
        if (d == 0 && p.named) {
#pragma unroll
            for (int k = 0; k < kIpt; ++k)
                if (base + k * kWave + lane < p.n && key[k] < (uint32_t)p.rows) p.named[key[k]] = 1;
        }
#pragma unroll
        for (int k = 0; k < kIpt; ++k) {
            const bool valid = base + k * kWave + lane < p.n;
            const uint32_t g = (key[k] >> shift) & (uint32_t)(bins - 1);
            uint64_t peers = __ballot(valid);
            for (int b = 0; b < p.bits; ++b) {
                const bool one = (g >> b) & 1;
                const uint64_t m = __ballot(one);
                peers &= one ? m : ~m;
            }
            const uint32_t below = (uint32_t)__popcll(peers & ((UINT64_C(1) << lane) - 1));
            const uint32_t start = mine[g];
            __builtin_amdgcn_wave_barrier();
            rank[k] = start + below;
            if (valid && below == 0) mine[g] = (uint16_t)(start + (uint32_t)__popcll(peers));
            __builtin_amdgcn_wave_barrier();
        }
        __syncthreads();
        uint32_t sum = 0;  // thread b: digit b
#pragma unroll
        for (int w = 0; w < W; ++w) sum += cnt[w][tid];
        uint32_t scan = sum;
#pragma unroll
        for (int o = 1; o < kWave; o <<= 1) {
            const uint32_t v = __shfl_up(scan, o);
            if (lane >= o) scan += v;
        }
        if (lane == 63) wsum[wave] = scan;
        __syncthreads();
        uint32_t at = scan - sum;
        for (int w = 0; w < wave; ++w) at += wsum[w];
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const uint32_t c = cnt[w][tid];
            cnt[w][tid] = (uint16_t)at;
            at += c;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kIpt; ++k) {
            if (base + k * kWave + lane < p.n) {
                const uint32_t to = cnt[wave][(key[k] >> shift) & (uint32_t)(bins - 1)] + rank[k];
                keys[to] = key[k];
                poss[to] = pos[k];
            }
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kIpt; ++k) {
            const int i = base + k * kWave + lane;
            key[k] = i < p.n ? keys[i] : 0u;
            pos[k] = i < p.n ? poss[i] : 0u;
        }
    }
#pragma unroll
    for (int k = 0; k < kIpt; ++k) {
        const int i = base + k * kWave + lane;
        if (i < p.n) {
            p.key_out[i] = key[k];
            p.pos_out[i] = pos[k];
        }
    }
}

// --------------------------------------------------------------------- sums

constexpr int kSlab = 512;          // columns of a wave
constexpr uint32_t kNone = 0xffffffffu;

struct SumArgs {
    const uint32_t *key, *pos;      // sorted
    const uint8_t* named;           // null: rows without a token are left alone
    const void* grad;
    void* out;
    float* part;                    // [chunks][2][dim]: the run that a chunk begins in, the one that it ends in
    int64_t rows, ld_grad, ld_out;
    int64_t units, fill_blocks;
    int32_t n, dim, slabs, chunks, accumulate, fill_rows;
    float scale;
};

template <GemmStore OT> __device__ __forceinline__ void put_row(const SumArgs& p, uint32_t row, int c, float (&v)[8])
{
    const int n = min(8, p.dim - c);
    const int64_t i = (int64_t)row * p.ld_out + c;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= p.scale;
    if (p.accumulate) {
        float o[8];
        load8<OT>(p.out, i, n, false, o);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += o[e];
    }
    store8<OT>(p.out, i, n, false, v);
}

__device__ __forceinline__ uint32_t lane_value(uint32_t v, int l) { return (uint32_t)__builtin_amdgcn_readlane((int)v, l); }

template <GemmStore ST, GemmStore OT, int S> __global__ void __launch_bounds__(kThreads) sum_runs(const SumArgs p)
{
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t sum_blocks = (p.units + kThreads / kWave - 1) / (kThreads / kWave);
    if ((int64_t)blockIdx.x >= sum_blocks) {  // rows without a token
        const int64_t r0 = ((int64_t)blockIdx.x - sum_blocks) * (kThreads / kWave) * p.fill_rows + wave * p.fill_rows;
        for (int64_t r = r0; r < min(r0 + p.fill_rows, p.rows); ++r) {
            if (p.named[r]) continue;
            for (int c = lane * 8; c < p.dim; c += kSlab) {
                float z[8] = {};
                store8<OT>(p.out, r * p.ld_out + c, min(8, p.dim - c), false, z);
            }
        }
        return;
    }
    const int64_t unit = (int64_t)blockIdx.x * (kThreads / kWave) + wave;
    if (unit >= p.units) return;
    const int chunk = (int)(unit / p.slabs);
    const int c = (int)(unit - (int64_t)chunk * p.slabs) * kSlab + lane * 8;
    // lane l holds entry chunk S - 1 + l: the one before the chunk, its S, the one after
    const int64_t i = (int64_t)chunk * S - 1 + lane;
    const bool there = i >= 0 && i < p.n && lane < S + 2;
    uint32_t key = there ? p.key[i] : kNone;
    const uint32_t pos = there ? p.pos[i] : 0u;
    if (key >= (uint32_t)p.rows) key = kNone;
    const int count = __popcll(__ballot(key != kNone && lane >= 1 && lane <= S));  // sorted: the first ones
    const bool col = c < p.dim;
    const int nc = min(8, p.dim - c);
    float acc[8] = {};
    bool begun = count > 0 && lane_value(key, 0) != lane_value(key, 1);  // the current run began in this chunk
    constexpr int B = 8;
    for (int e0 = 0; e0 < count; e0 += B) {
        float v[B][8];
#pragma unroll
        for (int e = 0; e < B; ++e) {
            if (e0 + e < count && col)
                load8<ST>(p.grad, (int64_t)lane_value(pos, e0 + e + 1) * p.ld_grad + c, nc, false, v[e]);
        }
#pragma unroll
        for (int e = 0; e < B; ++e) {
            if (e0 + e >= count) break;
            const uint32_t k = lane_value(key, e0 + e + 1);
            const bool last = lane_value(key, e0 + e + 2) != k;
            if (col) {
#pragma unroll
                for (int x = 0; x < 8; ++x) acc[x] += v[e][x];
            }
            if (last || e0 + e + 1 == S) {
                if (col) {
                    if (begun && last) put_row<OT>(p, k, c, acc);
                    else store8<GemmStore::F32>(p.part, (2 * (int64_t)chunk + (begun ? 1 : 0)) * p.dim + c, nc, false, acc);
                }
#pragma unroll
                for (int x = 0; x < 8; ++x) acc[x] = 0.f;
                begun = true;
            }
        }
    }
}

// Adds up the partial sums of the runs that cross chunks: block (chunk, slab) has
// the run that begins in its chunk and goes on after it. The later chunks are
// shared out over the waves in order.
constexpr int kJoinThreads = 512;
template <GemmStore OT, int S> __global__ void __launch_bounds__(kJoinThreads) join_runs(const SumArgs p)
{
    constexpr int W = kJoinThreads / kWave;
    __shared__ float part[W - 1][kWave][8 + 1];
    const int chunk = blockIdx.x;
    const int64_t first = (int64_t)chunk * S, after = first + S;
    if (after >= p.n) return;
    const uint32_t key = p.key[after];
    if (key >= (uint32_t)p.rows || p.key[after - 1] != key) return;
    if (p.key[first] == key && first > 0 && p.key[first - 1] == key) return;  // began in an earlier chunk
    const int lane = threadIdx.x & 63;
    // the last chunk that holds a part: 64 chunks' first entries are asked at once
    int last = chunk + 1;
    for (;;) {
        const int64_t i = (int64_t)(last + 1 + lane) * S;
        const uint64_t ends = __ballot(i >= p.n || p.key[min(i, (int64_t)p.n - 1)] != key);
        if (ends) {
            last += __ffsll((unsigned long long)ends) - 1;
            break;
        }
        last += 64;
    }
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c = blockIdx.y * kSlab + lane * 8;
    const int nc = min(8, p.dim - c);
    const int m = last - chunk, per = (m + W - 1) / W;
    const int from = chunk + 1 + wave * per, to = min(from + per, last + 1);
    float acc[8] = {};
    if (c < p.dim) {
        if (wave == 0) load8<GemmStore::F32>(p.part, (2 * (int64_t)chunk + 1) * p.dim + c, nc, false, acc);
        constexpr int B = 8;
        for (int k0 = from; k0 < to; k0 += B) {
            float v[B][8];
#pragma unroll
            for (int b = 0; b < B; ++b)
                if (k0 + b < to) load8<GemmStore::F32>(p.part, 2 * (int64_t)(k0 + b) * p.dim + c, nc, false, v[b]);
#pragma unroll
            for (int b = 0; b < B; ++b) {
                if (k0 + b < to) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) acc[e] += v[b][e];
                }
            }
        }
    }
    if (wave > 0) {
#pragma unroll
        for (int e = 0; e < 8; ++e) part[wave - 1][lane][e] = acc[e];
    }
    __syncthreads();
    if (wave > 0 || c >= p.dim) return;
#pragma unroll
    for (int w = 0; w < W - 1; ++w) {
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] += part[w][lane][e];
    }
    put_row<OT>(p, key, c, acc);
}

template <GemmStore ST, GemmStore OT, int S> int launch_sums(SumArgs p, hipStream_t stream)
{
    p.chunks = (int)ceil_div(p.n, S);
    p.units = (int64_t)p.chunks * p.slabs;
    const int64_t blocks = ceil_div(p.units, kThreads / kWave) + p.fill_blocks;
    if (blocks > INT32_MAX || p.slabs > 65535) return HIMUON_ERR_UNSUPPORTED;
    if (blocks > 0) {
        hipLaunchKernelGGL((sum_runs<ST, OT, S>), dim3((unsigned)blocks), dim3(kThreads), 0, stream, p);
        const int st = launch_status();
        if (st != HIMUON_OK) return st;
    }
    if (p.chunks < 2) return HIMUON_OK;
    hipLaunchKernelGGL((join_runs<OT, S>), dim3((unsigned)p.chunks, (unsigned)p.slabs), dim3(kJoinThreads), 0, stream, p);
    return launch_status();
}

template <GemmStore ST, GemmStore OT> int launch_sums_t(const SumArgs& p, int s, hipStream_t stream)
{
    return s == 8 ? launch_sums<ST, OT, 8>(p, stream) : launch_sums<ST, OT, 32>(p, stream);
}

// Entries per chunk: short chunks while long ones would leave much of the chip idle.
int chunk_size(int64_t n, int64_t dim) { return ceil_div(n, 32) * ceil_div(dim, kSlab) < 2048 ? 8 : 32; }

int key_bits(int64_t rows)
{
    int b = 1;
    while ((rows >> b) != 0) ++b;  // keys are 0 .. rows
    return b;
}

struct GradPlan {
    size_t key[2], pos[2], hist, named, part, total;
    int digits, bits, tiles, chunk;
};

GradPlan plan_grad(int64_t n, int64_t rows, int64_t dim)
{
    GradPlan g;
    const int kb = key_bits(rows);
    g.digits = (kb + 9) / 10;
    g.bits = std::max(2, (kb + g.digits - 1) / g.digits);  // (bins in groups of four)
    g.tiles = (int)ceil_div(n, kTile);
    g.chunk = chunk_size(n, dim);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t o = at;
        at += round_up(bytes, 256);
        return o;
    };
    for (int b = 0; b < 2; ++b) {
        g.key[b] = take((size_t)n * 4);
        g.pos[b] = take((size_t)n * 4);
    }
    g.hist = take(((size_t)g.tiles << g.bits) * 4);
    g.named = take((size_t)rows);
    g.part = take((size_t)ceil_div(n, g.chunk) * 2 * (size_t)dim * 4);
    g.total = at;
    return g;
}

int embed_grad_sizes(int64_t n, int64_t rows, int64_t dim)
{
    if (n < 0 || rows < 1 || dim < 1) return HIMUON_ERR_INVALID_ARG;
    if (n > INT32_MAX / 2 || rows >= INT32_MAX || dim > INT32_MAX - 1024) return HIMUON_ERR_UNSUPPORTED;
    return HIMUON_OK;
}

}  // namespace
}  // namespace himuon

extern "C" int himuon_embed(int64_t n_tokens, const void* tokens, int index, int64_t n_rows, int64_t dim,
                            const void* table, int64_t ld_table, void* out, int64_t ld_out, float scale, int dtype,
                            void* stream)
{
    using namespace himuon;
    if (n_tokens < 0 || n_rows < 1 || dim < 1 || ld_table < dim || ld_out < dim) return HIMUON_ERR_INVALID_ARG;
    if (!known_dtype(dtype) || !known_index(index)) return HIMUON_ERR_INVALID_ARG;
    if (!table || (n_tokens && (!tokens || !out || out == table))) return HIMUON_ERR_INVALID_ARG;
    if (n_tokens > INT32_MAX || n_rows > INT32_MAX || dim > INT32_MAX - 4096) return HIMUON_ERR_UNSUPPORTED;
    if (!small_product(n_rows, ld_table) || !small_product(n_tokens, ld_out)) return HIMUON_ERR_INVALID_ARG;
    if (n_tokens == 0) return HIMUON_OK;
    StreamDevice on(stream);
    if (on.status != HIMUON_OK) return on.status;
    EmbedArgs p{};
    p.tokens = tokens;
    p.table = table;
    p.out = out;
    p.n = n_tokens;
    p.rows = n_rows;
    p.ld_table = ld_table;
    p.ld_out = ld_out;
    p.dim = (int32_t)dim;
    p.wide = index == HIMUON_I64;
    p.scale = scale;
    const hipStream_t hs = static_cast<hipStream_t>(stream);
    return dtype == HIMUON_BF16 ? launch_embed_st<GemmStore::BF16>(p, hs) : launch_embed_st<GemmStore::F32>(p, hs);
}

extern "C" size_t himuon_embed_grad_workspace_size(int64_t n_tokens, int64_t n_rows, int64_t dim)
{
    using namespace himuon;
    if (embed_grad_sizes(n_tokens, n_rows, dim) != HIMUON_OK) return 0;
    return plan_grad(n_tokens, n_rows, dim).total;
}

extern "C" int himuon_embed_grad(int64_t n_tokens, const void* tokens, int index, int64_t n_rows, int64_t dim,
                                 const void* grad, int64_t ld_grad, int dtype, void* dtable, int64_t ld_dtable,
                                 int out_dtype, float scale, int accumulate, void* workspace, size_t workspace_bytes,
                                 void* stream)
{
    using namespace himuon;
    const int sizes = embed_grad_sizes(n_tokens, n_rows, dim);
    if (sizes != HIMUON_OK) return sizes;
    if (!known_dtype(dtype) || !known_dtype(out_dtype) || !known_index(index)) return HIMUON_ERR_INVALID_ARG;
    if (ld_grad < dim || ld_dtable < dim || !dtable) return HIMUON_ERR_INVALID_ARG;
    if (n_tokens && (!tokens || !grad || grad == dtable)) return HIMUON_ERR_INVALID_ARG;
    if (!small_product(n_rows, ld_dtable) || !small_product(n_tokens, ld_grad)) return HIMUON_ERR_INVALID_ARG;
    const GradPlan g = plan_grad(n_tokens, n_rows, dim);
    if (!workspace || workspace_bytes < g.total || ((uintptr_t)workspace & 15)) return HIMUON_ERR_WORKSPACE;
    if (n_tokens == 0 && accumulate) return HIMUON_OK;
    StreamDevice on(stream);
    if (on.status != HIMUON_OK) return on.status;
    const hipStream_t hs = static_cast<hipStream_t>(stream);
    uint8_t* const ws = static_cast<uint8_t*>(workspace);

    SortArgs s{};
    s.tokens = tokens;
    s.hist = reinterpret_cast<uint32_t*>(ws + g.hist);
    s.named = ws + g.named;
    s.rows = n_rows;
    s.n = (int32_t)n_tokens;
    s.wide = index == HIMUON_I64;
    s.tiles = g.tiles;
    s.bits = g.bits;
    int from = 0;
    const bool small = n_tokens > 0 && n_tokens <= kSmall;
    if (small) {
        s.first = 1;
        if (accumulate) s.named = nullptr;
        s.key_out = reinterpret_cast<uint32_t*>(ws + g.key[0]);
        s.pos_out = reinterpret_cast<uint32_t*>(ws + g.pos[0]);
        hipLaunchKernelGGL(sort_small, dim3(1), dim3(kSmallThreads), 0, hs, s, g.digits);
        const int st = launch_status();
        if (st != HIMUON_OK) return st;
    }
    for (int d = 0; !small && d < (n_tokens ? g.digits : 1); ++d) {
        s.first = d == 0;
        s.shift = d * g.bits;
        s.key_in = reinterpret_cast<const uint32_t*>(ws + g.key[from]);
        s.pos_in = reinterpret_cast<const uint32_t*>(ws + g.pos[from]);
        s.key_out = reinterpret_cast<uint32_t*>(ws + g.key[from ^ 1]);
        s.pos_out = reinterpret_cast<uint32_t*>(ws + g.pos[from ^ 1]);
        from ^= 1;
        const int clear = d == 0 ? (int)std::min<int64_t>(ceil_div(n_rows, kThreads * 16), 256) : 1;
        hipLaunchKernelGGL(sort_count, dim3((unsigned)std::max(g.tiles, clear)), dim3(kThreads), 0, hs, s);
        int st = launch_status();
        if (st != HIMUON_OK) return st;
        if (n_tokens == 0) break;
        hipLaunchKernelGGL(sort_scatter, dim3((unsigned)g.tiles), dim3(kThreads), 0, hs, s);
        st = launch_status();
        if (st != HIMUON_OK) return st;
    }
    SumArgs p{};
    p.key = reinterpret_cast<const uint32_t*>(ws + g.key[from]);
    p.pos = reinterpret_cast<const uint32_t*>(ws + g.pos[from]);
    p.named = accumulate ? nullptr : ws + g.named;
    p.grad = grad;
    p.out = dtable;
    p.part = reinterpret_cast<float*>(ws + g.part);
    p.rows = n_rows;
    p.ld_grad = ld_grad;
    p.ld_out = ld_dtable;
    p.n = (int32_t)n_tokens;
    p.dim = (int32_t)dim;
    p.slabs = (int32_t)ceil_div(dim, kSlab);
    p.accumulate = accumulate != 0;
    p.scale = scale;
    // about 16 KB to a wave
    p.fill_rows = (int32_t)std::max<int64_t>(1, std::min<int64_t>(64, 16384 / (dim * dtype_size(out_dtype))));
    p.fill_blocks = accumulate ? 0 : ceil_div(n_rows, (int64_t)p.fill_rows * (kThreads / kWave));
    if (dtype == HIMUON_BF16)
        return out_dtype == HIMUON_BF16 ? launch_sums_t<GemmStore::BF16, GemmStore::BF16>(p, g.chunk, hs)
                                        : launch_sums_t<GemmStore::BF16, GemmStore::F32>(p, g.chunk, hs);
    return out_dtype == HIMUON_BF16 ? launch_sums_t<GemmStore::F32, GemmStore::BF16>(p, g.chunk, hs)
                                    : launch_sums_t<GemmStore::F32, GemmStore::F32>(p, g.chunk, hs);
}
