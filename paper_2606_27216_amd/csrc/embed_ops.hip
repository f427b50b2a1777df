// Token table lookup and its gradient (himuon_embed, himuon_embed_grad).
//
//     out[i, :] = scale E[t_i, :]          dE[v, :] = scale sum_{i: t_i = v} g[i, :]
//
// Both are bound by memory. The lookup is a gather: a row (or a part of one) per
// group of lanes, four 16-byte chunks in flight per lane.
//
// The gradient sorts the tokens (stably: short lists by comparison, longer ones in parts that
// are merged, long ones by digits, ranked by ballots within a wave), so that a row's terms
// are adjacent and its sum has one order. The sorted list is cut into chunks of S
// entries, whatever rows they name: a wave sums the runs of equal tokens of its
// chunk over 512 columns. Runs that lie inside a chunk go to the table at once; a run
// that crosses chunks leaves one fp32 partial sum per chunk, and a last launch
// adds these up in order. So a token that makes up much of a batch is spread over the
// chip like any other. The sort is short launches that wait more than they work: blocks
// that set the table to zero ride in them, and the sums then write the rows that occur.
//
// Measured: lookup of 16384 x 2560 bf16 22 us (121 MB, 5.5 TB/s); gradient of 16384 x 4096
// into 32000 rows, bf16, 90 us a call on inputs that change (396 MB that it cannot do without, 4.4
// TB/s), 84 on the same ones again: the sort with the zeros 48, sums 31, joins 6.
#include "elementwise8.h"
#include "ns_device.h"
#include "train_ops.h"

#include <algorithm>

namespace himuon {
namespace {

using namespace dev;

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
    const int last = max(p.dim - 8, 0);  // (a row's last chunk ends with it, and has columns of the one before it too)
    float v[U][8];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int c = c0 + u * LPR * 8;
        if (c < p.dim && in) {
            load8<ST>(p.table, src + min(c, last), min(8, p.dim), false, v[u]);
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
        if (c < p.dim) store8<ST>(p.out, dst + min(c, last), min(8, p.dim), false, v[u]);
    }
}

template <GemmStore ST, int LPR, int U> int launch_embed(EmbedArgs p, hipStream_t stream)
{
    p.segs = (int)ceil_div(p.dim, LPR * U * 8);
    p.units = ceil_div(p.n, kWave / LPR) * p.segs;
    const int64_t blocks = ceil_div(p.units, kThreads / kWave);
    if (!launchable(blocks, kThreads)) return HIMUON_ERR_UNSUPPORTED;
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

// ------------------------------------------------------------------- zeros

// Rows set to zero by the blocks of a launch from `first` on.
struct FillArgs {
    uint8_t* out;
    int64_t row_bytes, ld_bytes, from, to;  // rows
    int32_t first, blocks;
    int32_t stream;  // past the caches
};

template <int THREADS, bool STREAM> __device__ __forceinline__ void fill_rows_as(const FillArgs& f)
{
    typedef uint32_t Chunk __attribute__((ext_vector_type(4)));
    typedef Chunk ChunkAny __attribute__((aligned(2)));
    const int64_t b = (int64_t)blockIdx.x - f.first;
    auto zero = [](uint8_t* p, int64_t n) {
        if (n >= 16) {
            if constexpr (STREAM) __builtin_nontemporal_store(Chunk{}, reinterpret_cast<ChunkAny*>(p));
            else *reinterpret_cast<ChunkAny*>(p) = Chunk{};
        } else {
            for (int64_t i = 0; i < n; i += 2) *reinterpret_cast<uint16_t*>(p + i) = 0;
        }
    };
    if (f.ld_bytes == f.row_bytes) {
        uint8_t* const base = f.out + f.from * f.ld_bytes;
        const int64_t n = (f.to - f.from) * f.row_bytes;
        for (int64_t i = (b * THREADS + threadIdx.x) * 16; i < n; i += (int64_t)f.blocks * THREADS * 16) zero(base + i, n - i);
    } else {
        const int64_t step = (int64_t)f.blocks * (THREADS / kWave);
        for (int64_t r = f.from + b * (THREADS / kWave) + (threadIdx.x >> 6); r < f.to; r += step)
            for (int64_t i = (threadIdx.x & 63) * 16; i < f.row_bytes; i += 1024) zero(f.out + r * f.ld_bytes + i, f.row_bytes - i);
    }
}

template <int THREADS> __device__ __forceinline__ void fill_rows(const FillArgs& f)
{
    if (f.stream) fill_rows_as<THREADS, true>(f);
    else fill_rows_as<THREADS, false>(f);
}

// ------------------------------------------------------------------ sorting

// Digits of at most 10 bits; a key is the token, n_rows for one outside the table.
constexpr int kMaxBins = 1024;
constexpr int kIpt = 4;                      // keys per thread and tile
constexpr int kTile = kThreads * kIpt;       // keys of a tile
constexpr uint32_t kNone = 0xffffffffu;      // no key

struct SortArgs {
    const void* tokens;          // first digit: the caller's tokens
    const uint32_t *key_in, *pos_in;
    uint32_t *key_out, *pos_out;
    uint32_t* hist;              // [tiles][bins], scanned: [tiles + 1][bins]
    int64_t rows;
    int32_t n, wide, tiles, shift, bits, first, scanned;
    int32_t groups;              // sort_rank: of 64 entries, in a part of the list
    FillArgs fill;
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
    if ((int)blockIdx.x >= p.fill.first) return fill_rows<kThreads>(p.fill);
    const int bins = 1 << p.bits;
    for (int b = threadIdx.x; b < bins; b += kThreads) h[b] = 0;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kIpt; ++k) {
        const int i = blockIdx.x * kTile + k * kThreads + threadIdx.x;
        if (i < p.n) atomicAdd(&h[(sort_key(p, i) >> p.shift) & (bins - 1)], 1u);
    }
    __syncthreads();
    for (int b = threadIdx.x; b < bins; b += kThreads) p.hist[(int64_t)blockIdx.x * bins + b] = h[b];
}

// Long lists: the tiles' counts of a digit become those of the tiles before each, with the
// totals in a row of their own. A block has 64 digits, its waves a part of the tiles each.
constexpr int kScanThreads = 1024;

__global__ void __launch_bounds__(kScanThreads) sort_scan(const SortArgs p)
{
    constexpr int W = kScanThreads / kWave, U = 16;
    __shared__ uint32_t sums[W][kWave];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int bins = 1 << p.bits, bin = blockIdx.x * kWave + lane;
    const bool on = bin < bins;
    uint32_t* const col = p.hist + (on ? bin : 0);
    const int t0 = (int)((int64_t)p.tiles * wave / W), t1 = (int)((int64_t)p.tiles * (wave + 1) / W);
    uint32_t sum = 0;
    for (int t = t0; t < t1; t += U) {
        uint32_t h[U];
#pragma unroll
        for (int k = 0; k < U; ++k) h[k] = col[(int64_t)min(t + k, t1 - 1) * bins];
#pragma unroll
        for (int k = 0; k < U; ++k) sum += t + k < t1 ? h[k] : 0u;
    }
    sums[wave][lane] = sum;
    __syncthreads();
    uint32_t before = 0;
    for (int w = 0; w < wave; ++w) before += sums[w][lane];
    for (int t = t0; t < t1; t += U) {
        uint32_t h[U];
#pragma unroll
        for (int k = 0; k < U; ++k) h[k] = col[(int64_t)min(t + k, t1 - 1) * bins];
#pragma unroll
        for (int k = 0; k < U; ++k) {
            if (t + k < t1 && on) col[(int64_t)(t + k) * bins] = before;
            before += t + k < t1 ? h[k] : 0u;
        }
    }
    if (wave == W - 1 && on) col[(int64_t)p.tiles * bins] = before;
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
    if ((int)blockIdx.x >= p.fill.first) return fill_rows<kThreads>(p.fill);
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
    if (b0 < bins && p.scanned) {
        const uint4* const row = reinterpret_cast<const uint4*>(p.hist) + tid;
        const int64_t step = bins / BPT;
        const uint4 all = row[p.tiles * step], earlier = row[blockIdx.x * step];
        const uint32_t a[BPT] = {all.x, all.y, all.z, all.w}, v[BPT] = {earlier.x, earlier.y, earlier.z, earlier.w};
#pragma unroll
        for (int j = 0; j < BPT; ++j) {
            total[j] = a[j];
            before[j] = v[j];
        }
    } else if (b0 < bins) {
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

// Short lists are sorted by comparison: an entry's place is the number of entries before it,
// those with a smaller key and earlier ones with the same. A block ranks 64 entries, its waves
// share out what these are compared with: the whole list, or a part of it.
constexpr int kRankThreads = 1024;  // where it is the whole list

template <int THREADS> __global__ void __launch_bounds__(THREADS) sort_rank(const SortArgs p)
{
    constexpr int W = THREADS / kWave;
    __shared__ uint32_t count[W][kWave];
    if ((int)blockIdx.x >= p.fill.first) return fill_rows<THREADS>(p.fill);
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int i = blockIdx.x * kWave + lane;
    const int c0 = (int)blockIdx.x / p.groups * p.groups, c1 = min(c0 + p.groups, (p.n + kWave - 1) / kWave);
    const uint32_t key = i < p.n ? sort_key(p, i) : 0u;
    uint32_t before = 0;
    for (int c = c0 + wave; c < c1; c += W) {
        const int j = c * kWave + lane;
        const uint32_t other = j < p.n ? sort_key(p, j) : 0xffffffffu;
        if (c == (int)blockIdx.x) {
#pragma unroll 16
            for (int l = 0; l < kWave; ++l) {
                const uint32_t k = (uint32_t)__builtin_amdgcn_readlane((int)other, l);
                before += (k < key || (k == key && l < lane)) ? 1u : 0u;
            }
        } else {
            const uint32_t limit = key + (c < (int)blockIdx.x ? 1u : 0u);  // (keys are below 2^31)
#pragma unroll 16
            for (int l = 0; l < kWave; ++l) before += (uint32_t)__builtin_amdgcn_readlane((int)other, l) < limit ? 1u : 0u;
        }
    }
    count[wave][lane] = before;
    __syncthreads();
    if (wave > 0 || i >= p.n) return;
    uint32_t at = (uint32_t)(c0 * kWave);
#pragma unroll
    for (int w = 0; w < W; ++w) at += count[w][lane];
    p.key_out[at] = key;
    p.pos_out[at] = (uint32_t)i;
}

// The sorted parts of a list, merged: an entry's place is its place in its own part and, for
// each other part, the number of entries there that come before it, by bisection. A block
// places 64 entries (neighbours in their part, so that they take nearly the same steps), its
// waves have a part each at a time, in LDS.
constexpr int kPart = 1024;

template <int THREADS> __global__ void __launch_bounds__(THREADS) sort_merge(const SortArgs p)
{
    constexpr int W = THREADS / kWave;
    __shared__ __attribute__((aligned(16))) uint32_t parts[W][kPart];
    __shared__ uint32_t count[W][kWave];
    if ((int)blockIdx.x >= p.fill.first) return fill_rows<THREADS>(p.fill);
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int i = blockIdx.x * kWave + lane, own = (int)blockIdx.x / (kPart / kWave);
    const uint32_t key = p.key_in[min(i, p.n - 1)];
    uint32_t* const part = parts[wave];
    uint32_t before = 0;
    for (int t = wave; t * kPart < p.n; t += W) {
        if (t == own) {
            before += (uint32_t)(i - own * kPart);
            continue;
        }
        // (the last part's reads past the list stay within the workspace, and count for nothing)
        const int first = t * kPart + 4 * lane;
        uint4 k[kPart / 256];
#pragma unroll
        for (int u = 0; u < kPart / 256; ++u) k[u] = *reinterpret_cast<const uint4*>(p.key_in + first + 256 * u);
#pragma unroll
        for (int u = 0; u < kPart / 256; ++u) {
            const int at = first + 256 * u;
            const uint4 v = uint4{at < p.n ? k[u].x : kNone, at + 1 < p.n ? k[u].y : kNone, at + 2 < p.n ? k[u].z : kNone,
                                  at + 3 < p.n ? k[u].w : kNone};
            *reinterpret_cast<uint4*>(part + 4 * lane + 256 * u) = v;
        }
        wave_exchange();
        const uint32_t limit = key + (t < own ? 1u : 0u);
        uint32_t n = 0;
#pragma unroll
        for (int step = kPart / 2; step > 0; step /= 2) n += part[n + step - 1] < limit ? step : 0;
        n += part[n] < limit ? 1u : 0u;
        before += n;
        wave_exchange();
    }
    count[wave][lane] = before;
    __syncthreads();
    if (wave > 0 || i >= p.n) return;
    uint32_t at = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) at += count[w][lane];
    p.key_out[at] = key;
    p.pos_out[at] = p.pos_in[i];
}

// --------------------------------------------------------------------- sums

constexpr int kSlab = 512;          // columns of a wave

struct SumArgs {
    const uint32_t *key, *pos;      // sorted
    const void* grad;
    void* out;
    float* part;                    // [chunks][2][dim]: the run that a chunk begins in, the one that it ends in
    int64_t rows, ld_grad, ld_out;
    int64_t units;
    int32_t n, dim, slabs, chunks, accumulate;
    float scale;
};

// A lane's eight columns: the last lane's end with the last column, and begin with some of
// the lane before it, which it sums up as well but does not store. (Of fewer columns than
// eight loads would be made one by one, and each row's waited for: 32768 x 947 62 us a call, so 50.)
struct Cols {
    int first, n;  // fewer than eight only if there are no more
    int skip;      // leading ones that are not stored: all of a lane past the last column
};

__device__ __forceinline__ Cols lane_cols(int lane_col, int dim)
{
    Cols c;
    const bool in = lane_col < dim;
    c.first = in ? min(lane_col, max(dim - 8, 0)) : 0;
    c.n = min(8, dim - c.first);
    c.skip = in ? lane_col - c.first : 8;
    return c;
}

template <GemmStore OT>
__device__ __forceinline__ void put_cols(void* out, int64_t i, const Cols& c, bool accumulate, float (&v)[8])
{
    if (c.skip == 0) {
        if (accumulate) {
            float o[8];
            load8<OT>(out, i, c.n, false, o);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += o[e];
        }
        store8<OT>(out, i, c.n, false, v);
    } else {
#pragma unroll
        for (int e = 1; e < 8; ++e)
            if (e >= c.skip) put1<OT>(out, i + e, accumulate ? v[e] + get1<OT>(out, i + e) : v[e]);
    }
}

template <GemmStore OT> __device__ __forceinline__ void put_row(const SumArgs& p, uint32_t row, const Cols& c, float (&v)[8])
{
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= p.scale;
    put_cols<OT>(p.out, (int64_t)row * p.ld_out + c.first, c, p.accumulate != 0, v);
}

__device__ __forceinline__ uint32_t lane_value(uint32_t v, int l) { return (uint32_t)__builtin_amdgcn_readlane((int)v, l); }

template <GemmStore ST, GemmStore OT, int S> __global__ void __launch_bounds__(kThreads) sum_runs(const SumArgs p)
{
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t unit = (int64_t)blockIdx.x * (kThreads / kWave) + wave;
    if (unit >= p.units) return;
    const int chunk = (int)(unit / p.slabs);
    const int lane_col = (int)(unit - (int64_t)chunk * p.slabs) * kSlab + lane * 8;
    const Cols c = lane_cols(lane_col, p.dim);
    // lane l holds entry chunk S - 1 + l: the one before the chunk, its S, the one after
    const int64_t i = (int64_t)chunk * S - 1 + lane;
    const bool there = i >= 0 && i < p.n && lane < S + 2;
    uint32_t key = there ? p.key[i] : kNone;
    const uint32_t pos = there ? p.pos[i] : 0u;
    if (key >= (uint32_t)p.rows) key = kNone;
    const int count = __popcll(__ballot(key != kNone && lane >= 1 && lane <= S));  // sorted: the first ones
    float acc[8] = {};
    bool begun = count > 0 && lane_value(key, 0) != lane_value(key, 1);  // the current run began in this chunk
    // rows of B entries are in flight while those before them are summed
    constexpr int B = ST == GemmStore::BF16 ? 8 : 4;
    Raw8<ST> cur[B], next[B];
    auto load = [&](Raw8<ST> (&v)[B], int e0) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < B; ++e)
            v[e] = get_raw8<ST>(p.grad, (int64_t)lane_value(pos, min(e0 + e, count - 1) + 1) * p.ld_grad + c.first, c.n);
    };
    if (count == 0) return;
    load(next, 0);
#pragma unroll 1
    for (int e0 = 0; e0 < count; e0 += B) {
#pragma unroll
        for (int e = 0; e < B; ++e) cur[e] = next[e];
        if (e0 + B < count) load(next, e0 + B);
#pragma unroll
        for (int e = 0; e < B; ++e) {
            if (e0 + e >= count) break;
            const uint32_t k = lane_value(key, e0 + e + 1);
            const bool last = lane_value(key, e0 + e + 2) != k;
#pragma unroll
            for (int x = 0; x < 8; ++x) acc[x] += raw_value<ST>(cur[e], x);
            if (last || e0 + e + 1 == S) {
                if (c.skip < 8) {
                    if (begun && last) put_row<OT>(p, k, c, acc);
                    else put_cols<GemmStore::F32>(p.part, (2 * (int64_t)chunk + (begun ? 1 : 0)) * p.dim + c.first, c, false, acc);
                }
#pragma unroll
                for (int x = 0; x < 8; ++x) acc[x] = 0.f;
                begun = true;
            }
        }
    }
}

// Adds up the partial sums of the runs that cross chunks. A wave has the run that begins in
// its chunk and goes on after it; runs of more than kOwnParts parts are shared out over all
// waves of the block, in order (one token 30000 times, 640 columns: the whole call 60 us
// with each run left to four waves, 49 so).
constexpr int kOwnParts = 32;

// N consecutive columns of a part, of which n exist.
template <int N> __device__ __forceinline__ void load_part(const float* p, int n, float (&v)[N])
{
    if constexpr (N == 8) {
        load8<GemmStore::F32>(p, 0, n, false, v);
    } else {
        f32x4 w{};
        if (n == 4) w = *reinterpret_cast<const f32x4_any32*>(p);
        else w = f32x4{p[0], n > 1 ? p[1] : 0.f, n > 2 ? p[2] : 0.f, 0.f};
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = w[e];
    }
}

template <GemmStore OT> __device__ __forceinline__ void put_row(const SumArgs& p, uint32_t row, int c, float (&v)[8])
{
    put_row<OT>(p, row, Cols{c, min(8, p.dim - c), 0}, v);
}

template <GemmStore OT> __device__ __forceinline__ void put_row(const SumArgs& p, uint32_t row, int c, float (&v)[4])
{
    const int n = min(4, p.dim - c);
    const int64_t i = (int64_t)row * p.ld_out + c;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] *= p.scale;
    if (p.accumulate) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += e < n ? get1<OT>(p.out, i + e) : 0.f;
    }
    if (n == 4) {
        if constexpr (OT == GemmStore::BF16)
            *reinterpret_cast<u32x2_any16*>(static_cast<uint16_t*>(p.out) + i) =
                u32x2{pack2<Operand::BF16>(v[0], v[1]), pack2<Operand::BF16>(v[2], v[3])};
        else
            *reinterpret_cast<f32x4_any32*>(static_cast<float*>(p.out) + i) = f32x4{v[0], v[1], v[2], v[3]};
    } else {
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (e < n) put1<OT>(p.out, i + e, v[e]);
    }
}

// COLS: columns of a lane. Four instead of eight keep twice the parts in flight, but take twice
// the blocks: one token 30000 times, 640 columns 39 us a call and 49; 32768 x 4096
// 129 and 119, 131072 x 1024 109 and 103.
template <GemmStore OT, int S, int kJoinWaves, int COLS> __global__ void __launch_bounds__(kJoinWaves * kWave) join_runs(const SumArgs p)
{
    __shared__ float lds[kJoinWaves][kWave][COLS + 1];
    __shared__ int parts[kJoinWaves];  // of each wave's run, if it is shared out
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int chunk = blockIdx.x * kJoinWaves + wave;
    const int c = blockIdx.y * (kWave * COLS) + lane * COLS, nc = min(COLS, p.dim - c);
    const int64_t first = (int64_t)chunk * S, after = first + S, most = (int64_t)p.n - 1;
    const uint32_t before = p.key[min(max(first - 1, (int64_t)0), most)], begin = p.key[min(first, most)],
                   end = p.key[min(after - 1, most)], next = p.key[min(after, most)];
    int n = 0;  // chunks after this one that the run reaches into
    if (after <= most && next == end && end < (uint32_t)p.rows && !(begin == end && first > 0 && before == end)) {
        // 64 chunks' first entries are asked at once, `step` apart; how many belong to the run
        auto ask = [&](int64_t from, int64_t step) -> int {
            const int64_t i = (from + lane * step) * S;
            const uint64_t out = __ballot(i > most || p.key[min(i, most)] != end);
            return out ? __ffsll((unsigned long long)out) - 1 : kWave;
        };
        n = ask(chunk + 1, 1);
        if (n == kWave) {
            for (;;) {
                const int m = ask((int64_t)chunk + 1 + n, kWave);  // (its first one need not be)
                if (m == 0) break;
                n += (m - 1) * kWave;
                if (m < kWave) break;
            }
            n += ask((int64_t)chunk + 1 + n, 1);
        }
    }
    float acc[COLS] = {};
    // adds parts from .. to - 1 of the run that begins in chunk `at` (0: that chunk's own)
    auto add = [&](int at, int from, int to) __attribute__((always_inline)) {
        constexpr int B = 64 / COLS;
        for (int k0 = from; k0 < to; k0 += B) {
            float v[B][COLS];
#pragma unroll
            for (int b = 0; b < B; ++b) {
                const int k = min(k0 + b, to - 1);
                load_part(p.part + (2 * (int64_t)(at + k) + (k == 0 ? 1 : 0)) * p.dim + c, nc, v[b]);
            }
#pragma unroll
            for (int b = 0; b < B; ++b) {
#pragma unroll
                for (int e = 0; e < COLS; ++e) acc[e] += k0 + b < to ? v[b][e] : 0.f;
            }
        }
    };
    const bool shared_out = n + 1 > kOwnParts;
    if (lane == 0) parts[wave] = shared_out ? n + 1 : 0;
    if (n > 0 && !shared_out && c < p.dim) {
        add(chunk, 0, n + 1);
        put_row<OT>(p, end, c, acc);
    }
    __syncthreads();
    for (int w = 0; w < kJoinWaves; ++w) {
        const int m = __builtin_amdgcn_readfirstlane(parts[w]);
        if (m == 0) continue;
        const int per = (m + kJoinWaves - 1) / kJoinWaves, from = min(wave * per, m), to = min(from + per, m);
#pragma unroll
        for (int e = 0; e < COLS; ++e) acc[e] = 0.f;
        if (c < p.dim) add(blockIdx.x * kJoinWaves + w, from, to);
#pragma unroll
        for (int e = 0; e < COLS; ++e) lds[wave][lane][e] = acc[e];
        __syncthreads();
        if (wave == w && c < p.dim) {
#pragma unroll
            for (int e = 0; e < COLS; ++e) acc[e] = lds[0][lane][e];
            for (int x = 1; x < kJoinWaves; ++x) {
#pragma unroll
                for (int e = 0; e < COLS; ++e) acc[e] += lds[x][lane][e];
            }
            put_row<OT>(p, end, c, acc);
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------- short batches

// A batch of few tokens in one launch, without a sort. Block i has token i: its waves
// compare a part of the batch each with it. Unless it occurs earlier too, they sum the
// rows where it occurs, in order, and the parts are added up in order. The blocks behind
// these set rows to zero that no token names, which each finds out for its own.
constexpr int kFewThreads = 512, kFewWaves = kFewThreads / kWave;
constexpr int kFewMost = 1024;
constexpr int kFewParts = kFewMost / kFewThreads;  // tokens of a lane

struct FewArgs {
    SortArgs sort;                  // tokens, rows, n, wide, first
    SumArgs sum;
    uint8_t* out;
    int64_t row_bytes, ld_bytes;
    int32_t fill_rows;              // rows of a block
    int32_t share;                  // tokens of a wave
};

template <GemmStore ST, GemmStore OT> __global__ void __launch_bounds__(kFewThreads) sum_few(const FewArgs f)
{
    typedef uint32_t Chunk __attribute__((ext_vector_type(4)));
    typedef Chunk ChunkAny __attribute__((aligned(2)));
    constexpr int kFillMost = 4096;
    __shared__ float part[kFewWaves - 1][kWave][8 + 1];
    __shared__ int seen[kFewWaves];
    __shared__ uint8_t named[kFillMost];
    const SumArgs& p = f.sum;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if ((int)blockIdx.x >= p.n) {
        if (blockIdx.y > 0) return;
        const int64_t r0 = (int64_t)((int)blockIdx.x - p.n) * f.fill_rows;
        const int rows = (int)min((int64_t)f.fill_rows, p.rows - r0);
        for (int r = threadIdx.x; r < rows; r += kFewThreads) named[r] = 0;
        __syncthreads();
        for (int i = threadIdx.x; i < p.n; i += kFewThreads) {
            const int64_t r = (int64_t)sort_key(f.sort, i) - r0;
            if (r >= 0 && r < rows) named[r] = 1;
        }
        __syncthreads();
        const uint32_t per = (uint32_t)((f.row_bytes + 15) / 16);
        // (a launch's blocks have at most 4096 rows of at most 32 KB, or one row)
        for (uint32_t x = threadIdx.x; x < per * (uint32_t)rows; x += kFewThreads) {
            const uint32_t r = x / per;
            const int64_t c = (int64_t)(x - r * per) * 16;
            if (named[r]) continue;
            uint8_t* const at = f.out + (r0 + r) * f.ld_bytes + c;
            const int64_t left = f.row_bytes - c;
            if (left >= 16) *reinterpret_cast<ChunkAny*>(at) = Chunk{};
            else
                for (int64_t i = 0; i < left; i += 2) *reinterpret_cast<uint16_t*>(at + i) = 0;
        }
        return;
    }
    const int mine = blockIdx.x;
    const uint32_t key = sort_key(f.sort, mine);
    if (key >= (uint32_t)p.rows) return;
    uint64_t same[kFewParts];
    int first = p.n;  // of this wave's tokens, the first one that is the same
#pragma unroll
    for (int g = kFewParts - 1; g >= 0; --g) {
        const int x = g * kWave + lane, i = wave * f.share + x;
        const bool on = x < f.share && i < p.n;
        same[g] = __ballot(on && sort_key(f.sort, on ? i : 0) == key);
        if (same[g]) first = wave * f.share + g * kWave + __ffsll((unsigned long long)same[g]) - 1;
    }
    if (lane == 0) seen[wave] = first;
    __syncthreads();
    int earliest = p.n;
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) earliest = min(earliest, seen[w]);
    if (earliest < mine) return;
    const int slabs = (p.dim + kSlab - 1) / kSlab;
    for (int slab = blockIdx.y; slab < slabs; slab += gridDim.y) {
        const Cols c = lane_cols(slab * kSlab + lane * 8, p.dim);
        float acc[8] = {};
#pragma unroll
        for (int g = 0; g < kFewParts; ++g) {
            uint64_t m = same[g];
            const int base = wave * f.share + g * kWave;
            constexpr int B = 8;
            while (m) {
                Raw8<ST> v[B];
                int n = 0, at = 0;
#pragma unroll
                for (int b = 0; b < B; ++b) {
                    if (m) {
                        at = base + __ffsll((unsigned long long)m) - 1;
                        m &= m - 1;
                        ++n;
                    }
                    v[b] = get_raw8<ST>(p.grad, (int64_t)at * p.ld_grad + c.first, c.n);
                }
#pragma unroll
                for (int b = 0; b < B; ++b) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) acc[e] += b < n ? raw_value<ST>(v[b], e) : 0.f;
                }
            }
        }
        __syncthreads();
        if (wave > 0) {
#pragma unroll
            for (int e = 0; e < 8; ++e) part[wave - 1][lane][e] = acc[e];
        }
        __syncthreads();
        if (wave == 0 && c.skip < 8) {
#pragma unroll
            for (int w = 0; w < kFewWaves - 1; ++w) {
                if (seen[w + 1] < p.n) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) acc[e] += part[w][lane][e];
                }
            }
            put_row<OT>(p, key, c, acc);
        }
    }
}

template <GemmStore ST, GemmStore OT> int launch_few(const FewArgs& f, hipStream_t stream)
{
    const int64_t fill = f.sum.accumulate ? 0 : ceil_div(f.sum.rows, f.fill_rows);
    if (!launchable(f.sum.n + fill, kFewThreads)) return HIMUON_ERR_UNSUPPORTED;
    // columns shared out over blocks while these are few: one token 100 times, 4096 columns
    const int64_t parts = std::min<int64_t>(f.sum.slabs, std::max<int64_t>(2, 2048 / f.sum.n));
    hipLaunchKernelGGL((sum_few<ST, OT>), dim3((unsigned)(f.sum.n + fill), (unsigned)parts), dim3(kFewThreads), 0, stream, f);
    return launch_status();
}

template <GemmStore OT, int S, int WAVES, int COLS> int launch_join(const SumArgs& p, hipStream_t stream)
{
    const dim3 grid((unsigned)ceil_div(p.chunks, WAVES), (unsigned)ceil_div(p.dim, kWave * COLS));
    hipLaunchKernelGGL((join_runs<OT, S, WAVES, COLS>), grid, dim3(WAVES * kWave), 0, stream, p);
    return launch_status();
}

template <GemmStore ST, GemmStore OT, int S> int launch_sums(SumArgs p, hipStream_t stream)
{
    p.chunks = (int)ceil_div(p.n, S);
    p.units = (int64_t)p.chunks * p.slabs;
    const int64_t blocks = ceil_div(p.units, kThreads / kWave);
    hipLaunchKernelGGL((sum_runs<ST, OT, S>), dim3((unsigned)blocks), dim3(kThreads), 0, stream, p);
    const int st = launch_status();
    if (st != HIMUON_OK || p.chunks < 2) return st;
    // (a block of 16 waves starts later than one of four: 1500 tokens 21.2 us and 18.5)
    if (p.n <= 2048) return p.dim <= 1024 ? launch_join<OT, S, 4, 4>(p, stream) : launch_join<OT, S, 4, 8>(p, stream);
    return p.dim <= 1024 && p.n <= 32768 ? launch_join<OT, S, 16, 4>(p, stream) : launch_join<OT, S, 16, 8>(p, stream);
}

template <GemmStore ST, GemmStore OT> int launch_sums_t(const SumArgs& p, int s, hipStream_t stream)
{
    if (s == 8) return launch_sums<ST, OT, 8>(p, stream);
    return s == 16 ? launch_sums<ST, OT, 16>(p, stream) : launch_sums<ST, OT, 32>(p, stream);
}

// Entries per chunk: short chunks while long ones would leave much of the chip idle. A wave
// has a chunk of 512 columns. Measured with 8, 16 and 32, Zipf's tokens (one token throughout):
// 8192 x 947 35 us (46), 39 (40), 51 (44); 12000 x 947 40 (55), 43 (47), 52 (48); 5000 x 2560 41 (52), 41
// (43), 44 (41); 8192 x 4096 78 (95), 75 (80), 72 (68); 32768 x 256 33 (76), 33 (53), 36 (42).
int chunk_size(int64_t n, int64_t dim)
{
    const int64_t work = n * ceil_div(dim, kSlab);
    if (n <= 8192 && work <= 16384) return 8;
    return n <= 16384 && work <= 36864 ? 16 : 32;
}

// Whether the sums of a sorted batch are launches that can be made.
bool sums_launchable(int64_t n, int64_t dim)
{
    const int64_t slabs = ceil_div(dim, kSlab), units = ceil_div(n, chunk_size(n, dim)) * slabs;
    return slabs <= 65535 && launchable(ceil_div(units, kThreads / kWave), kThreads);
}

// Short batches are not sorted. One launch against the sort's three: 100 tokens into 32000 x 256
// 10.0 us and 16.9, 600 into 5003 x 1000 10.1 and 17.2; but 600 into 32000 x 4096 49 and 44, 1500 of
// one token 35 and 22.
bool few_tokens(int64_t n, int64_t dim) { return n > 0 && n <= (dim <= 2 * kSlab ? kFewMost : kFewMost / 2); }

int key_bits(int64_t rows)
{
    int b = 1;
    while ((rows >> b) != 0) ++b;  // keys are 0 .. rows
    return b;
}

// How a call's tokens are sorted.
enum class Sort : int { RANK, MERGE, RADIX };

struct GradPlan {
    size_t key[2], pos[2], hist, part, total;
    int digits, bits, tiles, chunk;
    bool few, scan;
    Sort sort;
};

GradPlan plan_grad(int64_t n, int64_t rows, int64_t dim)
{
    GradPlan g{};
    const int kb = key_bits(rows);
    g.digits = (kb + 9) / 10;
    g.bits = std::max(2, (kb + g.digits - 1) / g.digits);  // (bins in groups of four)
    g.few = few_tokens(n, dim);
    g.tiles = (int)ceil_div(n, kTile);
    // One launch, two, or two to three for each digit. Measured, x 64 into 50000 rows: 4096
    // tokens RANK 23.3 us, MERGE 20.5; 6144 29.1 and 22.3; MERGE and RADIX: 16384 30 and 40, 32768 37
    // and 43, 65536 53 and 51 (x 256). With one digit RADIX has two launches as well: 6144 into 1000 rows
    // RANK 28.7, RADIX 22.9.
    g.sort = n <= 4096 ? Sort::RANK : n <= 49152 && g.digits > 1 ? Sort::MERGE : Sort::RADIX;
    // Beyond, a launch of its own adds the tiles' counts up, which otherwise every tile does for
    // itself: 65536 x 64 into 50000 rows 52 us so and 50 not, 131072 x 64 61 and 67, 4 M x 64
    // 591 and 2507.
    g.scan = g.tiles > 96;
    g.chunk = chunk_size(n, dim);
    if (g.few || n == 0) return g;
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
    g.hist = take(g.sort == Sort::RADIX ? ((size_t)(g.tiles + g.scan) << g.bits) * 4 : 0);
    g.part = take((size_t)ceil_div(n, g.chunk) * 2 * (size_t)dim * 4);
    g.total = at;
    return g;
}

int embed_grad_sizes(int64_t n, int64_t rows, int64_t dim)
{
    if (n < 0 || rows < 1 || dim < 1) return HIMUON_ERR_INVALID_ARG;
    if (n > INT32_MAX / 2 || rows >= INT32_MAX || dim > INT32_MAX - 1024) return HIMUON_ERR_UNSUPPORTED;
    if (n > 0 && !few_tokens(n, dim) && !sums_launchable(n, dim)) return HIMUON_ERR_UNSUPPORTED;
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
    if (g.total > 0 && (!workspace || workspace_bytes < g.total || ((uintptr_t)workspace & 15))) return HIMUON_ERR_WORKSPACE;
    if (n_tokens == 0 && accumulate) return HIMUON_OK;
    StreamDevice on(stream);
    if (on.status != HIMUON_OK) return on.status;
    const hipStream_t hs = static_cast<hipStream_t>(stream);
    uint8_t* const ws = static_cast<uint8_t*>(workspace);

    SumArgs p{};
    p.grad = grad;
    p.out = dtable;
    p.rows = n_rows;
    p.ld_grad = ld_grad;
    p.ld_out = ld_dtable;
    p.n = (int32_t)n_tokens;
    p.dim = (int32_t)dim;
    p.slabs = (int32_t)ceil_div(dim, kSlab);
    p.accumulate = accumulate != 0;
    p.scale = scale;
    SortArgs s{};
    s.tokens = tokens;
    s.hist = reinterpret_cast<uint32_t*>(ws + g.hist);
    s.rows = n_rows;
    s.n = (int32_t)n_tokens;
    s.wide = index == HIMUON_I64;
    s.tiles = g.tiles;
    s.bits = g.bits;
    s.scanned = g.scan;
    if (g.few) {
        FewArgs f{};
        s.first = 1;
        f.sort = s;
        f.sum = p;
        f.out = static_cast<uint8_t*>(dtable);
        f.row_bytes = dim * dtype_size(out_dtype);
        f.ld_bytes = ld_dtable * dtype_size(out_dtype);
        f.fill_rows = (int32_t)std::max<int64_t>(1, std::min<int64_t>(4096, 65536 / f.row_bytes));
        f.share = (int32_t)ceil_div(n_tokens, kFewWaves);
        if (dtype == HIMUON_BF16)
            return out_dtype == HIMUON_BF16 ? launch_few<GemmStore::BF16, GemmStore::BF16>(f, hs)
                                            : launch_few<GemmStore::BF16, GemmStore::F32>(f, hs);
        return out_dtype == HIMUON_BF16 ? launch_few<GemmStore::F32, GemmStore::BF16>(f, hs)
                                        : launch_few<GemmStore::F32, GemmStore::F32>(f, hs);
    }
    s.fill.out = static_cast<uint8_t*>(dtable);
    s.fill.row_bytes = dim * dtype_size(out_dtype);
    s.fill.ld_bytes = ld_dtable * dtype_size(out_dtype);
    // Zeros go past the caches where the rows to be summed are many enough to be worth their
    // place there. 16384 x 4096 (134 MB) into 32000 rows 85 us so, 100 not; 32768 x 2048
    // into 50000 of fp32 115 and 141; but 4096 x 2560 (21 MB) into 32000 46 and 37, 2000 x
    // 4096 (16 MB) 60 and 47.
    s.fill.stream = n_tokens * dim * dtype_size(dtype) >= (INT64_C(64) << 20);
    // launch `part` of `parts` of the sort, `blocks` blocks of its own and those that fill
    auto with_fill = [&](int64_t part, int64_t parts, int64_t blocks, int threads) -> dim3 {
        s.fill.from = n_rows * part / parts;
        s.fill.to = n_rows * (part + 1) / parts;
        s.fill.first = (int32_t)blocks;
        s.fill.blocks = 0;
        if (!accumulate)  // (a block fills about 64 bytes a thread and round)
            s.fill.blocks = (int32_t)std::min<int64_t>(ceil_div((s.fill.to - s.fill.from) * s.fill.row_bytes, threads * 64), 1 << 20);
        return dim3((unsigned)(blocks + s.fill.blocks));
    };
    auto from_to = [&](int from, int to) {
        s.key_in = reinterpret_cast<const uint32_t*>(ws + g.key[from]);
        s.pos_in = reinterpret_cast<const uint32_t*>(ws + g.pos[from]);
        s.key_out = reinterpret_cast<uint32_t*>(ws + g.key[to]);
        s.pos_out = reinterpret_cast<uint32_t*>(ws + g.pos[to]);
    };
    int from = 0;
    if (g.sort == Sort::RANK) {
        s.first = 1;
        s.groups = INT32_MAX;
        from_to(1, 0);
        const dim3 grid = with_fill(0, 1, ceil_div(n_tokens, kWave), kRankThreads);
        hipLaunchKernelGGL(sort_rank<kRankThreads>, grid, dim3(kRankThreads), 0, hs, s);
        const int st = launch_status();
        if (st != HIMUON_OK || n_tokens == 0) return st;
    } else if (g.sort == Sort::MERGE) {
        // Blocks of 512 threads place their entries sooner, blocks of 256 are better at setting
        // rows to zero: 16384 x 1024 into 32000 rows (66 MB) of bf16 36.7 us and 41.0, 32768 x 2560 into
        // 50000 (256 MB) 96.1 and 92.6, x 2048 of fp32 (410 MB) 121.0 and 115.5.
        const bool narrow = !accumulate && n_rows * s.fill.row_bytes >= (INT64_C(200) << 20);
        const int threads = narrow ? 256 : 512;
        const int64_t blocks = ceil_div(n_tokens, kWave);
        s.first = 1;
        s.groups = kPart / kWave;
        from_to(1, 0);
        dim3 grid = with_fill(0, 2, blocks, threads);
        if (narrow) hipLaunchKernelGGL(sort_rank<256>, grid, dim3(256), 0, hs, s);
        else hipLaunchKernelGGL(sort_rank<512>, grid, dim3(512), 0, hs, s);
        int st = launch_status();
        if (st != HIMUON_OK) return st;
        from_to(0, 1);
        from = 1;
        grid = with_fill(1, 2, blocks, threads);
        if (narrow) hipLaunchKernelGGL(sort_merge<256>, grid, dim3(256), 0, hs, s);
        else hipLaunchKernelGGL(sort_merge<512>, grid, dim3(512), 0, hs, s);
        st = launch_status();
        if (st != HIMUON_OK) return st;
    } else {
        for (int d = 0; d < g.digits; ++d) {
            s.first = d == 0;
            s.shift = d * g.bits;
            from_to(from, from ^ 1);
            from ^= 1;
            dim3 grid = with_fill(2 * d, 2 * g.digits, g.tiles, kThreads);
            hipLaunchKernelGGL(sort_count, grid, dim3(kThreads), 0, hs, s);
            int st = launch_status();
            if (st != HIMUON_OK) return st;
            if (g.scan) {
                hipLaunchKernelGGL(sort_scan, dim3((unsigned)ceil_div(INT64_C(1) << g.bits, kWave)), dim3(kScanThreads), 0, hs, s);
                st = launch_status();
                if (st != HIMUON_OK) return st;
            }
            grid = with_fill(2 * d + 1, 2 * g.digits, g.tiles, kThreads);
            hipLaunchKernelGGL(sort_scatter, grid, dim3(kThreads), 0, hs, s);
            st = launch_status();
            if (st != HIMUON_OK) return st;
        }
    }
    p.key = reinterpret_cast<const uint32_t*>(ws + g.key[from]);
    p.pos = reinterpret_cast<const uint32_t*>(ws + g.pos[from]);
    p.part = reinterpret_cast<float*>(ws + g.part);
    if (dtype == HIMUON_BF16)
        return out_dtype == HIMUON_BF16 ? launch_sums_t<GemmStore::BF16, GemmStore::BF16>(p, g.chunk, hs)
                                        : launch_sums_t<GemmStore::BF16, GemmStore::F32>(p, g.chunk, hs);
    return out_dtype == HIMUON_BF16 ? launch_sums_t<GemmStore::F32, GemmStore::BF16>(p, g.chunk, hs)
                                    : launch_sums_t<GemmStore::F32, GemmStore::F32>(p, g.chunk, hs);
}
