// The residual's addition with the norm of the sum, and the backward pass (himuon_add_norm,
// himuon_add_norm_grad).
//
// For a row of D elements, h = x + residual, r = (mean h^2 + eps)^(-1/2), gain w:
//     y = h r w
//     dh = g_h + r (g_y w - h r mean(g_y w h r)),   dw = sum over rows of g_y h r
// Memory bounds both: every array is read or written once (16384 x 4096 bf16: 105 us forward, 5.1 TB/s, and 110
// backward with the gain's 7; a copy of 2 GiB runs at 4.9); few rows the host (32 x 4096: 4.4 us of 10.8). A row is held in registers by a
// wave or by a block of four (rows of more than 1024 elements), which walks over rows with the
// gain, and in the backward pass the sums of its gradient, in registers too. A row's sums
// are its waves' in their order.
#include "elementwise8.h"
#include "train_ops.h"

#include <algorithm>
#include <cmath>

namespace himuon {
namespace {

constexpr int kThreads = 256;

struct NormArgs {
    const void *x, *res, *gain, *gy, *gh;
    void *h, *y;
    float* part;
    int64_t ldx, ldr, ldh, ldy, ldgy, ldgh, rows;
    int32_t width, units;
    float eps;
    double inv_width;
};

// A lane's chunks of eight elements of a row: NT lanes hold it, C chunks each.
template <int NT> __device__ __forceinline__ int chunk_at(int lane, int c) { return 8 * (lane + NT * c); }
__device__ __forceinline__ int chunk_size(int width, int at) { return width - at >= 8 ? 8 : width > at ? width - at : 0; }

template <GemmStore ST> __device__ __forceinline__ f32x8 get8n(const void* base, int64_t i, int n)
{
    const Raw8<ST> r = get_raw8<ST>(base, i, n);
    f32x8 v;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = raw_value<ST>(r, e);
    return v;
}

template <GemmStore ST> __device__ __forceinline__ void put8n(void* base, int64_t i, int n, f32x8 x)
{
    if (n == 8) {
        put8<ST>(base, i, x);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n) put1<ST>(base, i + e, x[e]);
    }
}

// The sum over a row's NT lanes, in every one of them. `slot` alternates from row to row.
// (Sums over rows are in 64 bits, which memory hides: r is then off by half a step of 32 bits, y's roundings
// to 16 and 8 bits fall where the definition's do, and rows whose squares leave fp32's range keep r and
// their gradient.)
template <int NT> __device__ __forceinline__ double row_sum(double v, double (*sums)[kThreads / 64], int slot)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    if constexpr (NT > 64) {
        if ((threadIdx.x & 63) == 0) sums[slot][threadIdx.x >> 6] = v;
        __syncthreads();
        v = (sums[slot][0] + sums[slot][1]) + (sums[slot][2] + sums[slot][3]);
    }
    return v;
}

// (mean + eps)^(-1/2) of a row's sum of squares.
__device__ __forceinline__ float scale_of(double sum, const NormArgs& p) { return (float)(1.0 / sqrt(sum / (double)p.width + (double)p.eps)); }

// r of a row and mean(g_y w h r), from its sums of h^2 and of g_y w h. (h r and that mean are of the gradients'
// size whatever h's is. An estimate of 2^-23 and a step of Newton's, which takes it to 2^-44: a division and
// a root of 64 bits would cost the registers of a wave. A row with an infinite element has r = 0, and adds nothing to the
// other columns' dw.)
struct RowTerms {
    float r, mean;
    __device__ __forceinline__ RowTerms(double s, double t, const NormArgs& p)
    {
        const double x = fma(s, p.inv_width, (double)p.eps), y = __builtin_amdgcn_rsq(x);
        const double root = x > 0.0 && x < INFINITY ? y * fma(-0.5 * x * y, y, 1.5) : y;
        r = (float)root;
        mean = (float)(t * root * p.inv_width);
    }
};

template <GemmStore ST, GemmStore GT, int NT, int C> __global__ void __launch_bounds__(kThreads) add_norm(const NormArgs p)
{
    __shared__ double sums[2][kThreads / 64];
    constexpr int R = kThreads / NT;
    const int lane = threadIdx.x % NT;
    const int unit = blockIdx.x * R + threadIdx.x / NT;
    f32x8 w[C];
    int n[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        n[c] = chunk_size(p.width, chunk_at<NT>(lane, c));
        w[c] = n[c] > 0 ? get8n<GT>(p.gain, chunk_at<NT>(lane, c), n[c]) : f32x8{};
    }
    int slot = 0;
    for (int64_t row = unit; row < p.rows; row += p.units, slot ^= 1) {
        f32x8 v[C];
#pragma unroll
        for (int c = 0; c < C; ++c) v[c] = n[c] > 0 ? get8n<ST>(p.x, row * p.ldx + chunk_at<NT>(lane, c), n[c]) : f32x8{};
        if (p.res) {
#pragma unroll
            for (int c = 0; c < C; ++c)
                if (n[c] > 0) v[c] += get8n<ST>(p.res, row * p.ldr + chunk_at<NT>(lane, c), n[c]);
        }
        double s = 0.0;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e) s = fma((double)v[c][e], (double)v[c][e], s);
        const float r = scale_of(row_sum<NT>(s, sums, slot), p);
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if (n[c] > 0) {
                if (p.res) put8n<ST>(p.h, row * p.ldh + chunk_at<NT>(lane, c), n[c], v[c]);
                put8n<ST>(p.y, row * p.ldy + chunk_at<NT>(lane, c), n[c], v[c] * r * w[c]);
            }
        }
    }
}

// (All of a launch's 1024 blocks are on the chip at once while a row has at most 4096 elements: four to a CU. With three of
// them 16384 x 4096 bf16 takes 171 us, not 113.)
template <GemmStore ST, GemmStore GT, int NT, int C> __global__ void __launch_bounds__(kThreads, (C <= 2 ? 4 : C == 4 ? 2 : 1)) add_norm_grad(const NormArgs p)
{
    __shared__ double sums[4][kThreads / 64];
    __shared__ float join[NT == 64 ? kThreads * C * 8 : 1];
    constexpr int R = kThreads / NT;
    const int lane = threadIdx.x % NT;
    const int unit = blockIdx.x * R + (R == 1 ? 0 : threadIdx.x / NT);
    f32x8 w[C], dw[C];
    int n[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        n[c] = chunk_size(p.width, chunk_at<NT>(lane, c));
        w[c] = n[c] > 0 ? get8n<GT>(p.gain, chunk_at<NT>(lane, c), n[c]) : f32x8{};
        dw[c] = f32x8{};
    }
    int slot = 0;
    for (int64_t row = unit; row < p.rows; row += p.units, slot ^= 2) {
        f32x8 h[C], g[C], a[C];
#pragma unroll
        for (int c = 0; c < C; ++c) {
            h[c] = n[c] > 0 ? get8n<ST>(p.h, row * p.ldh + chunk_at<NT>(lane, c), n[c]) : f32x8{};
            g[c] = n[c] > 0 ? get8n<ST>(p.gy, row * p.ldgy + chunk_at<NT>(lane, c), n[c]) : f32x8{};
            a[c] = p.gh && n[c] > 0 ? get8n<ST>(p.gh, row * p.ldgh + chunk_at<NT>(lane, c), n[c]) : f32x8{};
        }
        double s = 0.0, t = 0.0;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                s = fma((double)h[c][e], (double)h[c][e], s);
                t = fma((double)(g[c][e] * w[c][e]), (double)h[c][e], t);
                asm volatile("" : "+v"(s), "+v"(t));  // (one after the other: conversions ahead of them cost a wave's registers)
            }
        s = row_sum<NT>(s, sums, slot);
        t = row_sum<NT>(t, sums, slot + 1);
        const RowTerms f(s, t, p);
#pragma unroll
        for (int c = 0; c < C; ++c) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float n = h[c][e] * f.r;
                dw[c][e] = fmaf(g[c][e], n, dw[c][e]);
                a[c][e] = fmaf(f.r, fmaf(-n, f.mean, g[c][e] * w[c][e]), a[c][e]);
            }
            if (n[c] > 0) put8n<ST>(p.y, row * p.ldy + chunk_at<NT>(lane, c), n[c], a[c]);
        }
    }
    float* const out = p.part + (int64_t)blockIdx.x * p.width;
    if constexpr (NT == 64) {
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e) join[(c * 8 + e) * kThreads + threadIdx.x] = dw[c][e];
        __syncthreads();
        for (int i = threadIdx.x; i < 64 * C * 8; i += kThreads) {
            const int l = i & 63, ce = i >> 6, at = chunk_at<64>(l, ce >> 3) + (ce & 7);
            const float* const from = join + ce * kThreads + l;
            if (at < p.width) out[at] = (from[0] + from[64]) + (from[128] + from[192]);
        }
    } else {
#pragma unroll
        for (int c = 0; c < C; ++c)
            if (n[c] > 0) put8n<GemmStore::F32>(out, chunk_at<NT>(lane, c), n[c], dw[c]);
    }
}

// Rows that registers do not hold: a block reads each of them twice.
template <GemmStore ST, GemmStore GT> __global__ void __launch_bounds__(kThreads) add_norm_long(const NormArgs p)
{
    __shared__ double sums[2][kThreads / 64];
    int slot = 0;
    for (int64_t row = blockIdx.x; row < p.rows; row += p.units, slot ^= 1) {
        auto sum = [&](int at, int n) {
            f32x8 v = get8n<ST>(p.x, row * p.ldx + at, n);
            if (p.res) v += get8n<ST>(p.res, row * p.ldr + at, n);
            return v;
        };
        double s = 0.0;
        for (int at = 8 * threadIdx.x; at < p.width; at += 8 * kThreads) {
            const f32x8 v = sum(at, chunk_size(p.width, at));
#pragma unroll
            for (int e = 0; e < 8; ++e) s = fma((double)v[e], (double)v[e], s);
        }
        const float r = scale_of(row_sum<kThreads>(s, sums, slot), p);
        for (int at = 8 * threadIdx.x; at < p.width; at += 8 * kThreads) {
            const int n = chunk_size(p.width, at);
            const f32x8 v = sum(at, n), w = get8n<GT>(p.gain, at, n);
            if (p.res) put8n<ST>(p.h, row * p.ldh + at, n, v);
            put8n<ST>(p.y, row * p.ldy + at, n, v * r * w);
        }
    }
}

// The gain's gradient goes to `part` as its own blocks' sums: they are read and written there.
template <GemmStore ST, GemmStore GT> __global__ void __launch_bounds__(kThreads) add_norm_grad_long(const NormArgs p)
{
    __shared__ double sums[4][kThreads / 64];
    float* const out = p.part + (int64_t)blockIdx.x * p.width;
    for (int at = 8 * threadIdx.x; at < p.width; at += 8 * kThreads) put8n<GemmStore::F32>(out, at, chunk_size(p.width, at), f32x8{});
    int slot = 0;
    for (int64_t row = blockIdx.x; row < p.rows; row += p.units, slot ^= 2) {
        double s = 0.0, t = 0.0;
        for (int at = 8 * threadIdx.x; at < p.width; at += 8 * kThreads) {
            const int n = chunk_size(p.width, at);
            const f32x8 h = get8n<ST>(p.h, row * p.ldh + at, n), g = get8n<ST>(p.gy, row * p.ldgy + at, n), w = get8n<GT>(p.gain, at, n);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                s = fma((double)h[e], (double)h[e], s);
                t = fma((double)(g[e] * w[e]), (double)h[e], t);
            }
        }
        s = row_sum<kThreads>(s, sums, slot);
        t = row_sum<kThreads>(t, sums, slot + 1);
        const RowTerms f(s, t, p);
        for (int at = 8 * threadIdx.x; at < p.width; at += 8 * kThreads) {
            const int n = chunk_size(p.width, at);
            const f32x8 h = get8n<ST>(p.h, row * p.ldh + at, n), g = get8n<ST>(p.gy, row * p.ldgy + at, n), w = get8n<GT>(p.gain, at, n);
            f32x8 a = p.gh ? get8n<ST>(p.gh, row * p.ldgh + at, n) : f32x8{}, d = get8n<GemmStore::F32>(out, at, n);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float n = h[e] * f.r;
                d[e] = fmaf(g[e], n, d[e]);
                a[e] = fmaf(f.r, fmaf(-n, f.mean, g[e] * w[e]), a[e]);
            }
            put8n<GemmStore::F32>(out, at, n, d);
            put8n<ST>(p.y, row * p.ldy + at, n, a);
        }
    }
}

// The blocks' sums of 16 columns, the blocks shared out over 64 groups of 16 lanes.
constexpr int kSumThreads = 1024, kSumCols = 16;
template <GemmStore GT> __global__ void __launch_bounds__(kSumThreads) norm_gain_sums(const float* part, int rows, int width, void* dgain)
{
    constexpr int R = kSumThreads / kSumCols;
    __shared__ float sums[R][kSumCols + 1];
    const int x = threadIdx.x % kSumCols, group = threadIdx.x / kSumCols;
    const int col = blockIdx.x * kSumCols + x;
    float v[4] = {};
    if (col < width) {
        for (int r = group; r < rows; r += 4 * R) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float f = part[(int64_t)min(r + j * R, rows - 1) * width + col];
                v[j] += r + j * R < rows ? f : 0.f;
            }
        }
    }
    sums[group][x] = (v[0] + v[1]) + (v[2] + v[3]);
    __syncthreads();
    if (group >= 4) return;  // 16 rows to each of the first wave's four groups
    float t = 0.f;
#pragma unroll
    for (int r = 0; r < R / 4; ++r) t += sums[group * (R / 4) + r][x];
    t += __shfl_xor(t, 16);
    t += __shfl_xor(t, 32);
    if (group == 0 && col < width) put1<GT>(dgain, col, t);
}

// ---------------------------------------------------------------- host side

constexpr int64_t kMostWidth = INT64_C(1) << 26;
constexpr int kLongWidth = 8 * kThreads * 8;  // the widest row in registers

// Blocks of a call: units of one row (a wave's or a block's) that walk over the rows. Half as many / these / twice as
// many, us: forward bf16 16384 x 4096 105 / 109 / 108, x 1000 21.9 / 22.1 / 23.8, 4096 x 4096 22.2 / 22.5 / 24.0; backward bf16 16384 x
// 4096 140 / 109 / 115, x 2048 97 / 63 / 68, x 640 28 / 22.5 / 27, fp32 4096 x 4096 52 / 55 / 64.
int64_t norm_blocks(int64_t rows, int64_t width, bool grad)
{
    const int64_t per = width <= 1024 ? kThreads / 64 : 1;
    return std::max<int64_t>(1, std::min<int64_t>(ceil_div(rows, per), grad ? 1024 : 2048));
}

template <bool GRAD, GemmStore ST, GemmStore GT> int launch_norm(NormArgs p, hipStream_t stream)
{
    const int64_t blocks = norm_blocks(p.rows, p.width, GRAD);
    p.units = (int32_t)blocks * (p.width <= 1024 ? kThreads / 64 : 1);
    const dim3 grid((unsigned)blocks), block(kThreads);
#define HM_NORM(NT, C)                                                                              \
    do {                                                                                            \
        if constexpr (GRAD) hipLaunchKernelGGL((add_norm_grad<ST, GT, NT, C>), grid, block, 0, stream, p); \
        else hipLaunchKernelGGL((add_norm<ST, GT, NT, C>), grid, block, 0, stream, p);              \
    } while (0)
    if (p.width <= 512) HM_NORM(64, 1);
    else if (p.width <= 1024) HM_NORM(64, 2);
    else if (p.width <= 2048) HM_NORM(256, 1);
    else if (p.width <= 4096) HM_NORM(256, 2);
    else if (p.width <= 8192) HM_NORM(256, 4);
    else if (p.width <= kLongWidth) HM_NORM(256, 8);
    else if constexpr (GRAD) hipLaunchKernelGGL((add_norm_grad_long<ST, GT>), grid, block, 0, stream, p);
    else hipLaunchKernelGGL((add_norm_long<ST, GT>), grid, block, 0, stream, p);
#undef HM_NORM
    return launch_status();
}

template <bool GRAD> int launch_types(const NormArgs& p, int dtype, int gain, hipStream_t stream)
{
    if (dtype == HIMUON_BF16)
        return gain == HIMUON_BF16 ? launch_norm<GRAD, GemmStore::BF16, GemmStore::BF16>(p, stream)
                                   : launch_norm<GRAD, GemmStore::BF16, GemmStore::F32>(p, stream);
    return gain == HIMUON_BF16 ? launch_norm<GRAD, GemmStore::F32, GemmStore::BF16>(p, stream)
                               : launch_norm<GRAD, GemmStore::F32, GemmStore::F32>(p, stream);
}

int check_norm(int64_t rows, int64_t width, const void* gain, int gain_dtype, float eps, int dtype)
{
    if (rows < 0 || width < 1 || !gain || !known_dtype(dtype) || !known_dtype(gain_dtype) || !(eps >= 0.f) || !std::isfinite(eps))
        return HIMUON_ERR_INVALID_ARG;
    if (rows > INT32_MAX || width > kMostWidth) return HIMUON_ERR_UNSUPPORTED;
    return HIMUON_OK;
}

// A matrix of the call: its leading dimension, and that its last element has an index.
bool fits(int64_t rows, int64_t width, int64_t ld) { return ld >= width && small_product(rows, ld); }

}  // namespace
}  // namespace himuon

extern "C" int himuon_add_norm(int64_t n_tokens, int64_t width, const void* x, int64_t ld_x, const void* residual, int64_t ld_residual,
                               const void* gain, int gain_dtype, void* h, int64_t ld_h, void* y, int64_t ld_y, void* codes,
                               void* exponents, float eps, int dtype, void* stream)
{
    using namespace himuon;
    const int st = check_norm(n_tokens, width, gain, gain_dtype, eps, dtype);
    if (st != HIMUON_OK) return st;
    if (!codes != !exponents || ((uintptr_t)codes & 15)) return HIMUON_ERR_INVALID_ARG;
    if (!fits(n_tokens, width, ld_x) || !fits(n_tokens, width, ld_y) ||
        (residual && (!fits(n_tokens, width, ld_residual) || !fits(n_tokens, width, ld_h))))
        return HIMUON_ERR_INVALID_ARG;
    if (n_tokens == 0) return HIMUON_OK;
    if (!x || !y || (residual && (!h || h == y))) return HIMUON_ERR_INVALID_ARG;
    if (codes && n_tokens > INT64_C(1) << 29) return HIMUON_ERR_UNSUPPORTED;
    StreamDevice on(stream);
    if (on.status != HIMUON_OK) return on.status;
    NormArgs p{};
    p.x = x;
    p.res = residual;
    p.gain = gain;
    p.h = h;
    p.y = y;
    p.ldx = ld_x;
    p.ldr = ld_residual;
    p.ldh = ld_h;
    p.ldy = ld_y;
    p.rows = n_tokens;
    p.width = (int32_t)width;
    p.eps = eps;
    p.inv_width = 1.0 / (double)width;
    const int status = launch_types<false>(p, dtype, gain_dtype, static_cast<hipStream_t>(stream));
    if (status != HIMUON_OK || !codes) return status;
    return himuon_act_pack(n_tokens, width, y, ld_y, dtype, codes, exponents, stream);
}

extern "C" size_t himuon_add_norm_grad_workspace_size(int64_t n_tokens, int64_t width)
{
    using namespace himuon;
    if (n_tokens < 0 || width < 1 || n_tokens > INT32_MAX || width > kMostWidth) return 0;
    return round_up((size_t)norm_blocks(n_tokens, width, true) * (size_t)width * sizeof(float), 256);
}

extern "C" int himuon_add_norm_grad(int64_t n_tokens, int64_t width, const void* g_y, int64_t ld_g_y, const void* g_h, int64_t ld_g_h,
                                    const void* h, int64_t ld_h, const void* gain, int gain_dtype, void* dh, int64_t ld_dh,
                                    void* dgain, float eps, int dtype, void* workspace, size_t workspace_bytes, void* stream)
{
    using namespace himuon;
    const int st = check_norm(n_tokens, width, gain, gain_dtype, eps, dtype);
    if (st != HIMUON_OK) return st;
    if (!dgain) return HIMUON_ERR_INVALID_ARG;
    if (!fits(n_tokens, width, ld_g_y) || !fits(n_tokens, width, ld_h) || !fits(n_tokens, width, ld_dh) ||
        (g_h && !fits(n_tokens, width, ld_g_h)))
        return HIMUON_ERR_INVALID_ARG;
    // (without a row there is nothing to read: the gain's gradient becomes zero)
    if (n_tokens > 0 && (!g_y || !h || !dh)) return HIMUON_ERR_INVALID_ARG;
    if (!workspace || ((uintptr_t)workspace & 15) || workspace_bytes < himuon_add_norm_grad_workspace_size(n_tokens, width))
        return HIMUON_ERR_WORKSPACE;
    StreamDevice on(stream);
    if (on.status != HIMUON_OK) return on.status;
    NormArgs p{};
    p.gy = g_y;
    p.gh = g_h;
    p.gain = gain;
    p.h = const_cast<void*>(h);
    p.y = dh;
    p.part = static_cast<float*>(workspace);
    p.ldgy = ld_g_y;
    p.ldgh = ld_g_h;
    p.ldh = ld_h;
    p.ldy = ld_dh;
    p.rows = n_tokens;
    p.width = (int32_t)width;
    p.eps = eps;
    p.inv_width = 1.0 / (double)width;
    const hipStream_t hs = static_cast<hipStream_t>(stream);
    const int status = launch_types<true>(p, dtype, gain_dtype, hs);
    if (status != HIMUON_OK) return status;
    const int rows = (int)norm_blocks(n_tokens, width, true);
    const dim3 grid((unsigned)ceil_div(width, kSumCols));
    if (gain_dtype == HIMUON_BF16)
        hipLaunchKernelGGL(norm_gain_sums<GemmStore::BF16>, grid, dim3(kSumThreads), 0, hs, p.part, rows, (int)width, dgain);
    else
        hipLaunchKernelGGL(norm_gain_sums<GemmStore::F32>, grid, dim3(kSumThreads), 0, hs, p.part, rows, (int)width, dgain);
    return launch_status();
}
