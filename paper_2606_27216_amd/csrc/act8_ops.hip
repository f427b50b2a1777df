// Activations in 8 bits (himuon_act_pack, himuon_act_unpack) and the weight gradient
// that reads them (himuon_weight_grad).
//
// 32 tokens of a column share an exponent e, the least with max |x| <= 448 2^e; codes
// are 8-bit floats with 3 mantissa bits, so code * 2^e has 4 significant bits and is exact
// in bf16. A group lies along the weight gradient's sum, and a column's 32 codes are
// adjacent: they are the operand of 32 consecutive terms as they stand in memory.
#include "ns_device.h"
#include "train_ops.h"

#include <algorithm>

namespace himuon {
namespace {

using namespace dev;

constexpr int kThreads = 256;
constexpr int kGroup = HIMUON_ACT_GROUP;
constexpr uint32_t kMinCode = 27, kMaxCode = 246;  // exponent bytes of -100 and 119

typedef uint32_t u32_any8 __attribute__((aligned(1)));

// ------------------------------------------------------------ pack and unpack

// Columns of a lane: 8 bytes of a row.
template <GemmStore ST> constexpr int kCols = ST == GemmStore::BF16 ? 4 : 2;

// 8 bytes of a row from element i on, of which the first n elements exist.
template <GemmStore ST> __device__ __forceinline__ u32x2 load_cols(const void* x, int64_t i, int n)
{
    if constexpr (ST == GemmStore::BF16) {
        const uint16_t* const p = static_cast<const uint16_t*>(x) + i;
        if (n == 4) return *reinterpret_cast<const u32x2_any16*>(p);
        const uint32_t a = p[0], b = n > 1 ? p[1] : 0, c = n > 2 ? p[2] : 0;
        return u32x2{a | b << 16, c};
    } else {
        typedef u32x2 u32x2_any32 __attribute__((aligned(4)));
        const uint32_t* const p = static_cast<const uint32_t*>(x) + i;
        if (n == 2) return *reinterpret_cast<const u32x2_any32*>(p);
        return u32x2{p[0], 0u};
    }
}

// The bits of column j of a row as fp32.
template <GemmStore ST> __device__ __forceinline__ uint32_t col_bits(u32x2 w, int j)
{
    if constexpr (ST == GemmStore::BF16) return (j & 1) ? (w[j >> 1] & 0xffff0000u) : (w[j >> 1] << 16);
    else return w[j];
}

constexpr uint32_t kInf = 0x7f800000u;

// A wave takes 32 tokens of 64 lanes' columns; a lane quantises its columns one by one.
template <GemmStore ST>
__global__ void __launch_bounds__(kThreads) act_pack(const void* x, int64_t ld, int64_t tokens, int64_t cols, int64_t slabs,
                                                     int64_t units, uint8_t* codes, uint8_t* exps)
{
    constexpr int N = kCols<ST>;
    const int64_t unit = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
    if (unit >= units) return;
    const int64_t tb = unit / slabs;
    const int64_t c = (unit - tb * slabs) * (64 * N) + (threadIdx.x & 63) * N;
    if (c >= cols) return;
    const int n = (int)min((int64_t)N, cols - c);
    const int64_t t0 = tb * kGroup;
    const int rows = (int)min((int64_t)kGroup, tokens - t0);
    u32x2 raw[kGroup];
#pragma unroll
    for (int r = 0; r < kGroup; ++r) {
        const u32x2 w = load_cols<ST>(x, (t0 + min(r, rows - 1)) * ld + c, n);
        raw[r] = r < rows ? w : u32x2{0u, 0u};
    }
#pragma unroll
    for (int j = 0; j < N; ++j) {
        uint32_t top = 0;
#pragma unroll
        for (int r = 0; r < kGroup; ++r) top = max(top, col_bits<ST>(raw[r], j) & 0x7fffffffu);
        bool odd = false;  // something is not finite, or may exceed the largest code
        if (top >= kInf) {
            odd = true;
            top = 0;
#pragma unroll
            for (int r = 0; r < kGroup; ++r) {
                const uint32_t a = col_bits<ST>(raw[r], j) & 0x7fffffffu;
                top = a < kInf ? max(top, a) : top;
            }
        }
        // exponent field - 8, one more above 1.75 times a power of two
        const int e = (int)(top >> 23) - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
        const uint32_t code = (uint32_t)min(max(e, (int)kMinCode), (int)kMaxCode);
        odd = odd || code == kMaxCode;
        const float unit_inv = __uint_as_float((254u - code) << 23);
        uint32_t q[kGroup / 4];
        if (!odd) {
#pragma unroll
            for (int r = 0; r < kGroup; r += 4) {
                float v[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] = __uint_as_float(col_bits<ST>(raw[r + k], j)) * unit_inv;
                int w = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], 0, false);
                q[r / 4] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], w, true);
            }
        } else {
#pragma unroll
            for (int r = 0; r < kGroup; r += 4) {
                uint32_t d = 0;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const uint32_t b = col_bits<ST>(raw[r + k], j);
                    const float f = fminf(fmaxf(__uint_as_float(b) * unit_inv, -448.f), 448.f);
                    const uint32_t h = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f, f, 0, false) & 0xffu;
                    d |= ((b & 0x7fffffffu) >= kInf ? 0x7fu : h) << (8 * k);
                }
                q[r / 4] = d;
            }
        }
        if (j < n) {
            u32x4* const dst = reinterpret_cast<u32x4*>(codes + (tb * cols + c + j) * kGroup);
            dst[0] = u32x4{q[0], q[1], q[2], q[3]};
            dst[1] = u32x4{q[4], q[5], q[6], q[7]};
            exps[tb * cols + c + j] = (uint8_t)code;
        }
    }
}

// Two columns to a lane, 32 tokens.
template <GemmStore ST>
__global__ void __launch_bounds__(kThreads) act_unpack(const uint8_t* codes, const uint8_t* exps, int64_t tokens, int64_t cols,
                                                       int64_t slabs, int64_t units, void* x, int64_t ld)
{
    constexpr int N = 2;
    const int64_t unit = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
    if (unit >= units) return;
    const int64_t tb = unit / slabs;
    const int64_t c = (unit - tb * slabs) * (64 * N) + (threadIdx.x & 63) * N;
    if (c >= cols) return;
    const int n = (int)min((int64_t)N, cols - c);
    const int64_t t0 = tb * kGroup;
    const int rows = (int)min((int64_t)kGroup, tokens - t0);
    u32x4 q[N][2];
    float scale[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const int64_t g = tb * cols + c + min(j, n - 1);
        const u32x4* const src = reinterpret_cast<const u32x4*>(codes + g * kGroup);
        q[j][0] = src[0];
        q[j][1] = src[1];
        scale[j] = __uint_as_float((uint32_t)exps[g] << 23);
    }
#pragma unroll
    for (int r = 0; r < kGroup; ++r) {
        float v[N];
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int w = (int)q[j][r / 16][(r / 4) % 4];
            const f32x2 f = (r & 2) ? __builtin_amdgcn_cvt_pk_f32_fp8(w, true) : __builtin_amdgcn_cvt_pk_f32_fp8(w, false);
            v[j] = f[r & 1] * scale[j];
        }
        if (r >= rows) continue;
        const int64_t i = (t0 + r) * ld + c;
        if constexpr (ST == GemmStore::BF16) {
            uint16_t* const p = static_cast<uint16_t*>(x) + i;  // (exact: the upper halves)
            if (n == 2) *reinterpret_cast<u32_any16*>(p) = __float_as_uint(v[0]) >> 16 | (__float_as_uint(v[1]) & 0xffff0000u);
            else p[0] = (uint16_t)(__float_as_uint(v[0]) >> 16);
        } else {
            float* const p = static_cast<float*>(x) + i;
            p[0] = v[0];
            if (n == 2) p[1] = v[1];
        }
    }
}

// ------------------------------------------------------------ weight gradient

struct WgradArgs {
    const void* grad;
    const uint8_t *codes, *exps;
    void* out;
    int64_t tokens, ld_grad, ld_out;
    int32_t rows, cols, accumulate;
};

// 64 x 64 tiles, 32 tokens at a time through LDS: the gradient's columns turned so that
// tokens are adjacent (fp32: three bf16 terms of eight bits each), the codes widened.
template <GemmStore ST, GemmStore OT> __global__ void __launch_bounds__(kThreads) wgrad_tile(const WgradArgs p)
{
    constexpr int TERMS = ST == GemmStore::F32 ? 3 : 1;
    constexpr int PITCH = 40;
    __shared__ __attribute__((aligned(16))) uint16_t sa[TERMS][64][PITCH];
    __shared__ __attribute__((aligned(16))) uint16_t sb[64][PITCH];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, li = lane & 31, lh = lane >> 5;
    const int wi = (wave >> 1) * 32, wj = (wave & 1) * 32;
    const int64_t o0 = (int64_t)blockIdx.y * 64, j0 = (int64_t)blockIdx.x * 64;
    f32x16 acc = {};
    for (int64_t t0 = 0; t0 < p.tokens; t0 += kGroup) {
        {
            const int t = tid >> 3, o = (tid & 7) * 8;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const bool on = t0 + t < p.tokens && o0 + o + e < p.rows;
                float v = on ? get1<ST>(p.grad, (t0 + t) * p.ld_grad + o0 + o + e) : 0.f;
#pragma unroll
                for (int k = 0; k < TERMS; ++k) {
                    const uint32_t top = __float_as_uint(v) & 0xffff0000u;
                    sa[k][o + e][t] = (uint16_t)(top >> 16);
                    v = (top & kInf) == kInf ? 0.f : v - __uint_as_float(top);
                }
            }
        }
        {
            const int j = tid >> 2, part = (tid & 3) * 8;
            const int64_t g = (t0 / kGroup) * p.cols + min(j0 + j, (int64_t)p.cols - 1);
            const u32x2 w = *reinterpret_cast<const u32x2*>(p.codes + g * kGroup + part);
            const float unit = __uint_as_float((uint32_t)p.exps[g] << 23);
            u32x4 h;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int d = (int)w[e >> 1];
                const f32x2 f = (e & 1) ? __builtin_amdgcn_cvt_pk_f32_fp8(d, true) : __builtin_amdgcn_cvt_pk_f32_fp8(d, false);
                h[e] = __float_as_uint(f[0] * unit) >> 16 | (__float_as_uint(f[1] * unit) & 0xffff0000u);
            }
            *reinterpret_cast<u32x4*>(&sb[j][part]) = h;
        }
        __syncthreads();
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const u32x4 b = *reinterpret_cast<const u32x4*>(&sb[wj + li][16 * s + 8 * lh]);
#pragma unroll
            for (int k = 0; k < TERMS; ++k)
                acc = mma1<Operand::BF16>(b, *reinterpret_cast<const u32x4*>(&sa[k][wi + li][16 * s + 8 * lh]), acc);
        }
        __syncthreads();
    }
    const int64_t o = o0 + wi + li;
    if (o >= p.rows) return;
#pragma unroll
    for (int v = 0; v < 16; ++v) {
        const int64_t j = j0 + wj + 8 * (v >> 2) + 4 * lh + (v & 3);
        if (j >= p.cols) continue;
        const int64_t i = o * p.ld_out + j;
        put1<OT>(p.out, i, p.accumulate ? acc[v] + get1<OT>(p.out, i) : acc[v]);
    }
}

int act_sizes(int64_t tokens, int64_t cols)
{
    if (tokens < 0 || cols < 1) return HIMUON_ERR_INVALID_ARG;
    if (tokens > INT32_MAX - 1024 || cols > INT32_MAX - 4096) return HIMUON_ERR_UNSUPPORTED;
    return HIMUON_OK;
}

int wgrad_sizes(int64_t tokens, int64_t out, int64_t cols)
{
    if (out < 1) return HIMUON_ERR_INVALID_ARG;
    if (out > INT32_MAX - 4096) return HIMUON_ERR_UNSUPPORTED;
    return act_sizes(tokens, cols);
}

template <GemmStore ST, GemmStore OT> int launch_wgrad(const WgradArgs& p, hipStream_t stream)
{
    const int64_t gy = ceil_div(p.rows, 64);
    if (gy > 65535) return HIMUON_ERR_UNSUPPORTED;
    hipLaunchKernelGGL((wgrad_tile<ST, OT>), dim3((unsigned)ceil_div(p.cols, 64), (unsigned)gy), dim3(kThreads), 0, stream, p);
    return launch_status();
}

}  // namespace
}  // namespace himuon

extern "C" int himuon_act_pack(int64_t n_tokens, int64_t cols, const void* x, int64_t ld, int dtype, void* codes,
                               void* exponents, void* stream)
{
    using namespace himuon;
    const int sizes = act_sizes(n_tokens, cols);
    if (sizes != HIMUON_OK) return sizes;
    if (!known_dtype(dtype) || ld < cols || !small_product(n_tokens, ld)) return HIMUON_ERR_INVALID_ARG;
    if (n_tokens == 0) return HIMUON_OK;
    if (!x || !codes || !exponents || ((uintptr_t)codes & 15)) return HIMUON_ERR_INVALID_ARG;
    StreamDevice on(stream);
    if (on.status != HIMUON_OK) return on.status;
    const hipStream_t hs = static_cast<hipStream_t>(stream);
    const int64_t slabs = ceil_div(cols, 64 * (dtype == HIMUON_BF16 ? kCols<GemmStore::BF16> : kCols<GemmStore::F32>));
    const int64_t units = ceil_div(n_tokens, kGroup) * slabs, blocks = ceil_div(units, kThreads / 64);
    if (blocks > INT32_MAX) return HIMUON_ERR_UNSUPPORTED;
    uint8_t* const q = static_cast<uint8_t*>(codes);
    uint8_t* const e = static_cast<uint8_t*>(exponents);
    if (dtype == HIMUON_BF16)
        hipLaunchKernelGGL(act_pack<GemmStore::BF16>, dim3((unsigned)blocks), dim3(kThreads), 0, hs, x, ld, n_tokens, cols, slabs,
                           units, q, e);
    else
        hipLaunchKernelGGL(act_pack<GemmStore::F32>, dim3((unsigned)blocks), dim3(kThreads), 0, hs, x, ld, n_tokens, cols, slabs,
                           units, q, e);
    return launch_status();
}

extern "C" int himuon_act_unpack(int64_t n_tokens, int64_t cols, const void* codes, const void* exponents, void* x,
                                 int64_t ld, int dtype, void* stream)
{
    using namespace himuon;
    const int sizes = act_sizes(n_tokens, cols);
    if (sizes != HIMUON_OK) return sizes;
    if (!known_dtype(dtype) || ld < cols || !small_product(n_tokens, ld)) return HIMUON_ERR_INVALID_ARG;
    if (n_tokens == 0) return HIMUON_OK;
    if (!x || !codes || !exponents || ((uintptr_t)codes & 15)) return HIMUON_ERR_INVALID_ARG;
    StreamDevice on(stream);
    if (on.status != HIMUON_OK) return on.status;
    const hipStream_t hs = static_cast<hipStream_t>(stream);
    const int64_t slabs = ceil_div(cols, 128);
    const int64_t units = ceil_div(n_tokens, kGroup) * slabs, blocks = ceil_div(units, kThreads / 64);
    if (blocks > INT32_MAX) return HIMUON_ERR_UNSUPPORTED;
    const uint8_t* const q = static_cast<const uint8_t*>(codes);
    const uint8_t* const e = static_cast<const uint8_t*>(exponents);
    if (dtype == HIMUON_BF16)
        hipLaunchKernelGGL(act_unpack<GemmStore::BF16>, dim3((unsigned)blocks), dim3(kThreads), 0, hs, q, e, n_tokens, cols, slabs,
                           units, x, ld);
    else
        hipLaunchKernelGGL(act_unpack<GemmStore::F32>, dim3((unsigned)blocks), dim3(kThreads), 0, hs, q, e, n_tokens, cols, slabs,
                           units, x, ld);
    return launch_status();
}

extern "C" size_t himuon_weight_grad_workspace_size(int64_t n_tokens, int64_t out, int64_t cols, int dtype)
{
    using namespace himuon;
    if (wgrad_sizes(n_tokens, out, cols) != HIMUON_OK || !known_dtype(dtype)) return 0;
    return 256;
}

extern "C" int himuon_weight_grad(int64_t n_tokens, int64_t out, int64_t cols, const void* grad, int64_t ld_grad, int dtype,
                                  const void* codes, const void* exponents, void* dweight, int64_t ld_dweight, int out_dtype,
                                  int accumulate, void* workspace, size_t workspace_bytes, void* stream)
{
    using namespace himuon;
    const int sizes = wgrad_sizes(n_tokens, out, cols);
    if (sizes != HIMUON_OK) return sizes;
    if (!known_dtype(dtype) || !known_dtype(out_dtype) || ld_grad < out || ld_dweight < cols) return HIMUON_ERR_INVALID_ARG;
    if (!small_product(n_tokens, ld_grad) || !small_product(out, ld_dweight)) return HIMUON_ERR_INVALID_ARG;
    if (!dweight || (n_tokens && (!grad || !codes || !exponents || ((uintptr_t)codes & 15)))) return HIMUON_ERR_INVALID_ARG;
    if (!workspace || ((uintptr_t)workspace & 255) ||
        workspace_bytes < himuon_weight_grad_workspace_size(n_tokens, out, cols, dtype))
        return HIMUON_ERR_WORKSPACE;
    if (n_tokens == 0 && accumulate) return HIMUON_OK;
    StreamDevice on(stream);
    if (on.status != HIMUON_OK) return on.status;
    const hipStream_t hs = static_cast<hipStream_t>(stream);
    WgradArgs p{};
    p.grad = grad;
    p.codes = static_cast<const uint8_t*>(codes);
    p.exps = static_cast<const uint8_t*>(exponents);
    p.out = dweight;
    p.tokens = n_tokens;
    p.ld_grad = ld_grad;
    p.ld_out = ld_dweight;
    p.rows = (int32_t)out;
    p.cols = (int32_t)cols;
    p.accumulate = accumulate != 0;
    if (dtype == HIMUON_BF16)
        return out_dtype == HIMUON_BF16 ? launch_wgrad<GemmStore::BF16, GemmStore::BF16>(p, hs)
                                        : launch_wgrad<GemmStore::BF16, GemmStore::F32>(p, hs);
    return out_dtype == HIMUON_BF16 ? launch_wgrad<GemmStore::F32, GemmStore::BF16>(p, hs)
                                    : launch_wgrad<GemmStore::F32, GemmStore::F32>(p, hs);
}
