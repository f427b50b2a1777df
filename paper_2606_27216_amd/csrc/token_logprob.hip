// Log probabilities of given tokens, entropies and the most likely tokens of each row of logits,
// and the gradient of the logits (himuon_token_logprob, himuon_token_logprob_grad).
//
// With z = scale * logits, m the row's maximum, s = sum e^(z - m), u = sum e^(z - m) (z - m):
//     lse = m + log s,  logprob = z_t - m - log s,  entropy = log s - u / s
//     d = scale (g_lp (delta - p) - g_H p (log p + H)),  p = e^(z - lse)
// so one pass over the logits with a running maximum gives them all; memory bounds it. The
// most likely tokens come from a second look at few of them: every lane keeps the largest
// logit that it saw, the k-th largest of those is a bound that the row's k largest logits reach,
// and only the shares of lanes whose own reaches it are read again, by all lanes together.
// (bf16 4096 x 128000 with the top 20: 209 us, 5.0 TB/s; gradient of 8192 x 32000: 176 to 196 us, 5.4 TB/s and more.)
#include "elementwise8.h"
#include "train_ops.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

namespace himuon {
namespace {

constexpr float kLog2e = 1.44269504088896341f;
constexpr float kLn2 = 0.693147180559945309f;

struct LogprobArgs {
    const void *logits, *tokens;
    float *logprob, *entropy, *lse, *top_logprob;
    int64_t* top_index;
    const float *g_lp, *g_h;
    void* d;
    int64_t rows, ld, ldd, blocks;  // blocks: of a row (gradient)
    int32_t vocab, top, wide;
    float scale;
};

// Running maximum of the logits, and sums of powers of two: c = scale log2 e, z log2 e = c x. (Logits are
// subtracted before they are multiplied: so those of the type's lowest value are equal ones, not
// infinite, and what is rounded is their distance.) A distance below kNothing has the power 0, which takes it
// out of u: it is cut there, so that it stays finite with the number of a row's logits times it.
constexpr float kNothing = -1024.f;
struct Sums {
    float m = -INFINITY, s = 0.f, u = 0.f;

    __device__ __forceinline__ void rescale(float now, float c)
    {
        if (now > m) {
            const float d = (m - now) * c, f = __builtin_amdgcn_exp2f(d);  // (d may be minus infinity: nothing so far)
            u = f * fmaf(fmaxf(d, kNothing), s, u);
            s *= f;
            m = now;
        }
    }
    __device__ __forceinline__ void add(float x, float c)
    {
        const float d = (x - (m == -INFINITY ? 0.f : m)) * c, e = __builtin_amdgcn_exp2f(d);
        s += e;
        u = fmaf(e, fmaxf(d, kNothing), u);
    }
    __device__ __forceinline__ void join(float m2, float s2, float u2, float c)
    {
        const float now = fmaxf(m, m2);
        if (now == -INFINITY) {  // (nothing yet, or NaN)
            s += s2;
            u += u2;
            return;
        }
        const float d = (m - now) * c, d2 = (m2 - now) * c, f = __builtin_amdgcn_exp2f(d), f2 = __builtin_amdgcn_exp2f(d2);
        const float a = f * fmaf(fmaxf(d, kNothing), s, u), b = f2 * fmaf(fmaxf(d2, kNothing), s2, u2);
        u = a + b;
        s = f * s + f2 * s2;
        m = now;
    }
};

// Larger logits have larger keys, NaN the largest; of equal ones the first index.
__device__ __forceinline__ uint32_t order_of(float x)
{
    if (!(x == x)) return 0xfffffffeu;  // (so that no key is ~0)
    const uint32_t b = __float_as_uint(x + 0.f);  // (minus zero equals zero)
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ uint64_t key_of(float x, int index) { return (uint64_t)order_of(x) << 32 | (uint32_t)~index; }

template <int NT> __device__ __forceinline__ void group_sync()
{
    if constexpr (NT == 64) wave_exchange();
    else __syncthreads();
}

constexpr int kCand = 512;
template <int NT> struct Shared {
    float m[NT / 64 + 1], s[NT / 64 + 1], u[NT / 64 + 1];
    uint64_t best[NT / 64 + 1];
    uint32_t lane_top[256];
    uint16_t hot[NT];
    uint64_t cand[kCand];
    uint32_t bound, hot_count, count;
};

// The largest key of the group's lanes.
template <int NT> __device__ __forceinline__ uint64_t group_max(uint64_t v, Shared<NT>& sh, int lane)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        const uint64_t w = __shfl_xor((unsigned long long)v, o);
        v = w > v ? w : v;
    }
    if constexpr (NT > 64) {
        if ((lane & 63) == 0) sh.best[lane >> 6] = v;
        __syncthreads();
        for (int i = 0; i < NT / 64; ++i) v = sh.best[i] > v ? sh.best[i] : v;
        __syncthreads();
    }
    return v;
}

template <GemmStore ST, int NT, bool TOP> __global__ void __launch_bounds__(NT == 64 ? 256 : NT) logprob_rows(const LogprobArgs p)
{
    constexpr int GROUPS = NT == 64 ? 4 : 1;
    __shared__ Shared<NT> shared[GROUPS];
    Shared<NT>& sh = shared[NT == 64 ? threadIdx.x >> 6 : 0];
    const int lane = threadIdx.x % NT;
    const int64_t row = (int64_t)blockIdx.x * GROUPS + (NT == 64 ? threadIdx.x >> 6 : 0);
    if (row >= p.rows) return;
    const int64_t token = load_index(p.tokens, row, p.wide);
    if (token < 0 || token >= p.vocab) {
        if (lane == 0) p.logprob[row] = p.entropy[row] = p.lse[row] = 0.f;
        if (TOP && lane < p.top) {
            p.top_logprob[row * p.top + lane] = 0.f;
            p.top_index[row * p.top + lane] = -1;
        }
        return;
    }
    const int64_t base = row * p.ld;
    const float c = p.scale * kLog2e;
    const int vocab = p.vocab;

    // Four chunks at a time, all on their way before the first is used.
    constexpr int U = 4;
    Sums sum;
    float best = -INFINITY;
    auto take = [&](const Raw8<ST> (&raw)[U], auto whole, int left) __attribute__((always_inline)) {  // (the first `left` elements count)
        constexpr bool WHOLE = decltype(whole)::value;
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < 8 * U; ++i) {
            const float x = raw_value<ST>(raw[i >> 3], i & 7);
            top = WHOLE || 8 * NT * (i >> 3) + (i & 7) < left ? fmaxf(top, x) : top;
        }
        best = fmaxf(best, top);
        sum.rescale(top, c);
#pragma unroll
        for (int i = 0; i < 8 * U; ++i)
            if (WHOLE || 8 * NT * (i >> 3) + (i & 7) < left) sum.add(raw_value<ST>(raw[i >> 3], i & 7), c);
    };
    for (int at = 8 * lane; at < vocab; at += 8 * NT * U) {
        Raw8<ST> raw[U];
        const int left = vocab - at;
        if (8 * NT * (U - 1) + 8 <= left) {
#pragma unroll
            for (int i = 0; i < U; ++i) raw[i] = get_raw8<ST>(p.logits, base + at + 8 * NT * i, 8);
            take(raw, std::true_type{}, 0);
        } else {
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const int n = left - 8 * NT * i;
                if (n > 0) raw[i] = get_raw8<ST>(p.logits, base + at + 8 * NT * i, n < 8 ? n : 8);
            }
            take(raw, std::false_type{}, left);
        }
    }
    const float mine = best;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum.join(__shfl_xor(sum.m, o), __shfl_xor(sum.s, o), __shfl_xor(sum.u, o), c);
    if constexpr (NT > 64) {
        if ((lane & 63) == 0) {
            sh.m[lane >> 6] = sum.m;
            sh.s[lane >> 6] = sum.s;
            sh.u[lane >> 6] = sum.u;
        }
        __syncthreads();
        sum = Sums{};
        for (int i = 0; i < NT / 64; ++i) sum.join(sh.m[i], sh.s[i], sh.u[i], c);
    }
    // (all minus infinity: log probabilities are minus infinity, not their difference)
    const bool none = sum.m == -INFINITY && sum.s == 0.f;
    const float log_s = __builtin_amdgcn_logf(sum.s);  // of base 2
    auto log_p = [&](float x) { return none ? -INFINITY : ((x - sum.m) * c - log_s) * kLn2; };
    if (lane == 0) {
        p.logprob[row] = log_p(get1<ST>(p.logits, base + token));
        p.entropy[row] = none ? 0.f : (log_s - sum.u / sum.s) * kLn2;
        p.lse[row] = none ? -INFINITY : fmaf(sum.m, p.scale, log_s * kLn2);
    }
    if constexpr (!TOP) return;

    const int k = p.top;
    auto put = [&](int place, uint64_t key) {
        const int index = (int)~(uint32_t)key;
        p.top_index[row * k + place] = index;
        p.top_logprob[row * k + place] = log_p(get1<ST>(p.logits, base + index));
    };
    // A lane's largest key below `under`.
    auto next_key = [&](uint64_t under) {
        uint64_t found = 0;
        for (int at = 8 * lane; at < vocab; at += 8 * NT) {
            const int n = vocab - at >= 8 ? 8 : vocab - at;
            const Raw8<ST> raw = get_raw8<ST>(p.logits, base + at, n);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint64_t key = key_of(raw_value<ST>(raw, e), at + e);
                found = e < n && key < under && key > found ? key : found;
            }
        }
        return found;
    };
    // Bound: the k-th largest of 64 or 256 disjoint sets of lanes' largest logits.
    constexpr int SETS = NT == 64 ? 64 : 256;
    float set_top = mine;
#pragma unroll
    for (int o = 1; o < NT / SETS; o *= 2) set_top = fmaxf(set_top, __shfl_xor(set_top, o));
    if (lane % (NT / SETS) == 0) sh.lane_top[lane / (NT / SETS)] = order_of(set_top);
    if (lane == 0) sh.count = sh.hot_count = 0;
    group_sync<NT>();
    if (lane < 64) {
        uint32_t v[SETS / 64];
#pragma unroll
        for (int i = 0; i < SETS / 64; ++i) v[i] = sh.lane_top[64 * i + lane];
        uint32_t bound = 0;
        for (int bit = 31; bit >= 0; --bit) {
            const uint32_t trial = bound | 1u << bit;
            int at_least = 0;
#pragma unroll
            for (int i = 0; i < SETS / 64; ++i) at_least += __popcll(__ballot(v[i] >= trial));
            if (at_least >= k) bound = trial;
        }
        if (lane == 0) sh.bound = bound;
    }
    group_sync<NT>();
    const uint32_t bound = sh.bound;
    // (a row with NaN, or with fewer than k sets above minus infinity, is left to the search below)
    const bool plain = sum.s == sum.s && bound > order_of(-INFINITY);
    if (plain && order_of(mine) >= bound) sh.hot[atomicAdd(&sh.hot_count, 1u)] = (uint16_t)lane;  // (in any order: what they hold is ranked)
    group_sync<NT>();
    const int hot = (int)sh.hot_count, chunks = (vocab + 8 * NT - 1) / (8 * NT);
    // (more: many lanes' largest logits are equal to the bound, which bf16 logits' are at a top near the limit: of
    // normal logits two thirds of the rows at 64, 3% at 60, none at 56. The search below takes them.)
    if (hot <= (NT == 64 ? 64 : NT / 4)) {
        for (int i = lane; i < hot * chunks; i += NT) {
            const int h = i / chunks, at = 8 * (sh.hot[h] + NT * (i - h * chunks));
            if (at >= vocab) continue;
            const int n = vocab - at >= 8 ? 8 : vocab - at;
            const Raw8<ST> raw = get_raw8<ST>(p.logits, base + at, n);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float x = raw_value<ST>(raw, e);
                if (e < n && order_of(x) >= bound) {
                    const uint32_t place = atomicAdd(&sh.count, 1u);
                    if (place < kCand) sh.cand[place] = key_of(x, at + e);
                }
            }
        }
    }
    group_sync<NT>();
    const int count = (int)sh.count;
    if (plain && count >= k && count <= kCand) {
        for (int i = lane; i < count; i += NT) {
            const uint64_t key = sh.cand[i];
            int rank = 0;
            for (int j = 0; j < count; ++j) rank += sh.cand[j] > key;
            if (rank < k) put(rank, key);
        }
        return;
    }
    // Equal logits at the bound, few finite ones, NaN: the k largest one after the other.
    uint64_t own = next_key(~0ull);
    for (int i = 0; i < k; ++i) {
        const uint64_t key = group_max<NT>(own, sh, lane);
        if (own == key) {
            put(i, key);
            own = next_key(key);
        }
    }
}

// A block takes kGradCols columns of a row. Probabilities follow from lse, which is rounded by up to
// 2^-24 of itself, and they by as much: from far() on, one block finds the row's sum again and
// writes all of it (alone: d may be the logits). bf16: 1024, where that passes 2^-14, far below half a step of the
// result. fp32: 32, 2^-20 below it, what the exponents of likely tokens round by themselves (8192 x 32000: 532 us in that
// form, 394 in the other; bf16 251 and 179; 256 x 128000 fp32 128 and 47).
constexpr int kGradThreads = 256, kGradChunks = 4, kGradCols = 8 * kGradThreads * kGradChunks;
constexpr float kFarthest = 1048576.f;  // (half of lse's last place: 2^-4)
template <GemmStore ST> constexpr float far() { return ST == GemmStore::F32 ? 32.f : 1024.f; }

template <bool SUM> __device__ __forceinline__ float block_join(float v, float* parts)
{
    auto join = [](float a, float b) { return SUM ? a + b : fmaxf(a, b); };
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = join(v, __shfl_xor(v, o));
    if ((threadIdx.x & 63) == 0) parts[threadIdx.x >> 6] = v;
    __syncthreads();
    return join(join(parts[0], parts[1]), join(parts[2], parts[3]));
}

template <GemmStore ST> __global__ void __launch_bounds__(kGradThreads) logprob_grad(const LogprobArgs p)
{
    __shared__ float parts[2][kGradThreads / 64];
    const int64_t row = blockIdx.x / p.blocks;
    const int first = (int)(blockIdx.x - row * p.blocks) * kGradCols;
    const int64_t token = load_index(p.tokens, row, p.wide);
    const float lse = p.lse[row];
    const bool on = token >= 0 && token < p.vocab && lse != -INFINITY;
    const float gl = on && p.g_lp ? p.g_lp[row] * p.scale : 0.f, gh = on && p.g_h ? p.g_h[row] * p.scale : 0.f;
    const float entropy = p.g_h ? p.entropy[row] : 0.f;
    // Of a logit with this log probability; `q`: its probability.
    auto grad = [&](int at, float lp, float q) {
        return gl * ((at == token ? 1.f : 0.f) - q) - gh * (q * (fmaxf(lp, -1e30f) + entropy));
    };
    auto store = [&](int at, int n, f32x8 d) {
        const int64_t to = row * p.ldd + at;
        if (n == 8) {
            put8<ST>(p.d, to, d);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < n) put1<ST>(p.d, to + e, d[e]);
        }
    };
    if (on && fabsf(lse) >= far<ST>()) {
        // (one of the row's blocks, another one every eight rows: blocks are dealt out to eight XCDs in turn)
        if (blockIdx.x - row * p.blocks != (row >> 3) % p.blocks) return;
        const float c = p.scale * kLog2e;
        auto each = [&](auto work) {
            for (int at = 8 * (int)threadIdx.x; at < p.vocab; at += 8 * kGradThreads * kGradChunks) {
                Raw8<ST> raw[kGradChunks];
#pragma unroll
                for (int i = 0; i < kGradChunks; ++i) {
                    const int n = min(8, p.vocab - at - 8 * kGradThreads * i);
                    if (n > 0) raw[i] = get_raw8<ST>(p.logits, row * p.ld + at + 8 * kGradThreads * i, n);
                }
#pragma unroll
                for (int i = 0; i < kGradChunks; ++i) {
                    const int n = min(8, p.vocab - at - 8 * kGradThreads * i);
                    if (n > 0) work(at + 8 * kGradThreads * i, n, raw[i]);
                }
            }
        };
        // Powers of two relative to lse, whose sum is then near 1 and whose logarithm is what lse lacks; or to the
        // row's maximum, where lse may be off by too much.
        const bool by_max = fabsf(lse) >= kFarthest;
        float m = -INFINITY, s = 0.f;
        if (by_max) {
            each([&](int, int n, const Raw8<ST>& raw) {
#pragma unroll
                for (int e = 0; e < 8; ++e) m = e < n ? fmaxf(m, raw_value<ST>(raw, e)) : m;
            });
            m = block_join<false>(m, parts[0]);
        }
        auto power = [&](float x) { return by_max ? (x - m) * c : fmaf(x, p.scale, -lse) * kLog2e; };
        each([&](int, int n, const Raw8<ST>& raw) {
#pragma unroll
            for (int e = 0; e < 8; ++e) s += e < n ? __builtin_amdgcn_exp2f(power(raw_value<ST>(raw, e))) : 0.f;
        });
        const float log_s = __builtin_amdgcn_logf(block_join<true>(s, parts[1]));
        each([&](int at, int n, const Raw8<ST>& raw) {
            f32x8 d;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float lp = power(raw_value<ST>(raw, e)) - log_s;
                d[e] = grad(at + e, lp * kLn2, __builtin_amdgcn_exp2f(lp));
            }
            store(at, n, d);
        });
        return;
    }
    Raw8<ST> raw[kGradChunks];
#pragma unroll
    for (int i = 0; i < kGradChunks; ++i) {
        const int at = first + 8 * (kGradThreads * i + (int)threadIdx.x), n = p.vocab - at >= 8 ? 8 : p.vocab - at;
        if (on && n > 0) raw[i] = get_raw8<ST>(p.logits, row * p.ld + at, n);
    }
#pragma unroll
    for (int i = 0; i < kGradChunks; ++i) {
        const int at = first + 8 * (kGradThreads * i + (int)threadIdx.x), n = p.vocab - at >= 8 ? 8 : p.vocab - at;
        if (n <= 0) return;
        f32x8 d;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float lp = fmaf(raw_value<ST>(raw[i], e), p.scale, -lse);
            d[e] = on ? grad(at + e, lp, __builtin_amdgcn_exp2f(lp * kLog2e)) : 0.f;
        }
        store(at, n, d);
    }
}

// Lanes of a row: a wave's, or a block's of 256 or 512. bf16, us: with the top 5 8192 x 1500 18.6 with 64 lanes, 47 with 256, x 2048
// 15.5 and 45, x 4096 20.7 and 46 (the latter is taken), 256 x 3000 14.3 and 14.1; with the top 20 4096 x 32000 73 with 256,
// 87 with 512; 4096 x 128000 214 with 512, 229 with 1024.
int row_lanes(int64_t vocab) { return vocab <= 2048 ? 64 : vocab <= 32768 ? 256 : 512; }
int64_t row_blocks(int64_t rows, int64_t vocab) { return row_lanes(vocab) == 64 ? ceil_div(rows, 4) : rows; }

template <GemmStore ST, bool TOP> int launch_logprob(const LogprobArgs& p, hipStream_t stream)
{
    const int lanes = row_lanes(p.vocab);
    const dim3 grid((unsigned)row_blocks(p.rows, p.vocab)), block(std::max(lanes, 256));
    if (lanes == 64) hipLaunchKernelGGL((logprob_rows<ST, 64, TOP>), grid, block, 0, stream, p);
    else if (lanes == 256) hipLaunchKernelGGL((logprob_rows<ST, 256, TOP>), grid, block, 0, stream, p);
    else hipLaunchKernelGGL((logprob_rows<ST, 512, TOP>), grid, block, 0, stream, p);
    return launch_status();
}

int check_logprob(int64_t rows, int64_t vocab, int64_t ld, int dtype, int index, float scale)
{
    if (rows < 0 || vocab < 1 || ld < vocab || !known_dtype(dtype) || !known_index(index) || !(scale > 0.f) || !std::isfinite(scale))
        return HIMUON_ERR_INVALID_ARG;
    if (!small_product(rows, ld)) return HIMUON_ERR_INVALID_ARG;
    // (a lane's place in a row is counted in 32 bits)
    if (rows > INT32_MAX || vocab > INT32_MAX - 16384) return HIMUON_ERR_UNSUPPORTED;
    return HIMUON_OK;
}

}  // namespace
}  // namespace himuon

extern "C" int himuon_token_logprob(int64_t n_tokens, int64_t vocab, const void* logits, int64_t ld, int dtype, const void* tokens,
                                    int index, float scale, int top, float* logprob, float* entropy, float* lse, float* top_logprob,
                                    int64_t* top_index, void* stream)
{
    using namespace himuon;
    const int st = check_logprob(n_tokens, vocab, ld, dtype, index, scale);
    if (st != HIMUON_OK) return st;
    if (top < 0 || top > HIMUON_MAX_TOP || top > vocab) return HIMUON_ERR_INVALID_ARG;
    if (n_tokens == 0) return HIMUON_OK;
    if (!logits || !tokens || !logprob || !entropy || !lse || (top > 0 && (!top_logprob || !top_index))) return HIMUON_ERR_INVALID_ARG;
    if (!launchable(row_blocks(n_tokens, vocab), std::max(row_lanes(vocab), 256))) return HIMUON_ERR_UNSUPPORTED;
    StreamDevice on(stream);
    if (on.status != HIMUON_OK) return on.status;
    LogprobArgs p{};
    p.logits = logits;
    p.tokens = tokens;
    p.logprob = logprob;
    p.entropy = entropy;
    p.lse = lse;
    p.top_logprob = top_logprob;
    p.top_index = top_index;
    p.rows = n_tokens;
    p.ld = ld;
    p.vocab = (int32_t)vocab;
    p.top = top;
    p.wide = index == HIMUON_I64;
    p.scale = scale;
    const hipStream_t hs = static_cast<hipStream_t>(stream);
    if (dtype == HIMUON_BF16) return top ? launch_logprob<GemmStore::BF16, true>(p, hs) : launch_logprob<GemmStore::BF16, false>(p, hs);
    return top ? launch_logprob<GemmStore::F32, true>(p, hs) : launch_logprob<GemmStore::F32, false>(p, hs);
}

extern "C" int himuon_token_logprob_grad(int64_t n_tokens, int64_t vocab, const float* g_logprob, const float* g_entropy,
                                         const void* logits, int64_t ld, int dtype, const void* tokens, int index, const float* lse,
                                         const float* entropy, float scale, void* d, int64_t ld_d, void* stream)
{
    using namespace himuon;
    const int st = check_logprob(n_tokens, vocab, ld, dtype, index, scale);
    if (st != HIMUON_OK) return st;
    if (ld_d < vocab || !small_product(n_tokens, ld_d)) return HIMUON_ERR_INVALID_ARG;
    if (n_tokens == 0) return HIMUON_OK;
    if (!logits || !tokens || !lse || !d || (g_entropy && !entropy)) return HIMUON_ERR_INVALID_ARG;
    LogprobArgs p{};
    p.blocks = ceil_div(vocab, kGradCols);
    if (!small_product(n_tokens, p.blocks) || !launchable(n_tokens * p.blocks, kGradThreads)) return HIMUON_ERR_UNSUPPORTED;
    StreamDevice on(stream);
    if (on.status != HIMUON_OK) return on.status;
    p.logits = logits;
    p.tokens = tokens;
    p.lse = const_cast<float*>(lse);
    p.entropy = const_cast<float*>(entropy);
    p.g_lp = g_logprob;
    p.g_h = g_entropy;
    p.d = d;
    p.rows = n_tokens;
    p.ld = ld;
    p.ldd = ld_d;
    p.vocab = (int32_t)vocab;
    p.wide = index == HIMUON_I64;
    p.scale = scale;
    const hipStream_t hs = static_cast<hipStream_t>(stream);
    const dim3 grid((unsigned)(n_tokens * p.blocks));
    if (dtype == HIMUON_BF16) hipLaunchKernelGGL(logprob_grad<GemmStore::BF16>, grid, dim3(kGradThreads), 0, hs, p);
    else hipLaunchKernelGGL(logprob_grad<GemmStore::F32>, grid, dim3(kGradThreads), 0, hs, p);
    return launch_status();
}
