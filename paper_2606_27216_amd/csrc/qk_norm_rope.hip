// Per-head norms of queries and keys with the position rotation, and the backward
// pass (himuon_qk_norm_rope, himuon_qk_norm_rope_grad).
//
// For a head's vector x of D elements, r = (mean x^2 + eps)^(-1/2), gain w:
//     z = r x w,  y = R z           R turns the pairs of the position's angles
//     dz = R^T dy,  dw = sum over tokens and heads of dz r x,
//     dx = r (dz w - x r^2 mean(dz w x))
// so one pass over x (and dy) is all there is to read: both sums over a head are
// taken at once, and r is computed again in the backward pass.
//
// A lane holds eight pairs of a head, both elements of each, so the rotation needs no
// exchange; L lanes hold the head, a wave 64 / L heads. Where heads are many, a wave walks over
// those of one token, whose cosines and sines stay in registers with the gains. Where a
// token's heads fit the wave, each group of lanes keeps one head and the wave walks over
// tokens, several at a time. Memory bounds it: 8 x 1024 tokens, 32 + 32 heads of 128, bf16, forward
// 48 us (273 MB, 5.7 TB/s); 16 x 1024 tokens, 16 + 8 heads, backward 53 us and
// 4.6 for the gains' sums (306 MB, 5.8 TB/s).
#include "elementwise8.h"
#include "train_ops.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

namespace himuon {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int64_t kMostHeads = INT64_C(1) << 30;  // queries' and keys' (the kernels count them in 32 bits, 65536 ahead)

struct Strided {
    uint8_t* ptr;
    int64_t sb, ss, sh;
};

struct QkArgs {
    Strided q, k, qo, ko, gq, gk;  // forward: inputs, outputs; backward: inputs, their gradients, the outputs' gradients
    const void *wq, *wk;
    const float *cs, *sn;
    const void* positions;
    float* part;                   // backward: [blocks][2][D]
    int64_t tokens, seq, table_rows, units;
    int32_t hq, hk, dim, rot, wide, parts, gain_bf16, slots;
    float eps, inv_dim;
};

// Sum over the L lanes of a head (L consecutive lanes, a power of two).
template <int L> __device__ __forceinline__ float head_sum(float v)
{
    auto dpp = [](float x, auto ctrl) {
        return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), decltype(ctrl)::value, 0xf, 0xf, true));
    };
    if constexpr (L >= 2) v += dpp(v, std::integral_constant<int, 0xB1>{});   // lane ^ 1
    if constexpr (L >= 4) v += dpp(v, std::integral_constant<int, 0x4E>{});   // lane ^ 2
    if constexpr (L >= 8) v += dpp(v, std::integral_constant<int, 0x141>{});  // the other four of eight
    if constexpr (L >= 16) v += dpp(v, std::integral_constant<int, 0x140>{}); // the other eight of sixteen
    if constexpr (L >= 32) v += __shfl_xor(v, 16);
    if constexpr (L >= 64) v += __shfl_xor(v, 32);
    return v;
}

// The pairs of a head: the rotated ones first, then the others, each kind in runs of eight
// (side by side, INTER, the two kinds in the same runs); the last run of a kind ends with its
// last pair and repeats pairs of the run before it where their number is no multiple of eight.
enum class Runs : int {
    EXACT,  // whole runs of one kind, none of which repeats pairs
    WHOLE,  // whole runs
    SHORT   // a kind may have fewer than eight pairs
};

struct Place {
    int pair;     // the run's first pair
    int n;        // pairs that exist: 8, fewer if there are no eight of the kind, 0 for an idle lane
    int skip;     // leading ones that the run before has too: not to be counted again
    int a, b;     // first and second element of the first pair (the next ones follow; with INTER, side by side)
};

template <bool INTER> __device__ __forceinline__ void pair_elements(int pair, int dim, int rot, int& a, int& b)
{
    const int turned = rot / 2, rest = (dim - rot) / 2;
    if (INTER) {
        a = 2 * pair;
        b = a + 1;
    } else if (pair < turned) {
        a = pair;
        b = turned + pair;
    } else {
        a = rot + pair - turned;
        b = a + rest;
    }
}

template <bool INTER> __device__ __forceinline__ Place place(int l, int dim, int rot)
{
    const int turned = INTER ? dim / 2 : rot / 2, rest = dim / 2 - turned, runs = (turned + 7) / 8;
    const bool second = l >= runs;
    const int r = second ? l - runs : l, first = second ? turned : 0, count = second ? rest : turned;
    Place w;
    w.n = max(0, min(8, count - 8 * r));
    const int start = w.n > 0 ? min(8 * r, max(0, count - 8)) : 0;
    w.skip = w.n > 0 ? 8 * r - start : 0;
    if (w.n > 0) w.n = min(8, count);
    w.pair = w.n > 0 ? first + start : 0;
    pair_elements<INTER>(w.pair, dim, rot, w.a, w.b);
    return w;
}

// A lane's eight pairs: first and second elements.
struct Pairs {
    f32x8 u, v;
};

// The lane's pairs of the vector at base + i. (Idle lanes read the first run, if it is whole.)
template <GemmStore ST, bool INTER, Runs R> __device__ __forceinline__ Pairs load_pairs(const void* base, int64_t i, const Place& w)
{
    Pairs x;
    if (R != Runs::SHORT || w.n == 8 || w.n == 0) {
        if constexpr (INTER) {
            // (a head of fewer than eight pairs has no whole run: its idle lanes read nothing)
            if (R == Runs::SHORT && w.n == 0) {
                x.u = x.v = f32x8{};
                return x;
            }
            const f32x8 lo = get8<ST>(base, i + w.a), hi = get8<ST>(base, i + w.a + 8);
            x.u = f32x8{lo[0], lo[2], lo[4], lo[6], hi[0], hi[2], hi[4], hi[6]};
            x.v = f32x8{lo[1], lo[3], lo[5], lo[7], hi[1], hi[3], hi[5], hi[7]};
        } else {
            if (R == Runs::SHORT && w.n == 0) {
                x.u = x.v = f32x8{};
                return x;
            }
            x.u = get8<ST>(base, i + w.a);
            x.v = get8<ST>(base, i + w.b);
        }
    } else {
        constexpr int STEP = INTER ? 2 : 1;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int k = STEP * min(e, w.n - 1);
            const float a = get1<ST>(base, i + w.a + k), b = get1<ST>(base, i + w.b + k);
            x.u[e] = e < w.n ? a : 0.f;
            x.v[e] = e < w.n ? b : 0.f;
        }
    }
    return x;
}

template <GemmStore ST, bool INTER, Runs R>
__device__ __forceinline__ void store_pairs(void* base, int64_t i, const Place& w, const Pairs& x)
{
    if (w.n == 0) return;
    if (R != Runs::SHORT || w.n == 8) {
        if constexpr (INTER) {
            put8<ST>(base, i + w.a, f32x8{x.u[0], x.v[0], x.u[1], x.v[1], x.u[2], x.v[2], x.u[3], x.v[3]});
            put8<ST>(base, i + w.a + 8, f32x8{x.u[4], x.v[4], x.u[5], x.v[5], x.u[6], x.v[6], x.u[7], x.v[7]});
        } else {
            put8<ST>(base, i + w.a, x.u);
            put8<ST>(base, i + w.b, x.v);
        }
    } else {
        constexpr int STEP = INTER ? 2 : 1;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (e < w.n) {
                put1<ST>(base, i + w.a + STEP * e, x.u[e]);
                put1<ST>(base, i + w.b + STEP * e, x.v[e]);
            }
        }
    }
}

// Whether pair e of the lane counts in sums over the head. (EXACT: all of a lane's do, or none.)
template <Runs R> __device__ __forceinline__ bool counts(const Place& w, int e)
{
    return R == Runs::EXACT ? w.n > 0 : e >= w.skip && e < w.n;
}

template <bool INTER, Runs R> __device__ __forceinline__ Pairs load_gains(const QkArgs& p, const void* gain, const Place& w)
{
    if (p.gain_bf16) return load_pairs<GemmStore::BF16, INTER, R>(gain, 0, w);
    return load_pairs<GemmStore::F32, INTER, R>(gain, 0, w);
}

// The lane's cosines (u) and sines (v) of position t: 1 and 0 for what is not rotated.
template <bool INTER, Runs R> __device__ __forceinline__ Pairs load_turn(const QkArgs& p, int64_t t, const Place& w, bool used = true)
{
    const int half = p.rot / 2;
    const int64_t i = t * half + w.pair;
    Pairs x;
    x.u = f32x8{1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
    x.v = f32x8{};
    if (w.pair >= half || !used) return x;
    constexpr bool CUT = R == Runs::SHORT || (INTER && R == Runs::WHOLE);  // (a run that is not all rotated)
    if (!CUT || w.pair + 8 <= half) {
        x.u = get8<GemmStore::F32>(p.cs, i);
        x.v = get8<GemmStore::F32>(p.sn, i);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (w.pair + e < half) {
                x.u[e] = p.cs[i + e];
                x.v[e] = p.sn[i + e];
            }
        }
    }
    return x;
}

// The position of a token; false if it lies outside the table.
__device__ __forceinline__ bool token_position(const QkArgs& p, int64_t token, int64_t s, int64_t& t)
{
    t = p.positions ? load_index(p.positions, token, p.wide != 0) : s;
    const bool in = t >= 0 && t < p.table_rows;
    if (!in) t = 0;
    return in;
}

// x -> R (r x w), the head's sum over L lanes.
template <Runs R, int L>
__device__ __forceinline__ void forward_head(const QkArgs& p, const Place& w, const Pairs& g, const Pairs& turn, bool used, Pairs& x)
{
    float sq = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) sq += counts<R>(w, e) ? x.u[e] * x.u[e] + x.v[e] * x.v[e] : 0.f;
    const float r = rsqrtf(head_sum<L>(sq) * p.inv_dim + p.eps);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float z0 = x.u[e] * r * g.u[e], z1 = x.v[e] * r * g.v[e];
        x.u[e] = used ? z0 * turn.u[e] - z1 * turn.v[e] : 0.f;
        x.v[e] = used ? z1 * turn.u[e] + z0 * turn.v[e] : 0.f;
    }
}

// x, y = dL/d(output) -> x = dL/dx, d += the gain's terms.
template <Runs R, int L>
__device__ __forceinline__ void backward_head(const QkArgs& p, const Place& w, const Pairs& g, const Pairs& turn, bool used, Pairs& x,
                                              Pairs& y, Pairs& d)
{
    float sq = 0.f, dot = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float a = y.u[e] * turn.u[e] + y.v[e] * turn.v[e], c = y.v[e] * turn.u[e] - y.u[e] * turn.v[e];
        y.u[e] = a;  // dz
        y.v[e] = c;
        sq += counts<R>(w, e) ? x.u[e] * x.u[e] + x.v[e] * x.v[e] : 0.f;
        dot += counts<R>(w, e) ? a * g.u[e] * x.u[e] + c * g.v[e] * x.v[e] : 0.f;
    }
    sq = head_sum<L>(sq);
    dot = head_sum<L>(dot);
    const float r = rsqrtf(sq * p.inv_dim + p.eps);
    const float m = r * r * (dot * p.inv_dim);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        d.u[e] += used ? y.u[e] * (x.u[e] * r) : 0.f;
        d.v[e] += used ? y.v[e] * (x.v[e] * r) : 0.f;
        x.u[e] = used ? r * (y.u[e] * g.u[e] - x.u[e] * m) : 0.f;
        x.v[e] = used ? r * (y.v[e] * g.v[e] - x.v[e] * m) : 0.f;
    }
}

// ------------------------------------------------------- many heads: a wave, one token

template <GemmStore ST, bool INTER, Runs R, int L>
__device__ __forceinline__ void forward_heads(const QkArgs& p, const Strided& in, const Strided& out, const void* gain, int heads,
                                              int part, int64_t b, int64_t s, bool used, const Place& w, const Pairs& turn)
{
    constexpr int G = 64 / L;
    const int lane = threadIdx.x & 63;
    const Pairs g = load_gains<INTER, R>(p, gain, w);
    const int64_t bi = b * in.sb + s * in.ss, bo = b * out.sb + s * out.ss;
    for (int h = part * G + lane / L; h < heads; h += p.parts * G) {
        Pairs x = load_pairs<ST, INTER, R>(in.ptr, bi + h * in.sh, w);
        forward_head<R, L>(p, w, g, turn, used, x);
        store_pairs<ST, INTER, R>(out.ptr, bo + h * out.sh, w, x);
    }
}

template <GemmStore ST, bool INTER, Runs R, int L> __global__ void __launch_bounds__(kThreads) qk_forward(const QkArgs p)
{
    const int64_t unit = (int64_t)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (unit >= p.units) return;
    const int64_t token = unit / p.parts;
    const int part = (int)(unit - token * p.parts);
    const int64_t b = token / p.seq, s = token - b * p.seq;
    const Place w = place<INTER>(threadIdx.x & (L - 1), p.dim, p.rot);
    int64_t t;
    const bool used = token_position(p, token, s, t);
    Pairs turn{};
    if (used) turn = load_turn<INTER, R>(p, t, w);
    forward_heads<ST, INTER, R, L>(p, p.q, p.qo, p.wq, p.hq, part, b, s, used, w, turn);
    forward_heads<ST, INTER, R, L>(p, p.k, p.ko, p.wk, p.hk, part, b, s, used, w, turn);
}

template <GemmStore ST, bool INTER, Runs R, int L>
__device__ __forceinline__ void backward_heads(const QkArgs& p, const Strided& in, const Strided& grad, const Strided& out,
                                               const Pairs& g, int heads, int64_t b, int64_t s, bool used, const Place& w,
                                               const Pairs& turn, Pairs& d)
{
    constexpr int G = 64 / L;
    const int lane = threadIdx.x & 63;
    const int64_t bi = b * in.sb + s * in.ss, bg = b * grad.sb + s * grad.ss, bo = b * out.sb + s * out.ss;
    for (int h = lane / L; h < heads; h += G) {
        Pairs x = load_pairs<ST, INTER, R>(in.ptr, bi + h * in.sh, w);
        Pairs y = load_pairs<ST, INTER, R>(grad.ptr, bg + h * grad.sh, w);
        backward_head<R, L>(p, w, g, turn, used, x, y, d);
        store_pairs<ST, INTER, R>(out.ptr, bo + h * out.sh, w, x);
    }
}

// Element x (first or second of pair x / 2) of a block's partial sums for a gain.
template <bool INTER> __device__ __forceinline__ void put_gain(const QkArgs& p, int key, int x, float v)
{
    int a, b;
    pair_elements<INTER>(x >> 1, p.dim, p.rot, a, b);
    p.part[((int64_t)blockIdx.x * 2 + key) * p.dim + (x & 1 ? b : a)] = v;
}

// Blocks (.., 0) have the queries, (.., 1) the keys: one gain and one set of sums in
// registers. A wave takes tokens `units` apart; its sums stay in registers until the
// end, when the block adds its own up in LDS and leaves a row of partial sums.
template <GemmStore ST, bool INTER, Runs R, int L> __global__ void __launch_bounds__(kThreads) qk_backward(const QkArgs p)
{
    __shared__ float sums[kWaves][L * 16];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int key = blockIdx.y;
    const Place w = place<INTER>(threadIdx.x & (L - 1), p.dim, p.rot);
    const Strided in = key ? p.k : p.q, grad = key ? p.gk : p.gq, out = key ? p.ko : p.qo;
    const int heads = key ? p.hk : p.hq;
    const Pairs g = load_gains<INTER, R>(p, key ? p.wk : p.wq, w);
    Pairs d{};
    for (int64_t token = (int64_t)blockIdx.x * kWaves + wave; token < p.tokens; token += p.units) {
        const int64_t b = token / p.seq, s = token - b * p.seq;
        int64_t t;
        const bool used = token_position(p, token, s, t);
        const Pairs turn = load_turn<INTER, R>(p, t, w, used);
        backward_heads<ST, INTER, R, L>(p, in, grad, out, g, heads, b, s, used, w, turn, d);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        float u = d.u[e], v = d.v[e];
#pragma unroll
        for (int o = L; o < 64; o <<= 1) {
            u += __shfl_xor(u, o);
            v += __shfl_xor(v, o);
        }
        if (lane < L && counts<R>(w, e)) {
            sums[wave][2 * (w.pair + e)] = u;
            sums[wave][2 * (w.pair + e) + 1] = v;
        }
    }
    __syncthreads();
    for (int x = threadIdx.x; x < p.dim; x += kThreads) {
        float v = 0.f;
#pragma unroll
        for (int wv = 0; wv < kWaves; ++wv) v += sums[wv][x];
        put_gain<INTER>(p, key, x, v);
    }
}

// ------------------------------------- few heads: a group of lanes, one head; a wave, tokens

// A wave has 64 / L groups of lanes, `slots` of them (a power of two, the heads of a token
// rounded up) to a token. What a group without a head or a token does is not stored.
__device__ __forceinline__ int token_of(const QkArgs& p, int64_t first, int in_wave, bool& live, int64_t& b, int64_t& s)
{
    const int64_t token = first + in_wave;
    live = token < p.tokens;
    const uint32_t t = (uint32_t)(live ? token : p.tokens - 1), q = t / (uint32_t)p.seq;
    b = q;
    s = t - q * (uint32_t)p.seq;
    return (int)t;
}

template <GemmStore ST, bool INTER, Runs R, int L> __global__ void __launch_bounds__(kThreads) qk_forward_few(const QkArgs p)
{
    const int lane = threadIdx.x & 63, group = lane / L, slot = group & (p.slots - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tokens = 64 / L / p.slots;  // of a wave at a time
    const Place w = place<INTER>(threadIdx.x & (L - 1), p.dim, p.rot);
    const bool head = slot < p.hq + p.hk, key = head && slot >= p.hq;
    const int h = !head ? 0 : key ? slot - p.hq : slot;
    const Pairs g = load_gains<INTER, R>(p, key ? p.wk : p.wq, w);
    uint8_t* const src = key ? p.k.ptr : p.q.ptr;
    uint8_t* const dst = key ? p.ko.ptr : p.qo.ptr;
    const int64_t ib = key ? p.k.sb : p.q.sb, is = key ? p.k.ss : p.q.ss, i0 = h * (key ? p.k.sh : p.q.sh);
    const int64_t ob = key ? p.ko.sb : p.qo.sb, os = key ? p.ko.ss : p.qo.ss, o0 = h * (key ? p.ko.sh : p.qo.sh);
    for (int64_t first = ((int64_t)blockIdx.x * kWaves + wave) * tokens; first < p.tokens; first += p.units * tokens) {
        bool live;
        int64_t b, s, t;
        const int token = token_of(p, first, group / p.slots, live, b, s);
        const bool used = token_position(p, token, s, t);
        Pairs x = load_pairs<ST, INTER, R>(src, b * ib + s * is + i0, w);
        const Pairs turn = load_turn<INTER, R>(p, t, w, used);
        forward_head<R, L>(p, w, g, turn, used, x);
        if (live && head) store_pairs<ST, INTER, R>(dst, b * ob + s * os + o0, w, x);
    }
}

template <GemmStore ST, bool INTER, Runs R, int L> __global__ void __launch_bounds__(kThreads) qk_backward_few(const QkArgs p)
{
    constexpr int G = 64 / L;
    __shared__ float sums[kWaves * G][L * 16 + 1];
    const int lane = threadIdx.x & 63, group = lane / L, slot = group & (p.slots - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tokens = G / p.slots;
    const Place w = place<INTER>(threadIdx.x & (L - 1), p.dim, p.rot);
    const bool head = slot < p.hq + p.hk, key = head && slot >= p.hq;
    const int h = !head ? 0 : key ? slot - p.hq : slot;
    const Pairs g = load_gains<INTER, R>(p, key ? p.wk : p.wq, w);
    uint8_t* const src = key ? p.k.ptr : p.q.ptr;
    uint8_t* const ups = key ? p.gk.ptr : p.gq.ptr;
    uint8_t* const dst = key ? p.ko.ptr : p.qo.ptr;
    const int64_t ib = key ? p.k.sb : p.q.sb, is = key ? p.k.ss : p.q.ss, i0 = h * (key ? p.k.sh : p.q.sh);
    const int64_t gb = key ? p.gk.sb : p.gq.sb, gs = key ? p.gk.ss : p.gq.ss, g0 = h * (key ? p.gk.sh : p.gq.sh);
    const int64_t ob = key ? p.ko.sb : p.qo.sb, os = key ? p.ko.ss : p.qo.ss, o0 = h * (key ? p.ko.sh : p.qo.sh);
    Pairs d{};
    for (int64_t first = ((int64_t)blockIdx.x * kWaves + wave) * tokens; first < p.tokens; first += p.units * tokens) {
        bool live;
        int64_t b, s, t;
        const int token = token_of(p, first, group / p.slots, live, b, s);
        const bool used = token_position(p, token, s, t) && live && head;
        Pairs x = load_pairs<ST, INTER, R>(src, b * ib + s * is + i0, w);
        Pairs y = load_pairs<ST, INTER, R>(ups, b * gb + s * gs + g0, w);
        const Pairs turn = load_turn<INTER, R>(p, t, w, used);
        backward_head<R, L>(p, w, g, turn, used, x, y, d);
        if (live && head) store_pairs<ST, INTER, R>(dst, b * ob + s * os + o0, w, x);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if (counts<R>(w, e)) {
            sums[wave * G + group][2 * (w.pair + e)] = d.u[e];
            sums[wave * G + group][2 * (w.pair + e) + 1] = d.v[e];
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * p.dim; i += kThreads) {
        const int which = i >= p.dim, x = i - which * p.dim;
        float v = 0.f;
        for (int k = 0; k < kWaves * G; ++k) {
            const int at = k & (p.slots - 1);
            if (at < p.hq + p.hk && (at >= p.hq) == (which != 0)) v += sums[k][x];
        }
        put_gain<INTER>(p, which, x, v);
    }
}

// Sums of the blocks' rows for 16 of the 2 D columns, the rows shared out over 64 groups of
// 16 lanes.
constexpr int kSumThreads = 1024, kSumCols = 16;
template <GemmStore GT> __global__ void __launch_bounds__(kSumThreads) gain_sums(const float* part, int rows, int dim, void* dq, void* dk)
{
    constexpr int R = kSumThreads / kSumCols;
    __shared__ float sums[R][kSumCols + 1];
    const int x = threadIdx.x % kSumCols, group = threadIdx.x / kSumCols;
    const int col = blockIdx.x * kSumCols + x;
    float v[4] = {};
    if (col < 2 * dim) {
        for (int r = group; r < rows; r += 4 * R) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float f = part[(int64_t)min(r + j * R, rows - 1) * 2 * dim + col];
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
    if (group > 0 || col >= 2 * dim) return;
    if (col < dim) put1<GT>(dq, col, t);
    else put1<GT>(dk, col - dim, t);
}

// ---------------------------------------------------------------- host side

// Blocks of the backward pass, and rows of partial sums.
int64_t grad_blocks(int64_t tokens) { return std::max<int64_t>(1, std::min<int64_t>(ceil_div(tokens, kWaves), 1024)); }

template <bool BWD, GemmStore ST, bool INTER, Runs R, int L> int launch_l(QkArgs p, hipStream_t stream)
{
    constexpr int G = 64 / L;
    if constexpr (L <= 16) {
        if (p.hq + p.hk <= G) {
            p.slots = 1;
            while (p.slots < p.hq + p.hk) p.slots *= 2;
            // the forward pass leaves nothing behind: a wave for each of its tokens
            const int64_t blocks = BWD ? grad_blocks(p.tokens) : std::min<int64_t>(ceil_div(p.tokens * p.slots, G * kWaves), 4096);
            p.units = blocks * kWaves;
            if constexpr (BWD)
                hipLaunchKernelGGL((qk_backward_few<ST, INTER, R, L>), dim3((unsigned)blocks), dim3(kThreads), 0, stream, p);
            else
                hipLaunchKernelGGL((qk_forward_few<ST, INTER, R, L>), dim3((unsigned)blocks), dim3(kThreads), 0, stream, p);
            return launch_status();
        }
    }
    if constexpr (BWD) {
        const int64_t blocks = grad_blocks(p.tokens);
        p.units = blocks * kWaves;
        hipLaunchKernelGGL((qk_backward<ST, INTER, R, L>), dim3((unsigned)blocks, 2), dim3(kThreads), 0, stream, p);
    } else {
        // few tokens: a token's heads are shared out over several waves
        const int64_t groups = ceil_div(std::max(p.hq, p.hk), G);
        p.parts = (int32_t)std::max<int64_t>(1, std::min<int64_t>(groups, 4096 / std::max<int64_t>(1, p.tokens)));
        p.units = p.tokens * p.parts;
        const int64_t blocks = ceil_div(p.units, kWaves);
        if (!launchable(blocks, kThreads)) return HIMUON_ERR_UNSUPPORTED;
        hipLaunchKernelGGL((qk_forward<ST, INTER, R, L>), dim3((unsigned)blocks), dim3(kThreads), 0, stream, p);
    }
    return launch_status();
}

template <bool BWD, GemmStore ST, bool INTER, Runs R> int launch_runs(const QkArgs& p, int lanes, hipStream_t stream)
{
    if (lanes <= 4) return launch_l<BWD, ST, INTER, R, 4>(p, stream);
    if (lanes <= 8) return launch_l<BWD, ST, INTER, R, 8>(p, stream);
    if (lanes <= 16) return launch_l<BWD, ST, INTER, R, 16>(p, stream);
    if (lanes <= 32) return launch_l<BWD, ST, INTER, R, 32>(p, stream);
    // (32 runs hold the largest head unless both kinds have a cut one)
    if constexpr (!INTER && R != Runs::EXACT) return launch_l<BWD, ST, INTER, R, 64>(p, stream);
    return HIMUON_ERR_UNSUPPORTED;
}

// 7 x 182 tokens, 48 + 8 heads of 256 bf16, backward: EXACT 26 us, WHOLE (148 elements rotated,
// 17 lanes of 32 in use) 40, SHORT for the same 51.
template <bool BWD, GemmStore ST, bool INTER> int launch_st(const QkArgs& p, hipStream_t stream)
{
    const int turned = INTER ? p.dim / 2 : p.rot / 2, rest = p.dim / 2 - turned;
    // lanes to a head: one for each run of eight pairs
    const int lanes = (int)(ceil_div(turned, 8) + ceil_div(rest, 8));
    if (p.dim % 16 == 0 && p.rot % 16 == 0) return launch_runs<BWD, ST, INTER, Runs::EXACT>(p, lanes, stream);
    if ((turned == 0 || turned >= 8) && (rest == 0 || rest >= 8)) return launch_runs<BWD, ST, INTER, Runs::WHOLE>(p, lanes, stream);
    if constexpr (INTER) return launch_l<BWD, ST, INTER, Runs::SHORT, 4>(p, stream);  // (a head of fewer than eight pairs)
    else return launch_runs<BWD, ST, INTER, Runs::SHORT>(p, lanes, stream);
}

template <bool BWD> int launch_qk(const QkArgs& p, const himuon_qk_t* a, hipStream_t stream)
{
    if (a->dtype == HIMUON_BF16)
        return a->interleaved ? launch_st<BWD, GemmStore::BF16, true>(p, stream) : launch_st<BWD, GemmStore::BF16, false>(p, stream);
    return a->interleaved ? launch_st<BWD, GemmStore::F32, true>(p, stream) : launch_st<BWD, GemmStore::F32, false>(p, stream);
}

int check_args(const himuon_qk_t* a)
{
    if (!a || a->batch < 0 || a->seq < 0 || a->q_heads < 1 || a->k_heads < 1) return HIMUON_ERR_INVALID_ARG;
    if (a->head_dim < 2 || a->head_dim % 2 || a->rot_dim < 0 || a->rot_dim % 2 || a->rot_dim > a->head_dim)
        return HIMUON_ERR_INVALID_ARG;
    if (!known_dtype(a->dtype) || !known_dtype(a->gain_dtype) || !known_index(a->index)) return HIMUON_ERR_INVALID_ARG;
    if (!a->q_gain || !a->k_gain || a->table_rows < 0 || !(a->eps >= 0.f) || !std::isfinite(a->eps))
        return HIMUON_ERR_INVALID_ARG;
    if (a->rot_dim > 0 && a->table_rows > 0 && (!a->cos_table || !a->sin_table)) return HIMUON_ERR_INVALID_ARG;
    if (a->head_dim > HIMUON_MAX_HEAD_DIM) return HIMUON_ERR_UNSUPPORTED;
    if (a->batch > INT32_MAX || a->seq > INT32_MAX || a->table_rows > INT32_MAX) return HIMUON_ERR_UNSUPPORTED;
    if (a->batch * a->seq > INT32_MAX || (int64_t)a->q_heads + a->k_heads > kMostHeads) return HIMUON_ERR_UNSUPPORTED;
    return HIMUON_OK;
}

// An output's rows must not fall on each other.
bool distinct(const himuon_qk_t* a, const himuon_heads_t* h, int heads)
{
    return h && (a->batch < 2 || h->stride_batch) && (a->seq < 2 || h->stride_seq) && (heads < 2 || h->stride_head);
}

bool set(Strided& s, const himuon_heads_t* h)
{
    if (!h || !h->ptr) return false;
    s.ptr = static_cast<uint8_t*>(h->ptr);
    s.sb = h->stride_batch;
    s.ss = h->stride_seq;
    s.sh = h->stride_head;
    return true;
}

QkArgs common(const himuon_qk_t* a)
{
    QkArgs p{};
    p.wq = a->q_gain;
    p.wk = a->k_gain;
    p.cs = a->cos_table;
    p.sn = a->sin_table;
    p.positions = a->positions;
    p.tokens = a->batch * a->seq;
    p.seq = a->seq;
    p.table_rows = a->table_rows;
    p.hq = a->q_heads;
    p.hk = a->k_heads;
    p.dim = a->head_dim;
    p.rot = a->rot_dim;
    p.wide = a->index == HIMUON_I64;
    p.gain_bf16 = a->gain_dtype == HIMUON_BF16;
    p.parts = 1;
    p.eps = a->eps;
    p.inv_dim = 1.f / (float)a->head_dim;
    return p;
}

}  // namespace
}  // namespace himuon

extern "C" int himuon_qk_norm_rope(const himuon_qk_t* args, const himuon_heads_t* q, const himuon_heads_t* k,
                                   const himuon_heads_t* q_out, const himuon_heads_t* k_out, void* stream)
{
    using namespace himuon;
    const int st = check_args(args);
    if (st != HIMUON_OK) return st;
    if (args->batch == 0 || args->seq == 0) return HIMUON_OK;
    QkArgs p = common(args);
    if (!set(p.q, q) || !set(p.k, k) || !set(p.qo, q_out) || !set(p.ko, k_out)) return HIMUON_ERR_INVALID_ARG;
    if (!distinct(args, q_out, p.hq) || !distinct(args, k_out, p.hk)) return HIMUON_ERR_INVALID_ARG;
    StreamDevice on(stream);
    if (on.status != HIMUON_OK) return on.status;
    return launch_qk<false>(p, args, static_cast<hipStream_t>(stream));
}

extern "C" size_t himuon_qk_norm_rope_grad_workspace_size(int64_t batch, int64_t seq, int64_t head_dim)
{
    using namespace himuon;
    if (batch < 0 || seq < 0 || head_dim < 2 || head_dim > HIMUON_MAX_HEAD_DIM) return 0;
    if (batch > INT32_MAX || seq > INT32_MAX || batch * seq > INT32_MAX) return 0;
    return round_up((size_t)grad_blocks(batch * seq) * 2 * (size_t)head_dim * sizeof(float), 256);
}

extern "C" int himuon_qk_norm_rope_grad(const himuon_qk_t* args, const himuon_heads_t* g_q, const himuon_heads_t* g_k,
                                        const himuon_heads_t* q, const himuon_heads_t* k, const himuon_heads_t* dq,
                                        const himuon_heads_t* dk, void* dq_gain, void* dk_gain, void* workspace,
                                        size_t workspace_bytes, void* stream)
{
    using namespace himuon;
    int st = check_args(args);
    if (st != HIMUON_OK) return st;
    if (!dq_gain || !dk_gain) return HIMUON_ERR_INVALID_ARG;
    QkArgs p = common(args);
    // (without a token there is nothing to read: the gains' gradients become zero)
    if (p.tokens > 0 && (!set(p.gq, g_q) || !set(p.gk, g_k) || !set(p.q, q) || !set(p.k, k) || !set(p.qo, dq) || !set(p.ko, dk)))
        return HIMUON_ERR_INVALID_ARG;
    if (p.tokens > 0 && (!distinct(args, dq, p.hq) || !distinct(args, dk, p.hk))) return HIMUON_ERR_INVALID_ARG;
    if (!workspace || ((uintptr_t)workspace & 15) ||
        workspace_bytes < himuon_qk_norm_rope_grad_workspace_size(args->batch, args->seq, args->head_dim))
        return HIMUON_ERR_WORKSPACE;
    p.part = static_cast<float*>(workspace);
    StreamDevice on(stream);
    if (on.status != HIMUON_OK) return on.status;
    const hipStream_t hs = static_cast<hipStream_t>(stream);
    st = launch_qk<true>(p, args, hs);
    if (st != HIMUON_OK) return st;
    const int rows = (int)grad_blocks(p.tokens);
    const dim3 grid((unsigned)ceil_div(2 * p.dim, kSumCols));
    if (args->gain_dtype == HIMUON_BF16)
        hipLaunchKernelGGL(gain_sums<GemmStore::BF16>, grid, dim3(kSumThreads), 0, hs, p.part, rows, p.dim, dq_gain, dk_gain);
    else
        hipLaunchKernelGGL(gain_sums<GemmStore::F32>, grid, dim3(kSumThreads), 0, hs, p.part, rows, p.dim, dq_gain, dk_gain);
    return launch_status();
}
