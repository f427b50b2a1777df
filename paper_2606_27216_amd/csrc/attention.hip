// Attention over whole sequences (himuon_attention).
//
// For the queries of a sequence and the group of heads that share a key head:
//     s = c q k^T over the keys that a query sees,  o = softmax(s) v,  lse = log sum exp s
// in one pass over the keys with a running maximum m and sum l, o held unnormalised. The rows
// of a tile are (query, head of the group) pairs, so that a group's heads share the keys they
// read and short sequences fill their tiles. A wave holds 32 rows as columns of s^T = k q^T:
// a row's statistics are one lane's, and p^T is the second operand of o^T = v^T p^T as it
// stands.
//
// What bounds it: with many rows the issue of instructions, products (52% of the matrix cores' cycles; LDS is
// read in 26% of a CU's) and softmax side by side (causal bf16, heads of 128: 4 x 4096 tokens with 32 + 8 heads 542 us,
// 1.01 PFLOP/s; 16 x 1024 with 16 + 8 106, 37% and 18%; without exponentials in a trial the first took 9% less, without
// either product 18%); in fp32 the products (71% of the cycles; 8 x 1024 tokens 350 us, 98 TFLOP/s); with a query or some
// against a cache the memory (one query of each of 4 sequences against their 16384 to 32768 keys, 32 + 8 heads of 128: 99 us).
//
// bf16 probabilities are rounded to bf16 for their product with v, as the matrix cores take both operands in one type:
// results are off by 0.0021 to 0.0023 of their size (root mean square, against 64 bits), 0.0016 to 0.0017 if only they
// are rounded. fp32 arrays keep them in fp32.
#include "attn_device.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

namespace himuon {
namespace attn {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
static_assert(kTileRows == kRows * kWaves, "");

// A row's softmax as far as it has come: o unnormalised, the maximum m that its exponentials are
// relative to, their sum l (of this half's keys).
template <GemmStore ST, int DP> struct Running {
    using L = Lay<ST, DP>;
    f32x16 o[L::DT];
    float m, l, l2;  // l: in two parts

    HM_DEV void clear()
    {
#pragma unroll
        for (int t = 0; t < L::DT; ++t) o[t] = f32x16{};
        m = -INFINITY;
        l = l2 = 0.f;
    }

    // This lane's row sees the first `left` of the keys.
    static HM_DEV void hide(f32x16& s, int left, int lane)
    {
        left -= 4 * (lane >> 5);
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = result_row(i, 0) < left ? s[i] : -INFINITY;
    }
    static HM_DEV float top(const f32x16& s, float t, int from, int to)
    {
#pragma unroll
        for (int i = from; i < to; i += 2) {
            t = fmaxf(fmaxf(s[i], s[i + 1]), t);
            settle(t);
        }
        return t;
    }
    // The maximum follows once the scores leave it behind by 2^8: any value near it serves, and
    // most tiles then leave o as it is.
    HM_DEV void follow(float t, float c)
    {
        t = max_halves(t);
        if (__any(t * c > m * c + 8.f)) {
            const float now = fmaxf(m, t);
            const float f = now == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m - now) * c);
            m = now;
            l *= f;
            l2 *= f;
#pragma unroll
            for (int x = 0; x < L::DT; ++x)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[x][i] *= f;
        }
    }
    // What the exponentials are relative to.
    HM_DEV float base(float c) const { return m == -INFINITY ? 0.f : m * c; }
    // Elements [from, to) of s, an even number, to the operand p.
    HM_DEV void exponentials(const f32x16& s, Frag<ST> (&p)[2], float c, float mc, int from, int to)
    {
#pragma unroll
        for (int i = from; i < to; i += 2) {
            const float a = __builtin_amdgcn_exp2f(fmaf(s[i], c, -mc)), b = __builtin_amdgcn_exp2f(fmaf(s[i + 1], c, -mc));
            l += a;
            l2 += b;
            set_pair<ST>(p, i / 2, a, b);
            settle_pair<ST>(p, i / 2);
            settle(l);
            settle(l2);
        }
    }
    HM_DEV auto read_k(const uint8_t* kt, int lane) const
    {
        return [=](int i) __attribute__((always_inline)) { return L::row_frag(kt, lane & 31, i, lane >> 5); };
    }
    HM_DEV auto read_v(const uint8_t* vt, int lane) const
    {
        return [=](int i) __attribute__((always_inline)) { return L::col_frag(vt, 16 * (i / L::DT), 32 * (i % L::DT), lane); };
    }
};
template <GemmStore ST, int DP> using KeyFrags = Ahead<Frag<ST>, DP / 16, kDepth<ST, DP>>;
template <GemmStore ST, int DP> using ValueFrags = Ahead<Frag<ST>, DP / 16, kDepth<ST, DP>>;

// Tiles of 32 keys lie in rings of LDS buffers; a wave multiplies a tile's keys beside the
// exponentials of the tile before and that tile's values beside the next one's maximum, so that the
// matrix cores work while the vector ALU does.
template <GemmStore ST, int DP> constexpr int ring() { return Lay<ST, DP>::PITCH <= 512 ? 4 : 2; }

template <GemmStore ST, int DP, bool DMA>
__global__ void __launch_bounds__(kThreads, (Lay<ST, DP>::PITCH <= 256 ? 2 : 1)) attn_forward(const AttnArgs p)
{
    using L = Lay<ST, DP>;
    constexpr int R = ring<ST, DP>(), TILE = kRows * L::PITCH, VALUES = R * TILE;
    __shared__ __attribute__((aligned(16))) uint8_t lds[2 * R * TILE];  // [R] keys, [R] values
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x) >> 6, h = lane >> 5;
    const int G = p.group;

    const Item item = find_item<1, true>(p, blockIdx.x, gridDim.x);
    const int kh = item.kh;
    const Seq s = find_seq<false, kTileRows>(p, item.item, G);
    const int rows = s.q_cap * G, r0 = s.tile * kTileRows;  // (a sequence's rows are counted in 32 bits)
    if (r0 >= rows) return;

    const int r = r0 + wave * kRows + (lane & 31);
    const int query = (int)((uint32_t)r / (uint32_t)G);
    const int head = kh * G + (int)((uint32_t)r - (uint32_t)query * (uint32_t)G);
    const bool exists = r < rows, on = query < s.nq;

    // tiles of keys that the block's and the wave's rows see; keys seen by all of the wave's
    // rows, and by this lane's
    const int w0 = r0 + wave * kRows, in_use = s.nq * G;
    auto seen = [&](int row) { return row < in_use ? visible(p, s, (int)((uint32_t)row / (uint32_t)G)) : 0; };
    const int tiles = (seen(min(r0 + kTileRows, in_use) - 1) + kRows - 1) / kRows * (r0 < in_use);
    const int mine = (seen(min(w0 + kRows, in_use) - 1) + kRows - 1) / kRows * (w0 < in_use);
    const int n_all = seen(w0), n_lane = on ? visible(p, s, query) : 0;
    const int whole = min(tiles, s.nk / kRows);

    const int row_bytes = p.dim * L::ES;
    const uint8_t *kp = at(p.k, s.batch, s.k0, kh), *vp = at(p.v, s.batch, s.k0, kh);
    const Share<ST, DP, kRows, kThreads> share{(int)threadIdx.x};
    constexpr int NI = Share<ST, DP, kRows, kThreads>::NI;
    // The next tile of keys and of values, to its place in the ring: a whole one, or any.
    const bool exact = DMA && row_bytes == L::PITCH;
    uint32_t k_off[NI], v_off[NI];
#pragma unroll
    for (int i = 0; i < NI; ++i) {
        k_off[i] = share.offset(i, p.k.ss);
        v_off[i] = share.offset(i, p.v.ss);
    }
    auto load = [&](const uint8_t* from, int64_t stride, uint8_t* to, int t) __attribute__((always_inline)) {
        if (t >= tiles) return;
        share.template stage<DMA>(to, from + t * kRows * stride, row_bytes, t < whole, [&](int i) { return share.row(i) * stride; },
                                  [&](int i) { return t * kRows + share.row(i) < s.nk; });
    };
    auto load_k = [&](int t, int place) __attribute__((always_inline)) { load(kp, p.k.ss, lds + place * TILE, t); };
    auto load_v = [&](int t, int place) __attribute__((always_inline)) { load(vp, p.v.ss, lds + VALUES + place * TILE, t); };

    Running<ST, DP> run;
    run.clear();
    const float c = p.scale * kLog2e;
    if (tiles > 0) {
        if (DMA && p.dim < DP) {
            clear_lds<kThreads>(lds, 2 * R * TILE);
            __syncthreads();
        }
        // (values of tile t and keys of tile t + 1 travel together)
        load_k(0, 0);
#pragma unroll
        for (int t = 0; t < R - 1; ++t) {
            load_v(t, t);
            load_k(t + 1, t + 1);
        }
        Frag<ST> q[L::NS];
        load_row<DMA, ST, DP>(q, at(p.q, s.batch, s.q0 + query, head), on, p.dim, h);
        dev::dma_wait_barrier<0>();
        KeyFrags<ST, DP> fk;
        ValueFrags<ST, DP> fv;
        f32x16 x{};
        auto first_k = run.read_k(lds, lane);
        fk.fill(first_k);
        fk.run(first_k, [&](int i, const Frag<ST>& a) { mma<ST>(x, a, q[i]); });
        if (kRows > n_all) run.hide(x, n_lane, lane);
        if (mine > 0) run.follow(run.top(x, -INFINITY, 0, 16), c);
        // (a tile's place in the rings is known where it is used: its reads need no addresses of
        // their own)
        // (x: its scores, next: those of the tile behind it)
        auto step = [&](int t, auto place, f32x16& x, f32x16& next) __attribute__((always_inline)) {
            const int S = place;
            if (exact && t + R < whole) {
                dev::dma_wait_barrier<(R - 2) * 2 * NI>();
                share.copy(lds + VALUES + (S + R - 1) % R * TILE, vp + (t + R - 1) * (kRows * p.v.ss), v_off);
                share.copy(lds + S * TILE, kp + (t + R) * (kRows * p.k.ss), k_off);
            } else {
                dev::dma_wait_barrier<0>();
                load_v(t + R - 1, (S + R - 1) % R);
                load_k(t + R, S);
            }
            if (t >= mine) return;
            // (behind the wave's last tile the next scores are nothing's, and not used)
            const auto read_k = run.read_k(lds + (S + 1) % R * TILE, lane);
            const auto read_v = run.read_v(lds + VALUES + S * TILE, lane);
            const float mc = run.base(c);
            constexpr int N = L::NS, E = 4;  // E: exponentials while the first keys are on their way
            Frag<ST> pr[2];
            next = f32x16{};
            fk.fill(read_k);
            run.exponentials(x, pr, c, mc, 0, E);
            fk.run(read_k, [&](int i, const Frag<ST>& a) {
                mma<ST>(next, a, q[i]);
                run.exponentials(x, pr, c, mc, (E + (16 - E) * i / N) & ~1, (E + (16 - E) * (i + 1) / N) & ~1);
            });
            fv.fill(read_v);
            if ((t + 2) * kRows > n_all) run.hide(next, n_lane - (t + 1) * kRows, lane);
            float top = -INFINITY;
            fv.run(read_v, [&](int i, const Frag<ST>& a) {
                mma<ST>(run.o[i % L::DT], a, pr[i / L::DT]);
                top = run.top(next, top, (16 * i / N) & ~1, (16 * (i + 1) / N) & ~1);
            });
            if (t + 1 < mine) run.follow(top, c);
        };
        f32x16 y;
        if constexpr (ST == GemmStore::F32 || DP > 128) {  // (copies of the step cost registers)
            for (int t = 0; t < tiles; ++t) {
                step(t, t % R, x, y);
                x = y;
            }
        } else {
            for (int t = 0; t < tiles; t += R) {
                step(t, std::integral_constant<int, 0>{}, x, y);
                if (t + 1 < tiles) step(t + 1, std::integral_constant<int, 1>{}, y, x);
                if (t + 2 < tiles) step(t + 2, std::integral_constant<int, 2>{}, x, y);
                if (t + 3 < tiles) step(t + 3, std::integral_constant<int, 3>{}, y, x);
            }
        }
    }
    if (!exists) return;
    const float l = add_halves(run.l + run.l2);
    store_row<DMA, ST>(at(p.o, s.batch, s.q0 + query, head), run.o, on && l != 0.f, 1.f / l, p.dim, h);
    if (h == 0)
        p.lse[((int64_t)s.batch * p.q_len + s.q0 + query) * ((int64_t)p.hk * G) + head] =
            !on || l == 0.f ? -INFINITY : fmaf(run.m, p.scale, __logf(l));
}

// Few tiles: the waves of a block share 32 rows and take the keys in pieces, each with two tiles of 32
// keys of its own on the way and without a barrier; their results meet in LDS. Where the 32 rows are all
// that a group of heads has (a token or some of each sequence against many keys), the keys are
// shared out over `splits` blocks too, whose results meet in `part`: [splits] rows of DP sums and of
// {m, l}.
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
    const uint32_t w = blockIdx.x / (uint32_t)p.splits;
    const int kh = (int)(w % (uint32_t)p.hk);
    const Seq s = find_seq<false, kRows>(p, w / (uint32_t)p.hk, G);
    const int r0 = s.tile * kRows, rows = min(kRows, s.q_cap * G - r0), in_use = s.nq * G;
    if (rows <= 0) return;
    const int query = (r0 + (lane & 31)) / G, head = kh * G + r0 + (lane & 31) - query * G;
    const bool exists = (lane & 31) < rows, on = query < s.nq;
    Frag<ST> q[L::NS];
    load_row<DMA, ST, DP>(q, at(p.q, s.batch, s.q0 + query, head), on && exists, p.dim, h);

    const int n = r0 < in_use ? visible(p, s, (min(r0 + kRows, in_use) - 1) / G) : 0;  // seen by any row, by all, by this lane's
    const int n_all = visible(p, s, r0 / G), n_lane = on && exists ? visible(p, s, query) : 0;
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
        KeyFrags<ST, DP> fk;
        ValueFrags<ST, DP> fv;
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
            f32x16 x{};
            const auto read_k = run.read_k(at_k, lane);
            const auto read_v = run.read_v(at_k + TILE, lane);
            fk.fill(read_k);
            fk.run(read_k, [&](int i, const Frag<ST>& a) { mma<ST>(x, a, q[i]); });
            fv.fill(read_v);
            if ((t + 1) * kRows > n_all) run.hide(x, n_lane - t * kRows, lane);
            run.follow(run.top(x, -INFINITY, 0, 16), c);
            Frag<ST> pr[2];
            run.exponentials(x, pr, c, run.base(c), 0, 16);
            fv.run(read_v, [&](int i, const Frag<ST>& a) { mma<ST>(run.o[i % L::DT], a, pr[i / L::DT]); });
        }
    }
    run.l = add_halves(run.l + run.l2);
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
    const int token = (r0 + row) / G, hd = kh * G + r0 + row - token * G;
    const bool used = token < s.nq;
    float* const part = p.splits > 1 ? p.part + (((int64_t)w * p.splits + split) * kRows + row) * DS : nullptr;
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
    const uint32_t id = blockIdx.x * kWaves + (threadIdx.x >> 6), w = id / (uint32_t)rows;
    const int row = (int)(id - w * (uint32_t)rows), kh = (int)(w % (uint32_t)p.hk);
    if (w >= (uint32_t)p.batch * (uint32_t)p.hk) return;
    const Seq s = find_seq<false, kRows>(p, w / (uint32_t)p.hk, G);
    const float* const part = p.part + ((int64_t)w * p.splits * kRows + row) * DS;
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

template <class F> int by_dim(const AttnArgs& p, F f)
{
    if (p.dim <= 64) return f(std::integral_constant<int, 64>{});
    if (p.dim <= 128) return f(std::integral_constant<int, 128>{});
    return f(std::integral_constant<int, 256>{});
}

template <GemmStore ST, bool DMA> int launch_forward(AttnArgs p, Forward form, hipStream_t stream)
{
    return by_dim(p, [&](auto dim) {
        constexpr int DP = decltype(dim)::value;
        if (form == Forward::FEW_ROWS) {
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
        if (form == Forward::FEW_TILES) {
            constexpr int T = 64 * few_waves<ST, DP>();
            if (!set_grid<false>(p, kRows, T, &blocks)) return (int)HIMUON_ERR_UNSUPPORTED;
            StreamDevice on(stream);
            if (on.status != HIMUON_OK) return on.status;
            hipLaunchKernelGGL((attn_few<ST, DP, DMA>), dim3((unsigned)blocks), dim3(T), 0, stream, p);
            return launch_status();
        }
        if (!set_grid<false>(p, kTileRows, kThreads, &blocks)) return (int)HIMUON_ERR_UNSUPPORTED;
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
    if (!small_product(a->batch * (a->q_starts ? 1 : a->q_len), (int64_t)a->q_heads * 8) || !small_product(a->batch, a->k_len))
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
// 16-byte aligned, or a sequence's too far apart for 32-bit offsets.
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
    // (offsets in a sequence, and in a tile of 64 rows)
    if (t.ss < 0 || t.sh < 0 || t.ss > INT64_C(1) << 24 || t.sh > INT64_C(1) << 30 || tokens * t.ss + group * t.sh > UINT32_MAX - (INT64_C(1) << 28))
        *dma = false;
    return true;
}

}  // namespace attn
}  // namespace himuon

extern "C" size_t himuon_attention_workspace_size(const himuon_attn_t* args)
{
    using namespace himuon;
    using namespace himuon::attn;
    if (check_attn(args) != HIMUON_OK || empty_batch(args) || args->q_len == 0 || !few_rows(*args)) return 0;
    const int64_t splits = few_splits(*args);
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
    if (p.o.ptr == p.q.ptr || p.o.ptr == p.k.ptr || p.o.ptr == p.v.ptr) return HIMUON_ERR_INVALID_ARG;
    p.lse = lse;
    const Forward form = plan_forward(*args);
    if (form == Forward::FEW_ROWS) p.splits = (int32_t)few_splits(*args);
    const size_t need = himuon_attention_workspace_size(args);
    if (need > 0 && (!workspace || ((uintptr_t)workspace & 15) || workspace_bytes < need)) return HIMUON_ERR_WORKSPACE;
    p.part = static_cast<float*>(workspace);
    const hipStream_t hs = static_cast<hipStream_t>(stream);
    if (args->dtype == HIMUON_BF16)
        return dma ? launch_forward<GemmStore::BF16, true>(p, form, hs) : launch_forward<GemmStore::BF16, false>(p, form, hs);
    return dma ? launch_forward<GemmStore::F32, true>(p, form, hs) : launch_forward<GemmStore::F32, false>(p, form, hs);
}
