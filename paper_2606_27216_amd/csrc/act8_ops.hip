// Activations in 8 bits (himuon_act_pack, himuon_act_unpack) and the weight gradient
// that reads them (himuon_weight_grad).
//
// 32 tokens of a column share an exponent e, the least with max |x| <= 448 2^e; codes
// are 8-bit floats with 3 mantissa bits, so code * 2^e has 4 significant bits and is exact
// in bf16. A group lies along the weight gradient's sum, and a column's 32 codes are
// adjacent: they are the operand of 32 consecutive terms as they stand in memory.
#include "lds_dma.h"
#include "ns_device.h"
#include "train_ops.h"
#include "wgrad_plan.h"

#include <algorithm>
#include <type_traits>

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
// The codes cross LDS, so that a store writes 1 KB in a row: with each lane storing its own
// columns' 16-byte pieces, 8192 x 11008 bf16 took 71 us, so 57 (273 MB, 4.8 TB/s).
template <GemmStore ST>
__global__ void __launch_bounds__(kThreads) act_pack(const void* x, int64_t ld, int64_t tokens, int64_t cols, int64_t slabs,
                                                     int64_t units, uint8_t* codes, uint8_t* exps)
{
    constexpr int N = kCols<ST>;
    __shared__ u32x4 turn[kThreads / 64][64 * 2 * N];
    const int64_t unit = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
    if (unit >= units) return;
    const int lane = threadIdx.x & 63;
    u32x4* const mine = turn[threadIdx.x >> 6];
    const int64_t tb = unit / slabs;
    const int64_t c0 = (unit - tb * slabs) * (64 * N);
    // The last lane's columns end with the last column, and begin with `skip` of the lane
    // before it, which it does not store (nor does a lane past the last column any).
    const int64_t c = min(c0 + lane * N, max(cols - N, (int64_t)0));
    const int n = (int)min((int64_t)N, cols);
    const int skip = (int)min(c0 + lane * N - c, (int64_t)N);
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
        // piece h of the lane's own column j: at 2 N lane + 2 j + h, moved within its lane's
        // pieces so that the lanes of one access lie in different banks
        if (j >= skip) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
                mine[2 * N * lane + ((2 * (j - skip) + h) ^ (lane & (2 * N - 1)))] =
                    u32x4{q[4 * h], q[4 * h + 1], q[4 * h + 2], q[4 * h + 3]};
            if (j < n) exps[tb * cols + c + j] = (uint8_t)code;
        }
    }
    wave_exchange();
    u32x4* const dst = reinterpret_cast<u32x4*>(codes + (tb * cols + c0) * kGroup);
    const int pieces = 2 * (int)min((int64_t)(64 * N), cols - c0);
#pragma unroll
    for (int s = 0; s < 2 * N; ++s) {
        const int x = 64 * s + lane, owner = x / (2 * N);
        if (x < pieces) dst[x] = mine[2 * N * owner + ((x % (2 * N)) ^ (owner & (2 * N - 1)))];
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

// dweight = grad^T x: tokens are the sum's index. A workgroup owns a BM x BN tile of the
// result and walks over the tokens in slices of 32, one group of codes. Both operands go
// to LDS as they lie in memory, by DMA (global_load_lds) into a ring of NS slices with
// one barrier a slice:
//   - the gradient, 32 rows of BM bf16, in panels of 64 columns; ds_read_b64_tr_b16
//     turns 4 tokens x 16 columns on the way to the registers, so no pass transposes it;
//   - the codes, a column's 32 bytes, 16 of them to a lane: no transposition at all;
//   - the exponents, a byte a column.
// A wave widens codes to bf16 between the products, two to an instruction and the
// exponent applied by the same one; that is exact. The k index of a product is permuted
// alike in both operands: lane half h has tokens 16 h .. 16 h + 15 of the slice.
//
// An fp32 gradient, or one whose rows do not start on 16 bytes, is first laid out in the
// workspace as slices of bf16 rows, fp32 as three terms that follow each other (the
// codes' slice is then read three times in a row, from cache).
//
// Bound by the matrix cores under the board's power cap: 8192 x 11008 x 4096 takes 551 to 578
// us, 1.28 to 1.34 PFLOP/s (a large library product reaches 1.25 to 1.40 on the card, the
// library's bf16 product of this shape 0.9). The cores are busy for 68% of the launch's cycles: 688
// tiles of 256 are 2.7 rounds of the chip, and a slice takes longer than its 1024 cycles of
// products. Eight waves of 128 x 64 to a tile against four of 128 x 128 (560) and of 256 x 64,
// which widen each code once instead of twice (556); a ring of four or six slices 557.
struct WgradArgs {
    const uint16_t* a;           // gradient, or its terms in the workspace
    const uint8_t *codes, *exps;
    void* out;
    float* part;                 // [splits][rows][part_pitch] partial sums (splits > 1)
    int64_t lda, lde, ld_out, part_pitch;
    int32_t rows, cols;
    int32_t a_cols;              // columns of `a`, a multiple of 8
    int32_t slices, terms;       // slices in all; consecutive ones that share their codes
    int32_t tail;                // rows of the last slice, if fewer than 32 (else 0)
    int32_t splits, ti, tj, accumulate;
};

// Four consecutive results from column j on, of which n exist.
template <GemmStore OT> HM_DEV void put_result(void* out, int64_t i, int n, bool accumulate, f32x4 v)
{
    if (accumulate) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < n) v[e] += get1<OT>(out, i + e);
    }
    if (n == 4) {
        if constexpr (OT == GemmStore::BF16)
            *reinterpret_cast<u32x2_any16*>(static_cast<uint16_t*>(out) + i) =
                u32x2{pack2<Operand::BF16>(v[0], v[1]), pack2<Operand::BF16>(v[2], v[3])};
        else
            *reinterpret_cast<f32x4_any32*>(static_cast<float*>(out) + i) = v;
    } else {
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (e < n) put1<OT>(out, i + e, v[e]);
    }
}

// KG = 2: a workgroup has two such groups of waves, which share its slices out between them
// and add their sums up in LDS at the end.
template <GemmStore OT, int BM, int BN, int WGM, int WGN, int KG, int NS, int MINW>
__global__ void __launch_bounds__(64 * WGM * WGN * KG, MINW) wgrad_blocks(const WgradArgs p)
{
    constexpr int W = WGM * WGN;
    constexpr int RB = BM / 32 / WGM, CB = BN / 32 / WGN;  // 32-blocks of a wave
    static_assert(RB % 2 == 0, "whole panels to a wave");
    constexpr int ABYTES = BM * 64, BBYTES = BN * 32;
    constexpr int STAGE = ABYTES + BBYTES + W * 256;
    constexpr int AI = BM / 16 / W, BI = BN / 32 / W, NI = AI + BI + 1;  // DMA instructions per wave and slice
    static_assert(AI * 16 * W == BM && BI * 32 * W == BN, "whole DMA instructions");
    static_assert((NS - 2) * NI < 64, "the wait's counter");
    constexpr int PITCH = CB * 128 + 16;  // bytes of a row of results in LDS
    static_assert(KG == 1 || (KG == 2 && RB == 2), "each group finishes one of a wave's two block rows");
    constexpr int MEET = KG == 1 ? 0 : KG * W * CB * 4096;  // the groups' exchange
    constexpr int OUT = MEET + KG * W * 32 * PITCH, RING = STAGE * NS;
    __shared__ __attribute__((aligned(1024))) uint8_t lds_all[KG * RING > OUT ? KG * RING : OUT];

    const int lane = threadIdx.x & 63;
    const int group = KG == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / (64 * W));
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) - group * W;
    uint8_t* const lds = lds_all + group * RING;
    const int li = lane & 31, lh = lane >> 5, g16 = lane >> 4;
    const int wi = (wave / WGN) * RB * 32, wj = (wave % WGN) * CB * 32;

    // Workgroups go to the eight XCDs in turn; each XCD gets a contiguous run of tiles, in
    // bands of four tile rows, so that its tiles share operands in its L2.
    int split, i0, j0;
    {
        const int tiles = p.ti * p.tj, total = tiles * p.splits;
        const int b = blockIdx.x, x = b & 7, per = total >> 3, rem = total & 7;
        const int t = x * per + min(x, rem) + (b >> 3);
        split = t / tiles;
        int r = t - split * tiles;
        const int band = r / (4 * p.tj), h = min(4, p.ti - 4 * band);
        r -= band * 4 * p.tj;
        const int tj = r / h;
        i0 = (4 * band + (r - tj * h)) * BM;
        j0 = tj * BN;
    }
    // whole slices of the workgroup, of this group of waves, and the most of any group
    const int all0 = (int)((int64_t)p.slices * split / p.splits), all1 = (int)((int64_t)p.slices * (split + 1) / p.splits);
    const bool tail = p.tail != 0 && all1 == p.slices;
    const int all = all1 - all0 - (tail ? 1 : 0);
    const int s0 = all0 + all * group / KG, nk = all0 + all * (group + 1) / KG - s0, most = (all + KG - 1) / KG;

    // DMA sources. Gradient: instruction q of a wave fills 8 rows of a panel (128 bytes
    // each); the 64-byte halves of rows 2, 3, 6, 7, .. change places, so that a
    // transposing read's four rows lie in different banks. Columns past the last read
    // the last ones (their results are not stored).
    uint32_t va[AI], vb[BI];
    auto a_offset = [&](int q, int rows) -> uint32_t {
        const int u = q * W + wave;
        const int row = 8 * (u & 3) + (lane >> 3);
        const int col = 64 * (u >> 2) + 8 * ((lane & 7) ^ (4 * ((row >> 1) & 1)));
        return (uint32_t)min(row, rows - 1) * (uint32_t)(p.lda * 2) + 2u * (uint32_t)min(col, p.a_cols - 8 - i0);
    };
#pragma unroll
    for (int q = 0; q < AI; ++q) va[q] = a_offset(q, kGroup);
#pragma unroll
    for (int q = 0; q < BI; ++q) {
        const int col = 32 * (q * W + wave) + li;
        vb[q] = 32u * (uint32_t)min(col, p.cols - 1 - j0) + 16u * lh;
    }
    const int e0 = min(j0 + wj, (int)p.lde - 4);
    const uint32_t ve = (uint32_t)min(4 * lane, (int)p.lde - 4 - e0);
    const uint16_t* a_base = p.a + (int64_t)s0 * kGroup * p.lda + i0;
    const uint8_t* b_base = p.codes + ((int64_t)(s0 / p.terms) * p.cols + j0) * kGroup;
    const uint8_t* e_base = p.exps + (int64_t)(s0 / p.terms) * p.lde + e0;
    int term = s0 % p.terms;
    const uint32_t lds0 = lds_offset(lds);
    // DMA instruction q of the next slice, into ring buffer `buf`
    auto issue1 = [&](int buf, int q) {
        const uint32_t d = __builtin_amdgcn_readfirstlane(lds0 + buf * STAGE);
        if (q < AI) dma16(d + (q * W + wave) * 1024, va[q < AI ? q : 0], uniform_address(a_base));
        else if (q < AI + BI) dma16(d + ABYTES + ((q - AI) * W + wave) * 1024, vb[q < AI || q >= AI + BI ? 0 : q - AI], uniform_address(b_base));
        else dma4(d + ABYTES + BBYTES + wave * 256, ve, uniform_address(e_base));
    };
    auto advance = [&]() {
        a_base += (int64_t)kGroup * p.lda;
        if (++term == p.terms) {
            term = 0;
            b_base += (int64_t)p.cols * kGroup;
            e_base += p.lde;
        }
    };

    f32x16 acc[RB][CB];
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int j = 0; j < CB; ++j) acc[i][j] = f32x16{};

    // A slice is two steps of 16 tokens. The operands of a step are read while the step
    // before it is multiplied.
    u32x4 fa[2][RB], fb[2][CB], raw[CB];
    uint32_t scale[CB];
    const int arow = (16 * lh + ((lane & 15) >> 2)) * 128, acol = 32 * (g16 & 1) + 8 * (lane & 3), aswap = 64 * ((lane >> 3) & 1);
    const int ra[2] = {arow + (acol ^ aswap), arow + ((acol + 64) ^ aswap)};
    // half x of the operand of step s: four tokens a lane
    auto load_a = [&](const uint8_t* ta, int s, int i, int x) __attribute__((always_inline)) {
        const u32x2 v = tr_read(ta + ((wi >> 6) + (i >> 1)) * 4096 + 1024 * s + 512 * x + ra[i & 1]);
        fa[s][i][2 * x] = v[0];
        fa[s][i][2 * x + 1] = v[1];
    };
    auto load_b = [&](const uint8_t* ta, int j) __attribute__((always_inline)) {
        raw[j] = *reinterpret_cast<const u32x4*>(ta + ABYTES + (wj / 32 + j) * 1024 + lane * 16);
    };
    auto load_scale = [&](const uint8_t* ta, int j) __attribute__((always_inline)) {
        scale[j] = ta[ABYTES + BBYTES + wave * 256 + 32 * j + li];
    };
    auto widen = [&](int s, int j, int x) __attribute__((always_inline)) {
        const float f = __uint_as_float(scale[j] << 23);
        const uint32_t w = raw[j][2 * s + x];
        fb[s][j][2 * x] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, f, false));
        fb[s][j][2 * x + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, f, true));
    };
    // What goes out beside the products is spread over them, two or three instructions to each:
    // a product takes the matrix core 32 cycles, and a wave that issues ten others in one gap
    // leaves it idle (8192 x 4096 x 4096, four waves to a tile: bunched 223 us, spread 214).
    constexpr int PROD = RB * CB, HALF = PROD / 2;
    // the products of step 0 beside the operands of step 1
    auto first = [&](const uint8_t* ta) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < PROD; ++e) {
#pragma unroll
            for (int o = 0; o < 2 * RB; ++o)
                if (o * PROD / (2 * RB) == e) load_a(ta, 1, o >> 1, o & 1);
#pragma unroll
            for (int o = 0; o < 2 * CB; ++o)
                if ((2 * o + 1) * PROD / (4 * CB) == e) widen(1, o >> 1, o & 1);
            acc[e / CB][e % CB] = mma1<Operand::BF16>(fb[0][e % CB], fa[0][e / CB], acc[e / CB][e % CB]);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // the products of step 1 beside the next slice's operands (more) and the DMA into the
    // buffer that has become free (refill)
    auto second = [&](const uint8_t* ta, auto more, auto refill, int dst) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < PROD; ++e) {
            if constexpr (decltype(more)::value) {
#pragma unroll
                for (int o = 0; o < 2 * CB; ++o) {
                    if (o * HALF / (2 * CB) == e) {
                        if (o & 1) load_b(ta, o >> 1);
                        else load_scale(ta, o >> 1);
                    }
                    if (HALF + o * HALF / (2 * CB) == e) widen(0, o >> 1, o & 1);
                }
#pragma unroll
                for (int o = 0; o < 2 * RB; ++o)
                    if (HALF + o * HALF / (2 * RB) == e) load_a(ta, 0, o >> 1, o & 1);
            }
            acc[e / CB][e % CB] = mma1<Operand::BF16>(fb[1][e % CB], fa[1][e / CB], acc[e / CB][e % CB]);
            if constexpr (decltype(refill)::value) {
#pragma unroll
                for (int q = 0; q < NI; ++q)
                    if ((NI <= HALF ? q * HALF / NI : q * PROD / NI) == e) issue1(dst, q);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        if constexpr (decltype(refill)::value) advance();
    };
    auto load_first = [&](const uint8_t* ta) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < CB; ++j) {
            load_scale(ta, j);
            load_b(ta, j);
        }
#pragma unroll
        for (int o = 0; o < 2 * RB; ++o) load_a(ta, 0, o >> 1, o & 1);
#pragma unroll
        for (int o = 0; o < 2 * CB; ++o) widen(0, o >> 1, o & 1);
    };
    constexpr std::true_type yes{};
    constexpr std::false_type no{};

    if (nk > 0) {
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            if (s < nk) {
#pragma unroll
                for (int q = 0; q < NI; ++q) issue1(s, q);
                advance();
            }
        }
        if (nk >= NS) dma_wait_barrier<(NS - 1) * NI < 63 ? (NS - 1) * NI : 63>();
        else dma_wait_barrier<0>();
        load_first(lds);
        int buf = 0, k = 0;
        auto slice = [&](auto more, auto refill) __attribute__((always_inline)) {
            const int nbuf = buf + 1 == NS ? 0 : buf + 1;
            first(lds + buf * STAGE);
            // slice k + 1 has landed; every wave has read slice k
            if constexpr (decltype(more)::value) dma_wait_barrier<decltype(refill)::value ? (NS - 2) * NI : 0>();
            second(lds + nbuf * STAGE, more, refill, buf);
            buf = nbuf;
        };
        for (; k < nk - NS; ++k) slice(yes, yes);
        for (; k < nk - 1; ++k) slice(yes, no);
        slice(no, no);
    }
    if constexpr (KG > 1) {  // (a barrier a slice: the group with fewer slices keeps the other's count)
        for (int k = nk; k < most; ++k) dma_wait_barrier<0>();
    }
    // The last slice is cut: rows past the last token become zeros in LDS. (It is the last
    // group's, whose sources stand behind its last whole slice; other groups read along.)
    if (tail) {
        dma_wait_barrier<0>();
#pragma unroll
        for (int q = 0; q < AI; ++q) va[q] = a_offset(q, p.tail);
        if (group == KG - 1) {
#pragma unroll
            for (int q = 0; q < NI; ++q) issue1(0, q);
        }
        dma_wait_barrier<0>();
        for (int x = threadIdx.x % (64 * W); x < BM / 64 * (kGroup - p.tail) * 8; x += 64 * W) {
            const int c = x & 7, r = p.tail + (x >> 3) % (kGroup - p.tail), panel = (x >> 3) / (kGroup - p.tail);
            *reinterpret_cast<u32x4*>(lds + panel * 4096 + r * 128 + c * 16) = u32x4{};
        }
        __syncthreads();
        if (group == KG - 1) {
            load_first(lds);
            first(lds);
            second(lds, no, no, 0);
        }
    }

    dma_wait_barrier<0>();
    if constexpr (KG == 2) {
        // group g finishes block row g of each wave: it leaves the other one to its partner
        f32x4* const meet = reinterpret_cast<f32x4*>(lds_all);
        auto leave = [&](const f32x16 (&v)[CB]) __attribute__((always_inline)) {
#pragma unroll
            for (int j = 0; j < CB; ++j)
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    meet[(((group * W + wave) * CB + j) * 4 + g) * 64 + lane] = f32x4{v[j][4 * g], v[j][4 * g + 1], v[j][4 * g + 2], v[j][4 * g + 3]};
        };
        auto take = [&](f32x16 (&v)[CB]) __attribute__((always_inline)) {
#pragma unroll
            for (int j = 0; j < CB; ++j)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const f32x4 w = meet[((((group ^ 1) * W + wave) * CB + j) * 4 + g) * 64 + lane];
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[j][4 * g + e] += w[e];
                }
        };
        if (group == 0) leave(acc[1]);
        else leave(acc[0]);
        __syncthreads();
        if (group == 0) take(acc[0]);
        else take(acc[1]);
    }
    // Results through LDS, 32 rows of a wave at a time, so that stores are whole rows.
    uint8_t* const mine = lds_all + MEET + (group * W + wave) * 32 * PITCH;
    constexpr int LR = CB * 8;  // lanes to a row
#pragma unroll
    for (int i = 0; i < RB; ++i) {
        if (KG == 2 && i != group) continue;
#pragma unroll
        for (int j = 0; j < CB; ++j)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<f32x4*>(mine + li * PITCH + (32 * j + 8 * g + 4 * lh) * 4) =
                    f32x4{acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
        wave_exchange();
#pragma unroll 4
        for (int r = lane / LR; r < 32; r += 64 / LR) {
            const f32x4 v = *reinterpret_cast<const f32x4*>(mine + r * PITCH + (lane % LR) * 16);
            const int o = i0 + wi + 32 * i + r, j = j0 + wj + 4 * (lane % LR);
            if (o >= p.rows || j >= p.cols) continue;
            if (p.splits > 1)  // (rows of whole 16 bytes)
                *reinterpret_cast<f32x4*>(p.part + ((int64_t)split * p.rows + o) * p.part_pitch + j) = v;
            else
                put_result<OT>(p.out, (int64_t)o * p.ld_out + j, min(4, p.cols - j), p.accumulate != 0, v);
        }
        wave_exchange();
    }
}

// Small results: a 64 x 64 tile to a workgroup of eight waves that share the tokens out
// (wave w has groups w, w + 8, ..), each with the whole tile in registers. The operands
// come straight from memory in the products' own layout: a lane's 16 tokens of a row of
// the gradient are 16 loads of one element (32 lanes side by side), its 16 codes one load. No
// LDS, no barrier and no second layout of the gradient on the way, whatever its type and
// alignment; fp32 is cut into its three terms in registers. The waves' sums meet in LDS.
// 1111 x 1003 x 777: fp32 13 us with the call, 12 of them on the chip; bound by the latency of
// five groups in a row and by the cutting.
constexpr int kDirectWaves = 8;

template <GemmStore ST, GemmStore OT> __global__ void __launch_bounds__(64 * kDirectWaves, 2) wgrad_direct(const WgradArgs p)
{
    constexpr int TERMS = ST == GemmStore::F32 ? 3 : 1;
    constexpr int PITCH = 64 + 4;
    using Elem = typename std::conditional<ST == GemmStore::F32, uint32_t, uint16_t>::type;
    __shared__ __attribute__((aligned(16))) float sums[kDirectWaves][64][PITCH];
    const int lane = threadIdx.x & 63, li = lane & 31, lh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tiles = p.ti * p.tj;
    const int split = blockIdx.x / tiles, r = blockIdx.x - split * tiles;
    const int i0 = (r / p.tj) * 64, j0 = (r % p.tj) * 64;
    const int g0 = (int)((int64_t)p.slices * split / p.splits), g1 = (int)((int64_t)p.slices * (split + 1) / p.splits);

    // one group's operands: the gradient's elements [block][token], codes and exponents
    struct Group {
        uint32_t a[2][16];
        u32x4 b[2];
        uint32_t e[2];
    };
    // offsets of the lane's 16 tokens of block 0, from there to block 1; columns past the
    // last read the last one (their results are not stored)
    const uint32_t pitch = (uint32_t)(p.lda * (int64_t)sizeof(Elem));
    const uint32_t a0 = (uint32_t)min(i0 + li, p.rows - 1) * (uint32_t)sizeof(Elem);
    const uint32_t a1 = (uint32_t)min(i0 + 32 + li, p.rows - 1) * (uint32_t)sizeof(Elem) - a0;
    const uint32_t c0 = (uint32_t)min(j0 + li, p.cols - 1), c1 = (uint32_t)min(j0 + 32 + li, p.cols - 1);
    uint32_t off[16];
#pragma unroll
    for (int k = 0; k < 16; ++k) off[k] = a0 + (uint32_t)(16 * lh + k) * pitch;
    const uint8_t* const grad = reinterpret_cast<const uint8_t*>(p.a);
    auto load = [&](Group& g, int t) __attribute__((always_inline)) {
        const bool cut = p.tail && t == p.slices - 1;
        if (cut) {  // tokens past the last one read the last and become zeros
#pragma unroll
            for (int k = 0; k < 16; ++k) off[k] = a0 + (uint32_t)min(16 * lh + k, p.tail - 1) * pitch;
        }
        const uint8_t* const base = grad + (int64_t)t * kGroup * pitch;
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            g.a[0][k] = *reinterpret_cast<const Elem*>(base + off[k]);
            g.a[1][k] = *reinterpret_cast<const Elem*>(base + (off[k] + a1));
        }
        const int64_t c = (int64_t)t * p.cols;
        const uint8_t* const codes = p.codes + c * kGroup;
        const uint8_t* const exps = p.exps + c;
        g.b[0] = *reinterpret_cast<const u32x4*>(codes + (32u * c0 + 16u * lh));
        g.b[1] = *reinterpret_cast<const u32x4*>(codes + (32u * c1 + 16u * lh));
        g.e[0] = exps[c0];
        g.e[1] = exps[c1];
        if (cut) {
#pragma unroll
            for (int k = 0; k < 16; ++k) {
                g.a[0][k] = 16 * lh + k < p.tail ? g.a[0][k] : 0u;
                g.a[1][k] = 16 * lh + k < p.tail ? g.a[1][k] : 0u;
            }
        }
    };
    f32x16 acc[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[i][j] = f32x16{};
    auto multiply = [&](const Group& g) __attribute__((always_inline)) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            u32x4 b[2], a[TERMS][2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float f = __uint_as_float(g.e[j] << 23);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    b[j][e] = __builtin_bit_cast(uint32_t, (e & 1) ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(g.b[j][2 * s + e / 2], f, true)
                                                                   : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(g.b[j][2 * s + e / 2], f, false));
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t x = g.a[i][8 * s + 2 * e], y = g.a[i][8 * s + 2 * e + 1];
                    if constexpr (TERMS == 1) {
                        a[0][i][e] = x | y << 16;
                    } else {
                        float u = __uint_as_float(x), v = __uint_as_float(y);
#pragma unroll
                        for (int k = 0; k < TERMS; ++k) {
                            const float hu = __uint_as_float(__float_as_uint(u) & 0xffff0000u), hv = __uint_as_float(__float_as_uint(v) & 0xffff0000u);
                            a[k][i][e] = __builtin_amdgcn_perm(__float_as_uint(v), __float_as_uint(u), 0x07060302u);
                            // (an infinity has no rest, NaN keeps one; a rest is no infinity)
                            u = k == 0 && u == hu ? 0.f : u - hu;
                            v = k == 0 && v == hv ? 0.f : v - hv;
                        }
                    }
                }
#pragma unroll
            for (int k = 0; k < TERMS; ++k)
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j) acc[i][j] = mma1<Operand::BF16>(b[j], a[k][i], acc[i][j]);
        }
    };
    Group cur, next;
    const int n = g1 > g0 + wave ? (g1 - g0 - wave + kDirectWaves - 1) / kDirectWaves : 0;
    if (n > 0) load(next, g0 + wave);
#pragma unroll 1
    for (int k = 0; k < n; ++k) {  // (a uniform count, so that addresses stay in scalar registers)
        cur = next;
        if (k + 1 < n) load(next, g0 + wave + (k + 1) * kDirectWaves);
        multiply(cur);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<f32x4*>(&sums[wave][32 * i + li][32 * j + 8 * g + 4 * lh]) =
                    f32x4{acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
    __syncthreads();
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        const int q = threadIdx.x + x * 64 * kDirectWaves;
        const int o = q / 16, c = (q % 16) * 4;
        f32x4 v = *reinterpret_cast<const f32x4*>(&sums[0][o][c]);
#pragma unroll
        for (int w = 1; w < kDirectWaves; ++w) {
            const f32x4 u = *reinterpret_cast<const f32x4*>(&sums[w][o][c]);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += u[e];
        }
        if (i0 + o >= p.rows || j0 + c >= p.cols) continue;
        if (p.splits > 1)
            *reinterpret_cast<f32x4*>(p.part + ((int64_t)split * p.rows + i0 + o) * p.part_pitch + j0 + c) = v;
        else
            put_result<OT>(p.out, (int64_t)(i0 + o) * p.ld_out + j0 + c, min(4, p.cols - j0 - c), p.accumulate != 0, v);
    }
}

// Adds the splits' partial sums up in order.
template <GemmStore OT> __global__ void __launch_bounds__(kThreads) wgrad_join(const WgradArgs p)
{
    const int64_t per = p.part_pitch / 4, n = per * p.rows;
    for (int64_t x = (int64_t)blockIdx.x * kThreads + threadIdx.x; x < n; x += (int64_t)gridDim.x * kThreads) {
        const int64_t o = x / per;
        const int j = (int)(x - o * per) * 4;
        const float* const src = p.part + o * p.part_pitch + j;
        f32x4 v = *reinterpret_cast<const f32x4*>(src);
        for (int s = 1; s < p.splits; ++s) {
            const f32x4 w = *reinterpret_cast<const f32x4*>(src + (int64_t)s * p.rows * p.part_pitch);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += w[e];
        }
        put_result<OT>(p.out, o * p.ld_out + j, min(4, p.cols - j), p.accumulate != 0, v);
    }
}

struct StageArgs {
    const void* grad;       // laid out as slices of bf16 rows, if chunks > 0
    const uint8_t* exps;    // laid out in rows of whole 4 bytes, if exp_bytes > 0
    uint16_t* a;
    uint8_t* e;
    int64_t ld, tokens, chunks, exp_bytes;
    int32_t rows, pitch, cols, exp_pitch, grad_blocks;
};

// What a product cannot read where it lies. The gradient: [slice][32][pitch], fp32 as three
// terms of 8 bits each (x = h + m + l, cut, not rounded: all 24 bits, but none below 2^-133, the last
// one of bf16; infinities and NaN in the first alone); rows past the last token and columns past the last are zeros.
template <GemmStore ST> __global__ void __launch_bounds__(kThreads) stage_operands(const StageArgs p)
{
    if ((int)blockIdx.x >= p.grad_blocks) {
        const int64_t step = (int64_t)(gridDim.x - p.grad_blocks) * kThreads;
        for (int64_t x = (int64_t)(blockIdx.x - p.grad_blocks) * kThreads + threadIdx.x; x < p.exp_bytes; x += step) {
            const int64_t r = x / p.exp_pitch;
            const int c = (int)(x - r * p.exp_pitch);
            p.e[x] = p.exps[r * p.cols + min(c, p.cols - 1)];
        }
        return;
    }
    constexpr int TERMS = ST == GemmStore::F32 ? 3 : 1;
    const int per = p.pitch / 8;
    for (int64_t x = (int64_t)blockIdx.x * kThreads + threadIdx.x; x < p.chunks; x += (int64_t)p.grad_blocks * kThreads) {
        const int64_t t = x / per;
        const int o = (int)(x - t * per) * 8;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = 0.f;
        if (t < p.tokens) load8<ST>(p.grad, t * p.ld + o, min(8, p.rows - o), false, v);
#pragma unroll
        for (int k = 0; k < TERMS; ++k) {
            uint32_t h[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                uint32_t top = __float_as_uint(v[e]) & 0xffff0000u;
                if (v[e] != v[e]) top = 0x7fc00000u;
                h[e] = top >> 16;
                v[e] = (top & kInf) == kInf ? 0.f : v[e] - __uint_as_float(top);
            }
            const int64_t row = ((t / kGroup) * TERMS + k) * kGroup + t % kGroup;
            *reinterpret_cast<u32x4*>(p.a + row * p.pitch + o) =
                u32x4{h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16};
        }
    }
}

int act_sizes(int64_t tokens, int64_t cols)
{
    if (tokens < 0 || cols < 1) return HIMUON_ERR_INVALID_ARG;
    if (tokens > INT32_MAX / 4 || cols > (INT32_MAX >> 5) - 4096) return HIMUON_ERR_UNSUPPORTED;
    return HIMUON_OK;
}

int wgrad_sizes(int64_t tokens, int64_t out, int64_t cols)
{
    if (out < 1) return HIMUON_ERR_INVALID_ARG;
    if (out >= (INT32_MAX >> 5) - 4096) return HIMUON_ERR_UNSUPPORTED;
    return act_sizes(tokens, cols);
}

template <GemmStore OT> int join_splits(const WgradArgs& p, hipStream_t stream)
{
    const int st = launch_status();
    if (st != HIMUON_OK || p.splits == 1) return st;
    const int64_t blocks = std::min<int64_t>(ceil_div(p.part_pitch / 4 * p.rows, kThreads), 8192);
    hipLaunchKernelGGL(wgrad_join<OT>, dim3((unsigned)blocks), dim3(kThreads), 0, stream, p);
    return launch_status();
}

template <GemmStore OT, int BM, int BN, int WGM, int WGN, int KG, int NS, int MINW> int launch_tiles(WgradArgs p, hipStream_t stream)
{
    p.ti = (int32_t)ceil_div(p.rows, BM);
    p.tj = (int32_t)ceil_div(p.cols, BN);
    const int64_t total = (int64_t)p.ti * p.tj * p.splits;
    static_assert(64 * WGM * WGN * KG == (BM == 128 && KG == 1 ? 256 : 512), "tiles_launchable's threads");
    hipLaunchKernelGGL((wgrad_blocks<OT, BM, BN, WGM, WGN, KG, NS, MINW>), dim3((unsigned)total), dim3(64 * WGM * WGN * KG), 0,
                       stream, p);
    return join_splits<OT>(p, stream);
}

template <GemmStore OT> int launch_wgrad(WgradArgs p, Tile tile, int dtype, hipStream_t stream)
{
    // (rings: 130 KB, 104 KB and three times 52 KB of a CU's 160 KB)
    if (tile == Tile::B256) return launch_tiles<OT, 256, 256, 2, 4, 1, 5, 2>(p, stream);
    if (tile == Tile::B128_PAIR) return launch_tiles<OT, 128, 128, 2, 2, 2, 4, 2>(p, stream);
    if (tile == Tile::B128) return launch_tiles<OT, 128, 128, 2, 2, 1, 4, 2>(p, stream);
    p.ti = (int32_t)ceil_div(p.rows, 64);
    p.tj = (int32_t)ceil_div(p.cols, 64);
    const dim3 grid((unsigned)(p.ti * p.tj * p.splits));
    if (dtype == HIMUON_BF16)
        hipLaunchKernelGGL((wgrad_direct<GemmStore::BF16, OT>), grid, dim3(64 * kDirectWaves), 0, stream, p);
    else
        hipLaunchKernelGGL((wgrad_direct<GemmStore::F32, OT>), grid, dim3(64 * kDirectWaves), 0, stream, p);
    return join_splits<OT>(p, stream);
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
    if (!launchable(blocks, kThreads)) return HIMUON_ERR_UNSUPPORTED;
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
    if (!launchable(blocks, kThreads)) return HIMUON_ERR_UNSUPPORTED;
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

extern "C" size_t himuon_weight_grad_workspace_size(int64_t n_tokens, int64_t out, int64_t cols, const void* grad,
                                                    int64_t ld_grad, int dtype)
{
    using namespace himuon;
    if (wgrad_sizes(n_tokens, out, cols) != HIMUON_OK || !known_dtype(dtype) || ld_grad < out) return 0;
    const WgradPlan g = plan_wgrad(n_tokens, out, cols, grad, ld_grad, dtype);
    return tiles_launchable(g, out, cols) ? g.total : 0;
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
    const WgradPlan g = plan_wgrad(n_tokens, out, cols, grad, ld_grad, dtype);
    if (!tiles_launchable(g, out, cols)) return HIMUON_ERR_UNSUPPORTED;
    if (g.total > 0 && (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < g.total)) return HIMUON_ERR_WORKSPACE;
    if (n_tokens == 0 && accumulate) return HIMUON_OK;
    StreamDevice on(stream);
    if (on.status != HIMUON_OK) return on.status;
    const hipStream_t hs = static_cast<hipStream_t>(stream);
    uint8_t* const ws = static_cast<uint8_t*>(workspace);
    WgradArgs p{};
    p.a = static_cast<const uint16_t*>(grad);
    p.lda = ld_grad;
    p.a_cols = (int32_t)out;
    p.tail = (int32_t)(n_tokens % kGroup);
    p.codes = static_cast<const uint8_t*>(codes);
    p.exps = static_cast<const uint8_t*>(exponents);
    p.lde = cols;
    StageArgs s{};
    if (g.stage) {
        s.grad = grad;
        s.a = reinterpret_cast<uint16_t*>(ws);
        s.ld = ld_grad;
        s.tokens = n_tokens;
        s.rows = (int32_t)out;
        s.pitch = (int32_t)g.pitch;
        s.chunks = g.groups * kGroup * (g.pitch / 8);
        s.grad_blocks = (int32_t)std::min<int64_t>(ceil_div(s.chunks, kThreads), 16384);
        p.a = s.a;
        p.lda = g.pitch;
        p.a_cols = (int32_t)g.pitch;
        p.tail = 0;
    }
    if (g.tile != Tile::DIRECT && (cols % 4 || ((uintptr_t)exponents & 3))) {
        s.exps = p.exps;
        s.e = ws + g.exps_at;
        s.cols = (int32_t)cols;
        s.exp_pitch = (int32_t)g.exp_pitch;
        s.exp_bytes = g.groups * g.exp_pitch;
        p.exps = s.e;
        p.lde = g.exp_pitch;
    }
    const unsigned stage_blocks = (unsigned)(s.grad_blocks + std::min<int64_t>(ceil_div(s.exp_bytes, kThreads * 4), 1024));
    if (stage_blocks) {
        if (dtype == HIMUON_BF16) hipLaunchKernelGGL(stage_operands<GemmStore::BF16>, dim3(stage_blocks), dim3(kThreads), 0, hs, s);
        else hipLaunchKernelGGL(stage_operands<GemmStore::F32>, dim3(stage_blocks), dim3(kThreads), 0, hs, s);
        const int st = launch_status();
        if (st != HIMUON_OK) return st;
    }
    p.out = dweight;
    p.part = reinterpret_cast<float*>(ws + g.part_at);
    p.ld_out = ld_dweight;
    p.part_pitch = g.part_pitch;
    p.rows = (int32_t)out;
    p.cols = (int32_t)cols;
    p.slices = (int32_t)(g.tile == Tile::DIRECT ? g.groups : g.groups * g.terms);
    p.terms = g.terms;
    p.splits = g.splits;
    p.accumulate = accumulate != 0;
    return out_dtype == HIMUON_BF16 ? launch_wgrad<GemmStore::BF16>(p, g.tile, dtype, hs) : launch_wgrad<GemmStore::F32>(p, g.tile, dtype, hs);
}
