// What the attention kernels share (attention.hip, attention_grad.hip): operand fragments,
// tiles in LDS, and where a block's rows lie.
//
// Products run on 32 x 32 MFMA tiles. A product's result holds in lane l of a wave column
// l % 32 and, in register i, row 8 (i / 4) + 4 (l / 32) + i % 4. Products are laid out so that
// this is the next product's second operand as it stands: of 16 values of the contracted
// index, half 0 of the wave holds 0-3 and 8-11 and half 1 the others, and the first operand's
// reads follow that order. So scores never pass through LDS.
#pragma once

#include "attn_plan.h"
#include "lds_dma.h"
#include "train_ops.h"

namespace himuon {
namespace attn {

using dev::bf16x8;
using dev::f32x16;
using dev::f32x4;
using dev::u32x2;
using dev::u32x4;

constexpr float kLog2e = 1.44269504088896341f;

// ------------------------------------------------------------------ arguments

struct Heads {
    uint8_t* ptr;
    int64_t sb, ss, sh;  // strides in bytes: batch, token, head
};

struct AttnArgs {
    Heads q, k, v, o, g, dq, dk, dv;
    float* lse;         // [batch, q_len, q_heads]
    float2* stats;       // backward: {lse log2 e, rowsum(g o)} of every row of a group of heads
    float* part;        // few rows: partial results
    const void *qs, *ks, *ql, *kl;  // starts and lengths
    int64_t q_len, k_len;
    int32_t batch, hk, group, dim, causal, wide, packed, slots, splits;
    int32_t k_blocks, k_slots;  // backward, few tiles: the blocks of keys ahead of those of queries, and their slots
    float scale;
};

// ---------------------------------------------------------- fragments, products

// Eight values of the contracted index, for one row (column) of an operand.
template <GemmStore ST> struct Frag {
    u32x4 w[ST == GemmStore::BF16 ? 1 : 2];
};

template <GemmStore ST> HM_DEV void mma(f32x16& acc, const Frag<ST>& a, const Frag<ST>& b)
{
    if constexpr (ST == GemmStore::BF16) {
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a.w[0]), __builtin_bit_cast(bf16x8, b.w[0]), acc, 0,
                                                      0, 0);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.w[j >> 2][j & 3]), __uint_as_float(b.w[j >> 2][j & 3]), acc, 0,
                                                       0, 0);
    }
}

// Registers 8 t .. 8 t + 7 of a result as the second operand of the next product. (bf16:
// rounded to nearest even, by at most 2^-8 of each value; sums are taken of the unrounded ones.)
template <GemmStore ST> HM_DEV Frag<ST> as_operand(const f32x16& c, int t)
{
    Frag<ST> f;
    if constexpr (ST == GemmStore::BF16) {
#pragma unroll
        for (int j = 0; j < 4; ++j) f.w[0][j] = dev::pack2<Operand::BF16>(c[8 * t + 2 * j], c[8 * t + 2 * j + 1]);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) f.w[j >> 2][j & 3] = __float_as_uint(c[8 * t + j]);
    }
    return f;
}

// Values 2 i and 2 i + 1 of a result's registers in that operand.
template <GemmStore ST> HM_DEV void set_pair(Frag<ST> (&f)[2], int i, float a, float b)
{
    if constexpr (ST == GemmStore::BF16) {
        f[i >> 2].w[0][i & 3] = dev::pack2<Operand::BF16>(a, b);
    } else {
        f[i >> 2].w[(i & 3) >> 1][2 * (i & 1)] = __float_as_uint(a);
        f[i >> 2].w[(i & 3) >> 1][2 * (i & 1) + 1] = __float_as_uint(b);
    }
}

// Keeps that pair's computation where it stands (the compiler would move it down to its use
// behind the next branch, past the products that it is to run beside).
template <GemmStore ST> HM_DEV void settle_pair(Frag<ST> (&f)[2], int i)
{
    if constexpr (ST == GemmStore::BF16) {
        uint32_t w = f[i >> 2].w[0][i & 3];
        asm volatile("" : "+v"(w));
        f[i >> 2].w[0][i & 3] = w;
    } else {
        uint32_t a = f[i >> 2].w[(i & 3) >> 1][2 * (i & 1)], b = f[i >> 2].w[(i & 3) >> 1][2 * (i & 1) + 1];
        asm volatile("" : "+v"(a), "+v"(b));
        f[i >> 2].w[(i & 3) >> 1][2 * (i & 1)] = a;
        f[i >> 2].w[(i & 3) >> 1][2 * (i & 1) + 1] = b;
    }
}

template <GemmStore ST> HM_DEV float frag_value(const Frag<ST>& f, int e)
{
    if constexpr (ST == GemmStore::BF16) return __uint_as_float((e & 1) ? (f.w[0][e >> 1] & 0xffff0000u) : (f.w[0][e >> 1] << 16));
    else return __uint_as_float(f.w[e >> 2][e & 3]);
}

// Row of a result's register i in half h of the wave. (Compared with a bound, it is the bound
// less 4 h that is compared with a constant.)
HM_DEV constexpr int result_row(int i, int h) { return 8 * (i >> 2) + 4 * h + (i & 3); }

// The other half's value, combined.
HM_DEV float max_halves(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
HM_DEV float add_halves(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// ------------------------------------------------------------------ tiles in LDS

// Rows of DP elements, their 16-byte chunks permuted by the row so that neither 16 rows'
// reads of one chunk nor four rows' reads of four chunks (transposing) share a bank.
template <GemmStore ST, int DP> struct Lay {
    static constexpr int ES = ST == GemmStore::BF16 ? 2 : 4, PITCH = DP * ES, CH = PITCH / 16, NS = DP / 16, DT = DP / 32;

    HM_DEV static int swz(int row)
    {
        if constexpr (CH == 8) return ((row >> 1) & 1) << 2 | ((row >> 2) & 3);
        else if constexpr (ST == GemmStore::BF16) return (row & 3) << 2 | ((row >> 2) & 3);
        else return ((row >> 2) & 1) << 3 | (row & 3) << 1 | ((row >> 3) & 1);
    }

    // Elements 16 s + 8 h .. of row `row`.
    HM_DEV static Frag<ST> row_frag(const uint8_t* tile, int row, int s, int h)
    {
        const uint8_t* const p = tile + row * PITCH;
        const int f = swz(row);
        Frag<ST> r;
        if constexpr (ST == GemmStore::BF16) {
            r.w[0] = *reinterpret_cast<const u32x4*>(p + 16 * ((2 * s + h) ^ f));
        } else {
            r.w[0] = *reinterpret_cast<const u32x4*>(p + 16 * ((4 * s + 2 * h) ^ f));
            r.w[1] = *reinterpret_cast<const u32x4*>(p + 16 * ((4 * s + 2 * h + 1) ^ f));
        }
        return r;
    }

    // Column d0 + lane % 32 of rows k16 .. k16 + 15, in the order of a result's registers.
    HM_DEV static Frag<ST> col_frag(const uint8_t* tile, int k16, int d0, int lane)
    {
        const int h = lane >> 5;
        Frag<ST> r;
        if constexpr (ST == GemmStore::BF16) {
            u32x2 v[2];
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const int row = 8 * x + 4 * h + ((lane & 15) >> 2);
                const int chunk = (d0 / 8) ^ ((2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ swz(row));
                v[x] = dev::tr_read(tile + k16 * PITCH + row * PITCH + 16 * chunk + 8 * (lane & 1));
            }
            r.w[0] = u32x4{v[0][0], v[0][1], v[1][0], v[1][1]};
        } else {
            const int col = d0 + (lane & 31);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int row = result_row(j, h);
                r.w[j >> 2][j & 3] = *reinterpret_cast<const uint32_t*>(tile + (k16 + row) * PITCH + 16 * ((col >> 2) ^ swz(row)) + 4 * (col & 3));
            }
        }
        return r;
    }
};

// use(i, read(i)) for i = 0 .. N - 1 with the reads DEPTH steps ahead of their uses, and no
// further: reads that the compiler moves up all at once cost the registers of a second wave.
// fill() sends the first ones out before work that does not need them. A step stays together, so
// that a product's other half of work (a share of the vector ALU's) goes out beside it: left
// alone, the compiler puts the products first and the exponentials behind them.
template <class T, int N, int DEPTH> struct Ahead {
    T f[DEPTH];
    template <class Read> HM_DEV void fill(Read read)
    {
#pragma unroll
        for (int i = 0; i < DEPTH; ++i)
            if (i < N) f[i] = read(i);
        __builtin_amdgcn_sched_barrier(0);
    }
    template <class Read, class Use> HM_DEV void run(Read read, Use use)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            use(i, f[i % DEPTH]);
            if (i + DEPTH < N) f[i % DEPTH] = read(i + DEPTH);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
};

HM_DEV void settle(float& a) { asm volatile("" : "+v"(a)); }
HM_DEV void settle(f32x16& x, int i)
{
    float a = x[i];
    settle(a);
    x[i] = a;
}

// Fragments in flight: an LDS read takes as long as three or four 16-bit products, and less
// than one step's eight of fp32.
template <GemmStore ST, int DP> constexpr int kDepth = ST == GemmStore::BF16 ? 4 : DP <= 128 ? 2 : 1;

// 16 bytes of a row whose first `bytes` (> 0) count, from any address that is a multiple of
// the element's size.
template <GemmStore ST> HM_DEV u32x4 load_chunk(const uint8_t* p, int bytes)
{
    if (bytes >= 16) {
        if constexpr (ST == GemmStore::BF16) return *reinterpret_cast<const Chunk4Any16*>(p);
        else return *reinterpret_cast<const Chunk4Any32*>(p);
    }
    u32x4 r = {};
    if constexpr (ST == GemmStore::BF16) {
        const uint16_t* const e = reinterpret_cast<const uint16_t*>(p);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (2 * j < bytes) r[j >> 1] |= (uint32_t)e[j] << (16 * (j & 1));
    } else {
        const uint32_t* const e = reinterpret_cast<const uint32_t*>(p);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (4 * j < bytes) r[j] = e[j];
    }
    return r;
}

// An operand's fragments of one row in memory (zeros where it is not `on`), elements
// 16 s + 8 h .. of it. VEC: whole 16-byte chunks, aligned.
template <bool VEC, GemmStore ST, int DP> HM_DEV void load_row(Frag<ST> (&f)[DP / 16], const uint8_t* row, bool on, int dim, int h)
{
    constexpr int ES = ST == GemmStore::BF16 ? 2 : 4, C = 16 / ES;
#pragma unroll
    for (int s = 0; s < DP / 16; ++s) {
#pragma unroll
        for (int x = 0; x < 8 / C; ++x) {
            const int d = 16 * s + 8 * h + C * x;
            if constexpr (VEC) f[s].w[x] = on && d < dim ? *reinterpret_cast<const u32x4*>(row + d * ES) : u32x4{};
            else f[s].w[x] = on && d < dim ? load_chunk<ST>(row + d * ES, (dim - d) * ES) : u32x4{};
        }
    }
}

// A thread's share of a tile of ROWS rows that NT threads copy: which rows and which 16 bytes
// of them. (`tid`: its number among the NT, waves in one piece.)
template <GemmStore ST, int DP, int ROWS, int NT> struct Share {
    using L = Lay<ST, DP>;
    static constexpr int NI = ROWS * L::CH / NT;
    static constexpr int N = NI > 4 ? 4 : NI;  // copies that share m0
    static_assert(NI >= 1 && NI * NT == ROWS * L::CH, "");
    int tid;
    HM_DEV int slot(int i) const { return (tid & ~63) * NI + 64 * i + (tid & 63); }
    HM_DEV int row(int i) const { return slot(i) / L::CH; }
    HM_DEV int byte(int i) const { return 16 * ((slot(i) % L::CH) ^ L::swz(row(i))); }

    // Offsets of this thread's share of a tile of rows `stride` bytes apart, as copy() takes them.
    HM_DEV uint32_t offset(int i, int64_t stride) const { return (uint32_t)(row(i) * stride) + rest(i); }
    HM_DEV uint32_t rest(int i) const { return (uint32_t)(byte(i) + 4096 - 1024 * (i % N)); }

    // A whole tile of whole rows (DP elements), by DMA.
    HM_DEV void copy(uint8_t* tile, const uint8_t* base, const uint32_t (&off)[NI]) const
    {
        const uint64_t from = dev::uniform_address(base - 4096);
        const uint32_t to = lds_place(tile);
#pragma unroll
        for (int i = 0; i < NI; i += N) {
            uint32_t v[N];
#pragma unroll
            for (int j = 0; j < N; ++j) v[j] = off[i + j];
            dev::dma16_run<N>(to + 1024 * i, v, from);
        }
    }
    HM_DEV uint32_t lds_place(uint8_t* tile) const
    {
        return (uint32_t)__builtin_amdgcn_readfirstlane((int)(dev::lds_offset(tile) + 16 * NI * (tid & ~63)));
    }

    // Copies the rows to LDS: row i at base + off(i) (bytes), zeros where on(i) does not hold
    // and behind the row's `row_bytes`. DMA: whole 16-byte chunks, aligned; off below 2^32 - 2^28; where
    // the tile is `whole`, the places behind row_bytes stay as they are.
    template <bool DMA, class Off, class On>
    HM_DEV void stage(uint8_t* tile, const uint8_t* base, int row_bytes, bool whole, Off off, On on) const
    {
        if constexpr (DMA) {
            const uint64_t from = dev::uniform_address(base);
            const uint32_t to = lds_place(tile);
#pragma unroll(NI > 8 ? 4 : NI)
            for (int i = 0; i < NI; ++i) {
                const int b = byte(i);
                if ((whole || on(i)) && b < row_bytes) dev::dma16(to + 1024 * i, (uint32_t)off(i) + (uint32_t)b, from);
                else if (!whole) *reinterpret_cast<u32x4*>(tile + 16 * slot(i)) = u32x4{};
            }
        } else {
            constexpr int U = NI > 4 ? 4 : NI;
#pragma unroll 1
            for (int j = 0; j < NI; j += U) {
                u32x4 v[U];
#pragma unroll
                for (int i = 0; i < U; ++i) {
                    const int b = byte(i + j);
                    v[i] = on(i + j) && b < row_bytes ? load_chunk<ST>(base + off(i + j) + b, row_bytes - b) : u32x4{};
                }
#pragma unroll
                for (int i = 0; i < U; ++i) *reinterpret_cast<u32x4*>(tile + 16 * slot(i + j)) = v[i];
            }
        }
    }
};

// Waits until at most N of this wave's DMA are in flight (below 0: for none of them) and its
// LDS accesses are done.
template <int N> HM_DEV void wave_wait()
{
    constexpr int V = N < 0 || N > 63 ? 63 : N;
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((V & 15) | (V >> 4) << 14 | 7 << 4);
    __builtin_amdgcn_wave_barrier();
    asm volatile("" ::: "memory");
}

// Zeros in `bytes` of LDS (a multiple of 16).
template <int NT> HM_DEV void clear_lds(uint8_t* p, int bytes)
{
    for (int i = 16 * (int)threadIdx.x; i < bytes; i += 16 * NT) *reinterpret_cast<u32x4*>(p + i) = u32x4{};
}

// A lane's column of a transposed result, mul times it, as one row of `dim` elements in memory
// (zeros if the row is not `on`).
template <bool VEC, GemmStore ST, int DT> HM_DEV void store_row(uint8_t* row, const f32x16 (&acc)[DT], bool on, float mul, int dim, int h)
{
    constexpr int ES = ST == GemmStore::BF16 ? 2 : 4;
#pragma unroll
    for (int t = 0; t < DT; ++t) {
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const int d = 32 * t + result_row(i, h);
            const float a = on ? acc[t][i] * mul : 0.f, b = on ? acc[t][i + 1] * mul : 0.f, c = on ? acc[t][i + 2] * mul : 0.f,
                        e = on ? acc[t][i + 3] * mul : 0.f;
            if constexpr (VEC) {  // (dim is a multiple of four)
                if (d < dim) {
                    if constexpr (ST == GemmStore::BF16)
                        *reinterpret_cast<u32x2*>(row + d * ES) = u32x2{dev::pack2<Operand::BF16>(a, b), dev::pack2<Operand::BF16>(c, e)};
                    else
                        *reinterpret_cast<f32x4*>(row + d * ES) = f32x4{a, b, c, e};
                }
            } else {
                if (d < dim) put1<ST>(row, d, a);
                if (d + 1 < dim) put1<ST>(row, d + 1, b);
                if (d + 2 < dim) put1<ST>(row, d + 2, c);
                if (d + 3 < dim) put1<ST>(row, d + 3, e);
            }
        }
    }
}

// --------------------------------------------------------- where a block's rows lie

// Which key head and which work item (of find_seq) block `id` of `n` has; PARTS blocks share an item.
// (A launch has fewer than 2^24 blocks.)
//
// Blocks are dealt out to the eight XCDs in turn, so that id % 8 is the XCD: blocks that read the
// same keys run on one, whose L2 holds them. The longest tiles come first (LAST_FIRST: a sequence's
// last ones) over kMixed heads of sequences at a time: the keys of so many still fit the L2,
// and a launch ends with its shortest tiles. (16 + 8 heads of 128, one head of a sequence after the other / mixed,
// us: 16 x 1024 tokens bf16 forward 118 / 106, backward 392 / 343; 8 x 1024 fp32 461 / 350 and 1717 / 1100.)
constexpr uint32_t kMixed = 8;
struct Item {
    int kh, part;
    uint32_t item;
};
template <int PARTS, bool LAST_FIRST> HM_DEV Item find_item(const AttnArgs& p, uint32_t id, uint32_t n)
{
    Item a{};
    n /= PARTS;
    if (PARTS > 1 && n % 8 == 0) {
        a.part = (int)((id >> 3) % PARTS);
        id = (id & 7) | (id >> 3) / PARTS << 3;
    } else if (PARTS > 1) {
        a.part = (int)(id % PARTS);
        id /= PARTS;
    }
    const uint32_t tiles = (uint32_t)p.slots;
    if (p.packed) {
        const uint32_t x = id & 7, rest = n & 7, w = x * (n >> 3) + min(x, rest) + (id >> 3);
        a.kh = (int)(w / tiles);
        const uint32_t t = w - (uint32_t)a.kh * tiles;
        a.item = LAST_FIRST ? tiles - 1 - t : t;
        return a;
    }
    const uint32_t heads = (uint32_t)p.batch * (uint32_t)p.hk, each = heads % 8 == 0 ? heads / 8 : heads;  // of an XCD
    const uint32_t first = heads % 8 == 0 ? (id & 7) * each : 0, i = heads % 8 == 0 ? id >> 3 : id;
    const uint32_t set = i / (kMixed * tiles), c = min(kMixed, each - set * kMixed), r = i - set * kMixed * tiles, t = r / c;
    const uint32_t head = first + set * kMixed + (r - t * c);
    a.kh = (int)(head / (uint32_t)p.batch);
    a.item = (head - (uint32_t)a.kh * (uint32_t)p.batch) * tiles + (LAST_FIRST ? tiles - 1 - t : t);
    return a;
}

struct Seq {
    int64_t q0, k0;   // first token
    int32_t q_cap, k_cap, nq, nk;  // tokens, and those in use
    int32_t batch, tile;           // row of the batch (packed: 0), tile of the sequence
};

HM_DEV int64_t clamped(const void* p, int64_t i, bool wide, int64_t hi)
{
    const int64_t v = load_index(p, i, wide);
    return v < 0 ? 0 : v > hi ? hi : v;
}

// Work item `w` of a sequence's queries (KEYS: keys): the sequence and the tile of it, ROWS rows
// to a tile and `group` rows to a token. (All lanes of a wave call it.)
//
// Packed: tile t of sequence s has place floor(first row / ROWS) + s + t, counted with the tokens
// ahead of the first sequence as sequence 0 and those behind the last one as the last, so that
// the places need no sums over sequences and a grid of rows / ROWS + batch + 2 holds them
// all; a place behind a sequence's last tile has nothing to do. The sequence is the last whose first place
// is not behind w: 64 of them, evenly spread, are looked at together until it is one of 64 neighbours.
// (Starts that decrease leave results unspecified, and no access outside of the arrays.)
template <bool KEYS, int ROWS> HM_DEV Seq find_seq(const AttnArgs& p, uint32_t w, int group)
{
    Seq s{};
    const bool wide = p.wide;
    if (!p.packed) {
        s.batch = (int32_t)(w / (uint32_t)p.slots);
        s.tile = (int32_t)(w - (uint32_t)s.batch * (uint32_t)p.slots);
        s.q_cap = (int32_t)p.q_len;
        s.k_cap = (int32_t)p.k_len;
        s.nq = p.ql ? (int32_t)clamped(p.ql, s.batch, wide, p.q_len) : s.q_cap;
        s.nk = p.kl ? (int32_t)clamped(p.kl, s.batch, wide, p.k_len) : s.k_cap;
        return s;
    }
    const void* const starts = KEYS ? p.ks : p.qs;
    const int64_t len = KEYS ? p.k_len : p.q_len;
    auto place = [&](int i) { return i == 0 ? (int64_t)0 : clamped(starts, i - 1, wide, len) * group / ROWS + i; };
    int lo = 0;
    for (int n = p.batch + 2; n > 1;) {  // it is among lo .. lo + n - 1
        const int step = (n + 63) >> 6, i = (int)(threadIdx.x & 63) * step;
        const bool at_or_before = i < n && place(lo + min(i, n - 1)) <= (int64_t)w;
        const int k = max(0, __popcll(__ballot(at_or_before)) - 1) * step;
        lo += k;
        n = min(step, n - k);
    }
    const int64_t first = lo == 0 ? 0 : clamped(starts, lo - 1, wide, len);
    const int64_t tile = (int64_t)w - (first * group / ROWS + lo);
    if (tile < 0) return s;
    s.tile = (int32_t)tile;
    const bool real = lo > 0 && lo <= p.batch;
    if (!real) {  // tokens that belong to no sequence
        const int64_t end = lo == 0 ? clamped(starts, 0, wide, len) : len;
        (KEYS ? s.k0 : s.q0) = first;
        (KEYS ? s.k_cap : s.q_cap) = (int32_t)(end - first);
        return s;
    }
    s.q0 = clamped(p.qs, lo - 1, wide, p.q_len);
    s.k0 = clamped(p.ks, lo - 1, wide, p.k_len);
    const int64_t q1 = clamped(p.qs, lo, wide, p.q_len), k1 = clamped(p.ks, lo, wide, p.k_len);
    s.q_cap = (int32_t)(q1 > s.q0 ? q1 - s.q0 : 0);
    s.k_cap = (int32_t)(k1 > s.k0 ? k1 - s.k0 : 0);
    s.nq = p.ql ? (int32_t)clamped(p.ql, lo - 1, wide, s.q_cap) : s.q_cap;
    s.nk = p.kl ? (int32_t)clamped(p.kl, lo - 1, wide, s.k_cap) : s.k_cap;
    return s;
}

// Keys that query q of a sequence sees: the first of them, up to its own where causal, the
// last query lying on the last key.
HM_DEV int visible(const AttnArgs& p, const Seq& s, int q)
{
    if (!p.causal) return s.nk;
    const int64_t n = (int64_t)q + 1 + s.nk - s.nq;
    return n < 0 ? 0 : n > s.nk ? s.nk : (int)n;
}

// The first element of a token's head.
HM_DEV uint8_t* at(const Heads& t, int64_t batch, int64_t token, int64_t head) { return t.ptr + batch * t.sb + token * t.ss + head * t.sh; }

// ------------------------------------------------------------------- host side

int check_attn(const himuon_attn_t* a);
// (packed tokens may be there without a sequence: they get their zeros)
inline bool empty_batch(const himuon_attn_t* a) { return a->batch == 0 && !a->q_starts; }
AttnArgs attn_args(const himuon_attn_t* a);
bool set_heads(Heads& t, const himuon_heads_t* h, const himuon_attn_t* a, int64_t tokens, int heads, bool output, bool* dma);

// A grid of one block to each tile of `tile` rows (KEYS: keys) and key head (false: more than a launch holds).
template <bool KEYS> bool set_grid(AttnArgs& p, int tile, int threads, int64_t* blocks)
{
    const AttnTiles t = attn_tiles<KEYS>(p.packed, p.batch, KEYS ? p.k_len : p.q_len, p.group, p.hk, tile);
    if (t.slots > INT32_MAX || t.blocks < 0 || !launchable(t.blocks, threads)) return false;
    p.slots = (int32_t)t.slots;
    *blocks = t.blocks;
    return true;
}

}  // namespace attn
}  // namespace himuon
