// Host helpers shared by the entry points of the training-step operators
// (embed_ops.hip, qk_norm_rope.hip, act8_ops.hip).
#pragma once

#include "elementwise8.h"
#include "himuon_internal.h"
#include "ns_gemm_path.h"
#include "sizes.h"

namespace himuon {

// Makes the device of a call's stream current for the scope of an entry point.
struct StreamDevice {
    int cur = 0, dev = 0, status;
    explicit StreamDevice(void* stream) { status = stream_device(static_cast<hipStream_t>(stream), &cur, &dev); }
    ~StreamDevice()
    {
        if (status == HIMUON_OK && cur != dev) (void)hipSetDevice(cur);
    }
};

inline bool known_dtype(int d) { return d == HIMUON_F32 || d == HIMUON_BF16; }
inline bool known_index(int i) { return i == HIMUON_I32 || i == HIMUON_I64; }
inline int64_t dtype_size(int d) { return d == HIMUON_BF16 ? 2 : 4; }
inline int launch_status()
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? HIMUON_OK : set_hip_error(e);
}

// Element `i` of an index array of either width.
__device__ __forceinline__ int64_t load_index(const void* p, int64_t i, bool wide)
{
    return wide ? static_cast<const int64_t*>(p)[i] : (int64_t) static_cast<const int32_t*>(p)[i];
}

// Eight consecutive elements as fp32, held as one value (no private array), from
// and to any address that is a multiple of the element's size.
typedef float f32x8 __attribute__((ext_vector_type(8)));

// The same as they lie in memory, the first n of them (loads in flight take half the
// registers, and no instruction waits for them before they are used).
template <GemmStore ST> struct Raw8 {
    Chunk4 w[ST == GemmStore::BF16 ? 1 : 2];
};

template <GemmStore ST> __device__ __forceinline__ Raw8<ST> get_raw8(const void* base, int64_t i, int n)
{
    Raw8<ST> r;
    if constexpr (ST == GemmStore::BF16) {
        const uint16_t* const p = static_cast<const uint16_t*>(base) + i;
        if (n == 8) {
            r.w[0] = *reinterpret_cast<const Chunk4Any16*>(p);
        } else {
            uint32_t h[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) h[e] = e < n ? p[e] : 0u;
            r.w[0] = Chunk4{h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16};
        }
    } else {
        const float* const p = static_cast<const float*>(base) + i;
        if (n == 8) {
            r.w[0] = *reinterpret_cast<const Chunk4Any32*>(p);
            r.w[1] = *reinterpret_cast<const Chunk4Any32*>(p + 4);
        } else {
            uint32_t h[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) h[e] = e < n ? __float_as_uint(p[e]) : 0u;
            r.w[0] = Chunk4{h[0], h[1], h[2], h[3]};
            r.w[1] = Chunk4{h[4], h[5], h[6], h[7]};
        }
    }
    return r;
}

template <GemmStore ST> __device__ __forceinline__ float raw_value(const Raw8<ST>& r, int e)
{
    if constexpr (ST == GemmStore::BF16) return __uint_as_float((e & 1) ? (r.w[0][e >> 1] & 0xffff0000u) : (r.w[0][e >> 1] << 16));
    else return __uint_as_float(r.w[e >> 2][e & 3]);
}

template <GemmStore ST> __device__ __forceinline__ f32x8 get8(const void* base, int64_t i)
{
    float v[8];
    load8<ST>(base, i, 8, false, v);
    return f32x8{v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]};
}

template <GemmStore ST> __device__ __forceinline__ void put8(void* base, int64_t i, f32x8 x)
{
    float v[8] = {x[0], x[1], x[2], x[3], x[4], x[5], x[6], x[7]};
    store8<ST>(base, i, 8, false, v);
}

template <GemmStore ST> __device__ __forceinline__ float get1(const void* base, int64_t i)
{
    if constexpr (ST == GemmStore::BF16) return __uint_as_float((uint32_t) static_cast<const uint16_t*>(base)[i] << 16);
    else return static_cast<const float*>(base)[i];
}

template <GemmStore ST> __device__ __forceinline__ void put1(void* base, int64_t i, float v)
{
    if constexpr (ST == GemmStore::BF16) static_cast<uint16_t*>(base)[i] = __builtin_bit_cast(uint16_t, (__bf16)v);
    else static_cast<float*>(base)[i] = v;
}

// Between a wave's writes to LDS and reads of what its other lanes wrote: they are carried out
// in order, so only the compiler has to keep it.
__device__ __forceinline__ void wave_exchange()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
    asm volatile("" ::: "memory");
}

}  // namespace himuon
