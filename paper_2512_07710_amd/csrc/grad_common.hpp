// What the kernels of the training side share: rows of bf16 or fp32 in vectors of eight, sums over a block.
#pragma once
#include "e4m3.hpp"
#include "moe_internal.hpp"

namespace moe355 {

typedef float f32x4 __attribute__((ext_vector_type(4)));

__device__ inline uint32_t bf16_bits(float v) {                // round to nearest even, NaN stays NaN
    const uint32_t b = __float_as_uint(v);
    if ((b & 0x7FFFFFFFu) > 0x7F800000u) return (b >> 16) | 0x40;
    return (b + 0x7FFFu + ((b >> 16) & 1u)) >> 16;
}

__device__ inline uint32_t bf16_pair(float a, float b) {       // round to nearest even
    typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, v2bf{(__bf16)a, (__bf16)b});
}

// Eight consecutive elements of a row as fp32.  BF16: 16 bytes, else 32; `p` is aligned to 16.
struct vec8 {
    float v[8];
};
template <bool BF16, bool PAST = false>
__device__ inline vec8 load8(const void* row, int64_t i) {
    vec8 r;
    if (BF16) {
        const u32x4* const p = reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(row) + i);
        const u32x4 u = PAST ? __builtin_nontemporal_load(p) : *p;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            r.v[2 * j] = bf16lo(u[j]);
            r.v[2 * j + 1] = bf16hi(u[j]);
        }
    } else {
        const f32x4* const p = reinterpret_cast<const f32x4*>(static_cast<const float*>(row) + i);
        const f32x4 a = PAST ? __builtin_nontemporal_load(p) : p[0], b = PAST ? __builtin_nontemporal_load(p + 1) : p[1];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            r.v[j] = a[j];
            r.v[4 + j] = b[j];
        }
    }
    return r;
}
template <bool BF16, bool PAST = false>
__device__ inline void store8(void* row, int64_t i, const vec8& r) {
    if (BF16) {
        u32x4 u;
#pragma unroll
        for (int j = 0; j < 4; ++j) u[j] = bf16_bits(r.v[2 * j]) | (bf16_bits(r.v[2 * j + 1]) << 16);
        u32x4* const p = reinterpret_cast<u32x4*>(static_cast<uint16_t*>(row) + i);
        if (PAST) __builtin_nontemporal_store(u, p);
        else *p = u;
    } else {
        f32x4* const p = reinterpret_cast<f32x4*>(static_cast<float*>(row) + i);
        const f32x4 a = {r.v[0], r.v[1], r.v[2], r.v[3]}, b = {r.v[4], r.v[5], r.v[6], r.v[7]};
        if (PAST) {
            __builtin_nontemporal_store(a, p);
            __builtin_nontemporal_store(b, p + 1);
        } else {
            p[0] = a;
            p[1] = b;
        }
    }
}
// The same at any element (rows of odd length start at odd places) and past the caches, for rows that are requested ahead: as they lie in memory
typedef u32x4 __attribute__((aligned(2))) u32x4_any;
typedef f32x4 __attribute__((aligned(4))) f32x4_any;
// ODD: bf16 rows may begin inside a 32-bit word and are then read from that word on, with the word behind the vector, which the row reaches into: loads of 16
// bytes that are not aligned to four take longer (16744 x 4203 bf16, norm with residual 198 -> 170 us; its gradient 230 -> 240, which stays with the others)
template <bool BF16, bool ODD = false>
struct raw8 {
    u32x4 a[BF16 ? 1 : 2];
    uint32_t behind = 0, shift = 0;
    __device__ void load(const void* row, int64_t i) {
        const char* at = static_cast<const char*>(row) + i * (BF16 ? 2 : 4);
        if (BF16 && ODD) {
            shift = (uint32_t)(uintptr_t)at << 3 & 16;
            at -= shift >> 3;
            if (shift) behind = *reinterpret_cast<const uint32_t*>(at + 16);
        }
        const u32x4_any* const p = reinterpret_cast<const u32x4_any*>(at);
#pragma unroll
        for (int j = 0; j < (BF16 ? 1 : 2); ++j) a[j] = __builtin_nontemporal_load(p + j);
    }
    __device__ float at(int j) const {
        if (!BF16) return __uint_as_float(a[BF16 ? 0 : j >> 2][BF16 ? 0 : j & 3]);
        uint32_t w = a[0][j >> 1];
        if (ODD) w = __builtin_amdgcn_alignbit(j >> 1 == 3 ? behind : a[0][(j >> 1) + (j >> 1 < 3)], w, shift);
        return j & 1 ? bf16hi(w) : bf16lo(w);
    }
};
template <bool BF16>
__device__ inline void store8_any(void* row, int64_t i, const vec8& r) {
    if (BF16) {
        u32x4 u;
#pragma unroll
        for (int j = 0; j < 4; ++j) u[j] = bf16_bits(r.v[2 * j]) | (bf16_bits(r.v[2 * j + 1]) << 16);
        __builtin_nontemporal_store(u, reinterpret_cast<u32x4_any*>(static_cast<uint16_t*>(row) + i));
    } else {
        f32x4_any* const p = reinterpret_cast<f32x4_any*>(static_cast<float*>(row) + i);
        __builtin_nontemporal_store(f32x4{r.v[0], r.v[1], r.v[2], r.v[3]}, p);
        __builtin_nontemporal_store(f32x4{r.v[4], r.v[5], r.v[6], r.v[7]}, p + 1);
    }
}
__device__ inline vec8 load8_any(const float* row, int64_t i) {                // (kept in the caches)
    const f32x4_any* const p = reinterpret_cast<const f32x4_any*>(row + i);
    const f32x4 a = p[0], b = p[1];
    return vec8{{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]}};
}
template <bool BF16>
__device__ inline float load1(const void* row, int64_t i) {
    return BF16 ? __uint_as_float((uint32_t) static_cast<const uint16_t*>(row)[i] << 16) : static_cast<const float*>(row)[i];
}
template <bool BF16>
__device__ inline void store1(void* row, int64_t i, float v) {
    if (BF16) static_cast<uint16_t*>(row)[i] = (uint16_t)bf16_bits(v);
    else static_cast<float*>(row)[i] = v;
}
// v as an array of this type holds it
template <bool BF16>
__device__ inline float rounded(float v) {
    return BF16 ? __uint_as_float(bf16_bits(v) << 16) : v;
}
template <bool BF16>
__host__ __device__ inline const void* row_of(const void* p, int64_t elements) {
    return static_cast<const char*>(p) + elements * (BF16 ? 2 : 4);
}
template <bool BF16>
__host__ __device__ inline void* row_of(void* p, int64_t elements) {
    return static_cast<char*>(p) + elements * (BF16 ? 2 : 4);
}

__device__ inline float wave_sum(float v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}
// sum over a block's first `waves` waves, in every thread; `lds`: a float for each.  Called by the whole block.
__device__ inline float block_sum(float v, float* lds, int waves) {
    v = wave_sum(v);
    if (waves == 1) return v;
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.f;
    for (int w = 0; w < waves; ++w) v += lds[w];
    __syncthreads();
    return v;
}

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

}  // namespace moe355
