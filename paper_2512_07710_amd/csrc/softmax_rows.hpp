// Softmax over rows of logits: the sums that log-sum-exp and entropy are made of, and a row's logits and gradients in vectors of 16 bytes.
#pragma once
#include "grad_common.hpp"
#include "lanes.hpp"

namespace moe355 {

constexpr int SOFTMAX_MAX_WAVES = 16;          // of a block
constexpr float LOWEST = -1e30f;               // logits not above it are masked
constexpr float Y_LOWEST = -256.f;             // 2^y is zero from there on; in place of any y below (-inf among them) it makes 2^y y and 2^y (a y + b) zero
constexpr float LOG2E = 1.44269504088896340736f;
constexpr double LN2 = 0.69314718055994530942;

// Sums over logits v in units of log 2, y = (v - m) c with c = log2 e / temperature: s = sum 2^y, u = sum y 2^y, which log-sum-exp and entropy are
// made of.  m is the largest logit as it is, and comes off before the factor: the roundings of c and of the product are then relative to a distance
// from the maximum, where the softmax is decided, however large the logits themselves are (v c - m c would carry half a unit of the last place of
// v c into the exponent).  m = -inf: nothing but masked logits so far (or NaN, which the sums hold)
struct softmax_stats {
    float m, s, u;
};
__device__ inline void rebase(softmax_stats& t, float to, float c) {
    if (t.m == to) return;
    const float d = fmaxf((t.m - to) * c, Y_LOWEST), f = __builtin_amdgcn_exp2f(d);
    t.u = f * fmaf(t.s, d, t.u);
    t.s *= f;
    t.m = to;
}
// What a block's waves tell each other
struct block_scratch {
    float a[SOFTMAX_MAX_WAVES], b[SOFTMAX_MAX_WAVES];
};
__device__ inline float block_largest(float v, block_scratch& lds) {
    const int waves = blockDim.x >> 6, lane = threadIdx.x & 63;
    v = wave_largest(v);
    if (waves == 1) return v;
    if (lane == 0) lds.a[threadIdx.x >> 6] = v;
    __syncthreads();
    v = wave_largest(lane < waves ? lds.a[lane] : -INFINITY);
    __syncthreads();
    return v;
}
// the block's sums over one m, in every thread
__device__ inline softmax_stats block_sums(softmax_stats t, block_scratch& lds) {
    const int waves = blockDim.x >> 6, lane = threadIdx.x & 63;
    t.s = wave_total(t.s);
    t.u = wave_total(t.u);
    if (waves == 1) return t;
    if (lane == 0) {
        lds.a[threadIdx.x >> 6] = t.s;
        lds.b[threadIdx.x >> 6] = t.u;
    }
    __syncthreads();
    t.s = wave_total(lane < waves ? lds.a[lane] : 0.f);
    t.u = wave_total(lane < waves ? lds.b[lane] : 0.f);
    return t;
}
// the same for sums over different m
__device__ inline softmax_stats block_join(softmax_stats t, float c, block_scratch& lds) {
    const float m = block_largest(t.m, lds);
    if (m > -INFINITY) rebase(t, m, c);        // (otherwise there is nothing but masked logits, or NaN, which the sums hold)
    return block_sums(t, lds);
}

// 16 bytes of a row, at any element: rows of odd length start at odd places
typedef u32x2 __attribute__((aligned(2))) u32x2_any;
template <bool BF16>
struct row_type {
    static constexpr int N = BF16 ? 8 : 4;     // elements of a vector
    static __device__ u32x4 none() { return BF16 ? u32x4{0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u} : u32x4{0xFF800000u, 0xFF800000u, 0xFF800000u, 0xFF800000u}; }
    static __device__ u32x4 load(const void* row, int64_t i) { return *reinterpret_cast<const u32x4_any*>(static_cast<const char*>(row) + i * 16); }
    static __device__ float at(const u32x4& v, int j) {
        return BF16 ? (j & 1 ? bf16hi(v[j >> 1]) : bf16lo(v[j >> 1])) : __uint_as_float(v[j]);
    }
};

// vector i of N gradients
template <bool BF16, int N>
__device__ inline void store_grad(void* row, int64_t i, const float (&g)[N]) {
    char* const p = static_cast<char*>(row) + i * N * (BF16 ? 2 : 4);
    if constexpr (BF16 && N == 8) *reinterpret_cast<u32x4_any*>(p) = u32x4{bf16_pair(g[0], g[1]), bf16_pair(g[2], g[3]), bf16_pair(g[4], g[5]), bf16_pair(g[6], g[7])};
    else if constexpr (BF16) *reinterpret_cast<u32x2_any*>(p) = u32x2{bf16_pair(g[0], g[1]), bf16_pair(g[2], g[3])};
    else
#pragma unroll
        for (int h = 0; h < N; h += 4)
            *reinterpret_cast<u32x4_any*>(p + h * 4) = u32x4{__float_as_uint(g[h]), __float_as_uint(g[h + 1]), __float_as_uint(g[h + 2]), __float_as_uint(g[h + 3])};
}

// 2^x and log2 x to fp32's resolution of 2^x and of x itself, whatever their size: whole part and rest apart, and the rest of a logarithm
// from 2^-log2(x) x - 1.  (fp64's own functions take three times as long, and a block waits for them.)
__device__ inline double exp2_of(double x) {
    if (!(x > -1000.0 && x < 1000.0)) return (double)__builtin_amdgcn_exp2f((float)x);         // (0, infinite or NaN)
    const double k = rint(x);
    return ldexp((double)__builtin_amdgcn_exp2f((float)(x - k)), (int)k);
}
__device__ inline double log2_of(float x) {
    const float l = __builtin_amdgcn_logf(x);
    const float whole = rintf(l), part = l - whole;
    const float rest = fmaf(ldexpf(x, -(int)whole), __builtin_amdgcn_exp2f(-part), -1.f);
    return (double)l + (double)rest * (1.0 / LN2);
}
// Sums of a thread that meets its logits in any number of goes
template <bool BF16>
struct running_sums {
    static constexpr int N = row_type<BF16>::N;
    softmax_stats st{-INFINITY, 0.f, 0.f};
    const float c;                             // log2 e / temperature
    __device__ explicit running_sums(float c_) : c(c_) {}
    __device__ void take(float top) {          // before logits up to `top` are added
        if (top > LOWEST && top > st.m) rebase(st, top, c);
    }
    __device__ void one(float v, float m) {
        const float y = (v - m) * c, e = __builtin_amdgcn_exp2f(y);
        st.s += e;
        st.u = fmaf(e, fmaxf(y, Y_LOWEST), st.u);
    }
    __device__ float base() const { return st.m > -INFINITY ? st.m : 0.f; }    // (0: all are masked, 2^y = 0)
    template <int M>
    __device__ static float largest(const u32x4 (&v)[M]) {
        float top = -INFINITY;
#pragma unroll
        for (int n = 0; n < M; ++n)
#pragma unroll
            for (int j = 0; j < N; ++j) top = fmaxf(top, row_type<BF16>::at(v[n], j));
        return top;
    }
    template <int M>
    __device__ void sum(const u32x4 (&v)[M]) {
        const float b = base();
#pragma unroll
        for (int n = 0; n < M; ++n)
#pragma unroll
            for (int j = 0; j < N; ++j) one(row_type<BF16>::at(v[n], j), b);
    }
    template <int M>
    __device__ void add(const u32x4 (&v)[M]) {
        take(largest(v));
        sum(v);
    }
    __device__ void add_one(float v) {
        take(v);
        one(v, base());
    }
};

}  // namespace moe355
