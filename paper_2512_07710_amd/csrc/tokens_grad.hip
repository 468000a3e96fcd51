// Token rows in expert order, and the gradients of that order and of the weighted combine.
#include "grad_common.hpp"

namespace moe355 {
namespace {

constexpr int TOKEN_THREADS = 256;

// 16 bytes of a row
template <bool BF16>
struct piece {
    static constexpr int N = BF16 ? 8 : 4;
    static __device__ const u32x4* at(const void* rows, int64_t row, int d, int i) { return static_cast<const u32x4*>(rows) + row * (d / N) + i; }
    static __device__ u32x4* at(void* rows, int64_t row, int d, int i) { return static_cast<u32x4*>(rows) + row * (d / N) + i; }
    static __device__ float value(const u32x4& v, int j) { return BF16 ? (j & 1 ? bf16hi(v[j >> 1]) : bf16lo(v[j >> 1])) : __uint_as_float(v[j]); }
};

// One block per token and part of its columns; a thread owns 16 bytes of the row.  d is a multiple of 128.
template <bool BF16>
__global__ __launch_bounds__(TOKEN_THREADS) void dispatch_kernel(const void* __restrict__ x, const int32_t* __restrict__ inv_perm, int d, int k,
                                                                 int N, int parts, void* __restrict__ x_perm) {
    typedef piece<BF16> P;
    const int t = blockIdx.x / parts, i = (blockIdx.x % parts) * blockDim.x + threadIdx.x;
    if (i >= d / P::N) return;
    const u32x4 v = *P::at(x, t, d, i);
    for (int j = 0; j < k; ++j) {
        const int row = inv_perm[(int64_t)t * k + j];
        if ((uint32_t)row < (uint32_t)N) *P::at(x_perm, row, d, i) = v;
    }
}

// (the rows of four slots are on their way at a time)
template <bool BF16>
__global__ __launch_bounds__(TOKEN_THREADS) void dispatch_back_kernel(const void* __restrict__ dx_perm, const int32_t* __restrict__ inv_perm,
                                                                      const void* dx_add, int d, int k, int N, int parts, void* dx) {
    typedef piece<BF16> P;
    constexpr int AT_ONCE = 4;
    const int t = blockIdx.x / parts, i = (blockIdx.x % parts) * blockDim.x + threadIdx.x;
    if (i >= d / P::N) return;
    const int32_t* const rows = inv_perm + (int64_t)t * k;
    float sum[P::N] = {};
    for (int j0 = 0; j0 < k; j0 += AT_ONCE) {
        u32x4 v[AT_ONCE];
        bool there[AT_ONCE];
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
            const int row = j0 + u < k ? rows[j0 + u] : -1;
            there[u] = (uint32_t)row < (uint32_t)N;
            if (there[u]) v[u] = __builtin_nontemporal_load(P::at(dx_perm, row, d, i));
        }
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u)
            if (there[u])
#pragma unroll
                for (int c = 0; c < P::N; ++c) sum[c] += P::value(v[u], c);
    }
    if (dx_add) {
        const u32x4 v = *P::at(dx_add, t, d, i);
#pragma unroll
        for (int c = 0; c < P::N; ++c) sum[c] += P::value(v, c);
    }
    u32x4 out;
#pragma unroll
    for (int c = 0; c < 4; ++c) out[c] = BF16 ? bf16_pair(sum[(2 * c) % P::N], sum[(2 * c + 1) % P::N]) : __float_as_uint(sum[c]);
    *P::at(dx, t, d, i) = out;
}

// One block per token.
template <bool BF16>
__global__ __launch_bounds__(TOKEN_THREADS) void combine_back_kernel(const void* __restrict__ dy, const float* __restrict__ y_perm,
                                                                     const int32_t* __restrict__ inv_perm, const float* __restrict__ topk_w,
                                                                     const int32_t* __restrict__ topk_idx, int d, int k, int E, int N,
                                                                     void* __restrict__ dy_perm, float* __restrict__ dw,
                                                                     float* __restrict__ dlogits) {
    __shared__ float lds[MAX_K][TOKEN_THREADS / 64], s_dw[MAX_K];
    const int t = blockIdx.x, waves = blockDim.x >> 6;
    for (int j = 0; j < k; ++j) {
        const int row = inv_perm[(int64_t)t * k + j];
        const float w = topk_w[(int64_t)t * k + j];
        float dot = 0.f;
        if ((uint32_t)row < (uint32_t)N)
            for (int c = threadIdx.x * 8; c < d; c += blockDim.x * 8) {
                const vec8 g = load8<BF16>(dy, (int64_t)t * d + c), y = load8<false, true>(y_perm, (int64_t)row * d + c);
                vec8 o;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    dot = fmaf(g.v[i], y.v[i], dot);
                    o.v[i] = w * g.v[i];
                }
                store8<BF16, true>(dy_perm, (int64_t)row * d + c, o);
            }
        dot = wave_sum(dot);
        if ((threadIdx.x & 63) == 0) lds[j][threadIdx.x >> 6] = dot;
    }
    __syncthreads();
    if ((int)threadIdx.x < k) {
        float v = 0.f;
        for (int w = 0; w < waves; ++w) v += lds[threadIdx.x][w];
        s_dw[threadIdx.x] = v;
        dw[(int64_t)t * k + threadIdx.x] = v;
    }
    if (!dlogits) return;
    __syncthreads();
    float mean = 0.f;
    for (int j = 0; j < k; ++j) mean = fmaf(topk_w[(int64_t)t * k + j], s_dw[j], mean);
    for (int e = threadIdx.x; e < E; e += blockDim.x) {
        float v = 0.f;
        for (int j = 0; j < k; ++j)
            if (topk_idx[(int64_t)t * k + j] == e) v += topk_w[(int64_t)t * k + j] * (s_dw[j] - mean);
        dlogits[(int64_t)t * E + e] = v;
    }
}

// blocks a token and threads a block, of equal width
int token_parts(int d, int32_t dtype, int& threads) {
    const int pieces = d / (dtype == MOE_BF16 ? 8 : 4), parts = (pieces + TOKEN_THREADS - 1) / TOKEN_THREADS;
    threads = ((pieces + parts - 1) / parts + 63) / 64 * 64;
    return parts;
}

}  // namespace

hipError_t launch_dispatch(moe_ctx* c, const void* x, const int32_t* inv_perm, int32_t dtype, void* x_perm) {
    const moe_dims& D = c->dims;
    int threads;
    const int parts = token_parts(D.d, dtype, threads);
    const auto kernel = dtype == MOE_BF16 ? dispatch_kernel<true> : dispatch_kernel<false>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(D.T * parts)), dim3(threads), 0, c->stream, x, inv_perm, D.d, D.k, D.T * D.k, parts, x_perm);
    return hipGetLastError();
}

hipError_t launch_dispatch_backward(moe_ctx* c, const void* dx_perm, const int32_t* inv_perm, const void* dx_add, int32_t dtype, void* dx) {
    const moe_dims& D = c->dims;
    int threads;
    const int parts = token_parts(D.d, dtype, threads);
    const auto kernel = dtype == MOE_BF16 ? dispatch_back_kernel<true> : dispatch_back_kernel<false>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(D.T * parts)), dim3(threads), 0, c->stream, dx_perm, inv_perm, dx_add, D.d, D.k, D.T * D.k, parts,
                       dx);
    return hipGetLastError();
}

hipError_t launch_combine_backward(moe_ctx* c, const void* dy, const float* y_perm, const int32_t* inv_perm, const float* topk_w,
                                   const int32_t* topk_idx, int32_t dtype, void* dy_perm, float* dw, float* dlogits) {
    const moe_dims& D = c->dims;
    const auto kernel = dtype == MOE_BF16 ? combine_back_kernel<true> : combine_back_kernel<false>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)D.T), dim3(TOKEN_THREADS), 0, c->stream, dy, y_perm, inv_perm, topk_w, topk_idx, D.d, D.k, D.E,
                       D.T * D.k, dy_perm, dw, dlogits);
    return hipGetLastError();
}

}  // namespace moe355
