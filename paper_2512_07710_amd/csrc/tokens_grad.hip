// Token rows in expert order, and the gradients of that order and of the weighted combine.
#include "grad_common.hpp"

namespace moe355 {
namespace {

constexpr int TOKEN_THREADS = 256, COMBINE_MAX_THREADS = 1024;

// 16 bytes of a row
template <bool BF16>
struct piece {
    static constexpr int N = BF16 ? 8 : 4;
    static __device__ const u32x4* at(const void* rows, int64_t row, int d, int i) { return static_cast<const u32x4*>(rows) + row * (d / N) + i; }
    static __device__ u32x4* at(void* rows, int64_t row, int d, int i) { return static_cast<u32x4*>(rows) + row * (d / N) + i; }
    static __device__ float value(const u32x4& v, int j) { return BF16 ? (j & 1 ? bf16hi(v[j >> 1]) : bf16lo(v[j >> 1])) : __uint_as_float(v[j]); }
};

// x_perm[row(t,j)] = x[t]: a copy, bound by the k rows that it writes.  One block per token and part of its columns; a thread owns 16 bytes of the row
// (d is a multiple of 128), reads them once and writes them k times.  16 x 7168 bf16, k = 8 takes 6 us, the time of any short launch.
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

// dx[t] = sum_j dx_perm[row(t,j)] + dx_add[t], summed in 32 bits in the order of the slots, rounded once.  The split of dispatch_kernel; the rows of four
// slots are on their way at a time: 777 x 2176 f32, k = 5 7.7 us (one slot after the other, 8 columns to a thread: 12.0).
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

// dy_perm[row(t,j)] = w(t,j) dy[t],  dw(t,j) = dy[t] . y_perm[row(t,j)],  dlogits[t,e] = sum over slots with idx = e of w (dw - sum_i w_i dw_i): the
// weights are a softmax over the chosen experts' logits, so their Jacobian is diag(w) - w w^T.
// One block per token: dw of all its slots meet in LDS, where the logits' gradient is made.  A thread owns four columns of every blockDim-th piece
// and has four pieces on their way.  Bound by the bytes of the expert rows, read once and written once, both past the caches: 32768 x 7168, k = 8,
// bf16 2260 us = 5.21 TB/s (a copy: 4.87).  With eight columns to a thread the fp32 row came in loads that leave out every other 16 bytes and one
// piece at a time: 2365 us, and 777 x 2176 f32, k = 5 23.6 us where this takes 19.6.
template <bool BF16, int THREADS>
__global__ __launch_bounds__(THREADS) void combine_back_kernel(const void* __restrict__ dy, const float* __restrict__ y_perm,
                                                               const int32_t* __restrict__ inv_perm, const float* __restrict__ topk_w,
                                                               const int32_t* __restrict__ topk_idx, int d, int k, int E, int N,
                                                               void* __restrict__ dy_perm, float* __restrict__ dw,
                                                               float* __restrict__ dlogits) {
    __shared__ float lds[MAX_K][THREADS / 64], s_dw[MAX_K];
    constexpr int AT_ONCE = 4;
    const int t = blockIdx.x, waves = blockDim.x >> 6, step = blockDim.x * 4;
    for (int j = 0; j < k; ++j) {
        const int row = inv_perm[(int64_t)t * k + j];
        const float w = topk_w[(int64_t)t * k + j];
        float dot = 0.f;
        if ((uint32_t)row < (uint32_t)N)
            for (int c0 = threadIdx.x * 4; c0 < d; c0 += AT_ONCE * step) {
                f32x4 y[AT_ONCE], g[AT_ONCE];
#pragma unroll
                for (int u = 0; u < AT_ONCE; ++u) {
                    const int c = c0 + u * step;
                    if (c >= d) continue;
                    y[u] = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(y_perm + (int64_t)row * d + c));
                    if (BF16) {
                        const u32x2 v = *reinterpret_cast<const u32x2*>(static_cast<const uint16_t*>(dy) + (int64_t)t * d + c);
                        g[u] = f32x4{bf16lo(v[0]), bf16hi(v[0]), bf16lo(v[1]), bf16hi(v[1])};
                    } else {
                        g[u] = *reinterpret_cast<const f32x4*>(static_cast<const float*>(dy) + (int64_t)t * d + c);
                    }
                }
#pragma unroll
                for (int u = 0; u < AT_ONCE; ++u) {
                    const int c = c0 + u * step;
                    if (c >= d) continue;
#pragma unroll
                    for (int i = 0; i < 4; ++i) dot = fmaf(g[u][i], y[u][i], dot);
                    const f32x4 o = g[u] * w;
                    if (BF16)
                        __builtin_nontemporal_store(u32x2{bf16_pair(o[0], o[1]), bf16_pair(o[2], o[3])},
                                                    reinterpret_cast<u32x2*>(static_cast<uint16_t*>(dy_perm) + (int64_t)row * d + c));
                    else
                        __builtin_nontemporal_store(o, reinterpret_cast<f32x4*>(static_cast<float*>(dy_perm) + (int64_t)row * d + c));
                }
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
    // Few tokens leave most CUs idle: a row to as many threads as there are columns for.  d = 4096, k = 5, bf16, 256 threads and 1024: 64 tokens 14.4 us
    // and 8.4, 512 tokens 18.1 and 14.5, 1024 tokens 27.7 and 28.8, 4096 (d = 5120, k = 8) 201 and 206.
    const bool few = D.T < 1024;
    const int threads = !few ? TOKEN_THREADS : D.d / 4 < COMBINE_MAX_THREADS ? (D.d / 4 + 63) / 64 * 64 : COMBINE_MAX_THREADS;
    const auto kernel = dtype == MOE_BF16 ? (few ? combine_back_kernel<true, COMBINE_MAX_THREADS> : combine_back_kernel<true, TOKEN_THREADS>)
                                          : (few ? combine_back_kernel<false, COMBINE_MAX_THREADS> : combine_back_kernel<false, TOKEN_THREADS>);
    hipLaunchKernelGGL(kernel, dim3((unsigned)D.T), dim3(threads), 0, c->stream, dy, y_perm, inv_perm, topk_w, topk_idx, D.d, D.k, D.E,
                       D.T * D.k, dy_perm, dw, dlogits);
    return hipGetLastError();
}

}  // namespace moe355
