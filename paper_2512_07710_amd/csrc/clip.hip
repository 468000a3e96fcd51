// The norm of a list of gradients, and the list scaled down to a largest norm.
#include "grad_common.hpp"

namespace moe355 {
namespace {

constexpr int LIST_THREADS = 256, LIST_MAX = 128;              // gradients of a launch: they travel in the kernel's arguments
constexpr int LIST_MAX_BLOCKS = 1 << 22;

// Consecutive pieces of `chunk` elements of the gradients, one for each block
struct list_args {
    const void* grads[LIST_MAX];
    void* outs[LIST_MAX];
    int64_t counts[LIST_MAX];
    uint32_t first[LIST_MAX + 1];              // block of each gradient's first piece
    uint32_t bf16[LIST_MAX / 32];              // types, a bit each
    int n;
    int64_t chunk;
};
struct list_piece {
    const void* grad;
    void* out;
    int64_t begin, end;
    bool bf16;
};
__device__ inline list_piece piece_of(const list_args& a, uint32_t block) {
    int lo = 0, hi = a.n - 1;                  // the last gradient that begins at this block or before it (empty ones begin where the next does)
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (a.first[mid] <= block) lo = mid;
        else hi = mid - 1;
    }
    const int64_t begin = (int64_t)(block - a.first[lo]) * a.chunk, count = a.counts[lo];
    return list_piece{a.grads[lo], a.outs[lo], begin, begin + a.chunk < count ? begin + a.chunk : count, (a.bf16[lo / 32] >> (lo % 32) & 1) != 0};
}

template <bool BF16>
__device__ inline double squares(const list_piece& p) {
    double sum = 0.0;
    for (int64_t i = p.begin + threadIdx.x; i < p.end; i += LIST_THREADS) {
        const double v = load1<BF16>(p.grad, i);
        sum = fma(v, v, sum);
    }
    return sum;
}
__device__ inline double block_total(double v, double* lds) {  // in thread 0
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    for (int w = 1; w < LIST_THREADS / 64; ++w) v += threadIdx.x == 0 ? lds[w] : 0.0;
    return v;
}
__global__ __launch_bounds__(LIST_THREADS) void squares_kernel(const list_args a, double* __restrict__ sums) {
    __shared__ double s[LIST_THREADS / 64];
    const list_piece p = piece_of(a, blockIdx.x);
    const double sum = block_total(p.bf16 ? squares<true>(p) : squares<false>(p), s);
    if (threadIdx.x == 0) sums[blockIdx.x] = sum;
}
__global__ __launch_bounds__(LIST_THREADS) void norm_total_kernel(const double* __restrict__ sums, int64_t n, double* __restrict__ sum_sq, float* norm) {
    __shared__ double s[LIST_THREADS / 64];
    double v = 0.0;
    for (int64_t i = threadIdx.x; i < n; i += LIST_THREADS) v += sums[i];
    v = block_total(v, s);
    if (threadIdx.x == 0) {
        *sum_sq = v;
        if (norm) *norm = (float)sqrt(v);
    }
}

template <bool BF16>
__device__ inline void scale_piece(const list_piece& p, float factor) {
    for (int64_t i = p.begin + threadIdx.x; i < p.end; i += LIST_THREADS) store1<BF16>(p.out, i, load1<BF16>(p.grad, i) * factor);
}
__device__ inline float clip_factor(double sum_sq, float max_norm) {
    const double f = (double)max_norm / sqrt(sum_sq);
    return sum_sq == 0.0 || f >= 1.0 ? 1.f : (float)f;         // (NaN stays)
}
__global__ __launch_bounds__(LIST_THREADS) void clip_kernel(const list_args a, const double* __restrict__ sum_sq, float max_norm) {
    const float factor = clip_factor(*sum_sq, max_norm);
    const list_piece p = piece_of(a, blockIdx.x);
    if (factor == 1.f && p.grad == p.out) return;
    if (p.bf16) scale_piece<true>(p, factor);
    else scale_piece<false>(p, factor);
}

// The list in launches of LIST_MAX gradients: launch(arguments, blocks)
template <class Launch>
hipError_t for_list(const void* const* grads, void* const* outs, const int64_t* counts, const int32_t* dtypes, int32_t n, int64_t chunk, Launch launch) {
    list_args a;
    hipError_t e = hipSuccess;
    a.chunk = chunk;
    for (int at = 0; at < n && e == hipSuccess; at += LIST_MAX) {
        a.n = n - at < LIST_MAX ? n - at : LIST_MAX;
        uint32_t blocks = 0;
        for (uint32_t& w : a.bf16) w = 0;
        for (int i = 0; i < a.n; ++i) {
            a.grads[i] = grads[at + i];
            a.outs[i] = outs ? outs[at + i] : const_cast<void*>(grads[at + i]);
            a.counts[i] = counts[at + i];
            a.first[i] = blocks;
            a.bf16[i / 32] |= (uint32_t)(dtypes[at + i] == MOE_BF16) << (i % 32);
            blocks += (uint32_t)((counts[at + i] + chunk - 1) / chunk);
        }
        a.first[a.n] = blocks;
        if (blocks) {
            launch(a, blocks);
            e = hipGetLastError();
        }
    }
    return e;
}
// Elements of a piece: so many that all pieces have a place for their sum
int64_t list_chunk(const int64_t* counts, int32_t n, int64_t& pieces) {
    for (int64_t chunk = 16384;; chunk *= 2) {
        pieces = 0;
        for (int i = 0; i < n; ++i) pieces += (counts[i] + chunk - 1) / chunk;
        if (pieces <= LIST_MAX_BLOCKS) return chunk;
    }
}

}  // namespace

hipError_t launch_grad_norm(moe_ctx* c, const void* const* grads, const int64_t* counts, const int32_t* dtypes, int32_t n, double* sum_sq, float* norm) {
    static_assert(LIST_MAX_BLOCKS * sizeof(double) <= GRAD_WS_BYTES, "a sum for each piece");
    int64_t pieces;
    const int64_t chunk = list_chunk(counts, n, pieces);
    double* const sums = static_cast<double*>(c->grad_ws);
    int64_t done = 0;
    const hipError_t e = for_list(grads, nullptr, counts, dtypes, n, chunk, [&](const list_args& a, uint32_t blocks) {
        squares_kernel<<<blocks, LIST_THREADS, 0, c->stream>>>(a, sums + done);
        done += blocks;
    });
    if (e != hipSuccess) return e;
    norm_total_kernel<<<1, LIST_THREADS, 0, c->stream>>>(sums, pieces, sum_sq, norm);
    return hipGetLastError();
}

hipError_t launch_clip_grads(hipStream_t s, const void* const* grads, const int64_t* counts, const int32_t* dtypes, int32_t n, const double* sum_sq,
                             float max_norm, void* const* outs) {
    int64_t pieces;
    const int64_t chunk = list_chunk(counts, n, pieces);
    return for_list(grads, outs, counts, dtypes, n, chunk,
                    [&](const list_args& a, uint32_t blocks) { clip_kernel<<<blocks, LIST_THREADS, 0, s>>>(a, sum_sq, max_norm); });
}

}  // namespace moe355
