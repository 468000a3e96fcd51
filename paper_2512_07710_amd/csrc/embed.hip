// Rows of an embedding table for token ids, and the table's gradient by sorted tokens.
#include "grad_common.hpp"

namespace moe355 {
namespace {

constexpr int EMBED_THREADS = 256, EMBED_MAX_GRID = 1 << 22;
constexpr int SORT_CHUNK = 1024, MERGE_WAYS = 32;
constexpr uint64_t NO_KEY = ~(uint64_t)0;      // behind every key
constexpr uint32_t NO_ID = 0xFFFFFFFFu;        // of the keys of tokens outside the table: behind the others

// Eight columns of a row from column i on, those that there are
template <bool BF16>
__device__ inline vec8 row_load8(const void* row, int64_t i, int d) {
    if (i + 8 <= d) {
        raw8<BF16> r;
        r.load(row, i);
        vec8 v;
#pragma unroll
        for (int j = 0; j < 8; ++j) v.v[j] = r.at(j);
        return v;
    }
    vec8 v = {};
    for (int j = 0; i + j < d; ++j) v.v[j] = load1<BF16>(row, i + j);
    return v;
}
template <bool BF16>
__device__ inline void row_store8(void* row, int64_t i, int d, const vec8& v) {
    if (i + 8 <= d) store8_any<BF16>(row, i, v);
    else
        for (int j = 0; i + j < d; ++j) store1<BF16>(row, i + j, v.v[j]);
}

struct embed_args {
    const int32_t* ids;
    const void* table;
    void* y;
    int64_t ld, ld_y, first;
    int V, d, parts;
    float scale;
};
// y[t] = scale table[ids[t]]: a copy, one block per token and part of its columns
template <bool BF16, bool OUT_BF16>
__global__ __launch_bounds__(EMBED_THREADS) void embed_kernel(const embed_args a) {
    const int64_t b = a.first + blockIdx.x, t = b / a.parts;
    const int i = ((int)(b % a.parts) * EMBED_THREADS + threadIdx.x) * 8;
    if (i >= a.d) return;
    const int id = a.ids[t];
    vec8 v = {};
    if ((uint32_t)id < (uint32_t)a.V) {
        v = row_load8<BF16>(row_of<BF16>(a.table, id * a.ld), i, a.d);
#pragma unroll
        for (int j = 0; j < 8; ++j) v.v[j] *= a.scale;
    }
    row_store8<OUT_BF16>(row_of<OUT_BF16>(a.y, t * a.ld_y), i, a.d, v);
}

// Keys (id, token) in ascending order: tokens of one id stand together in the order of the batch.  Each block sorts SORT_CHUNK tokens
__global__ __launch_bounds__(SORT_CHUNK) void sort_tokens_kernel(const int32_t* __restrict__ ids, int64_t T, int V, uint64_t* __restrict__ keys) {
    __shared__ uint64_t s[SORT_CHUNK];
    const int i = threadIdx.x;
    const int64_t t = (int64_t)blockIdx.x * SORT_CHUNK + i;
    uint64_t mine = NO_KEY;
    if (t < T) {
        const uint32_t id = (uint32_t)ids[t];
        mine = (uint64_t)(id < (uint32_t)V ? id : NO_ID) << 32 | (uint32_t)t;
    }
    s[i] = mine;
    __syncthreads();
    for (int size = 2; size <= SORT_CHUNK; size *= 2)
        for (int step = size / 2; step > 0; step /= 2) {
            const uint64_t other = s[i ^ step];
            const bool up = !(i & size), low = !(i & step);
            mine = (mine < other) == (up == low) ? mine : other;
            __syncthreads();
            s[i] = mine;
            __syncthreads();
        }
    if (t < T) keys[t] = mine;
}

// Sorted runs of `run` keys, MERGE_WAYS of them to one: a key's place is the number of keys in the runs that are smaller (no two are equal)
__global__ __launch_bounds__(EMBED_THREADS) void merge_tokens_kernel(const uint64_t* __restrict__ keys, int64_t T, int64_t run, uint64_t* __restrict__ out) {
    const int64_t i = (int64_t)blockIdx.x * EMBED_THREADS + threadIdx.x;
    if (i >= T) return;
    const uint64_t mine = keys[i];
    const int64_t first = i / (run * MERGE_WAYS) * (run * MERGE_WAYS);
    int64_t place = first;
    for (int64_t at = first; at < T && at < first + run * MERGE_WAYS; at += run) {
        int64_t lo = at, hi = at + run < T ? at + run : T;
        while (lo < hi) {
            const int64_t mid = (lo + hi) / 2;
            if (keys[mid] < mine) lo = mid + 1;
            else hi = mid;
        }
        place += lo - at;
    }
    out[place] = mine;
}

struct embed_back_args {
    const void* dy;
    const uint64_t* keys;
    void* dtable;
    int64_t ld, ld_grad, T, first;
    int V, d, parts, accumulate;
    float scale;
};
template <bool GRAD_BF16>
__global__ __launch_bounds__(EMBED_THREADS) void embed_zero_kernel(const embed_back_args a) {
    const int64_t b = a.first + blockIdx.x;
    const int i = ((int)(b % a.parts) * EMBED_THREADS + threadIdx.x) * 8;
    if (i < a.d) row_store8<GRAD_BF16>(row_of<GRAD_BF16>(a.dtable, b / a.parts * a.ld_grad), i, a.d, vec8{});
}
// One block per sorted token and part of the columns; that of a token's first occurrence adds up all of them
template <bool BF16, bool GRAD_BF16>
__global__ __launch_bounds__(EMBED_THREADS) void embed_sum_kernel(const embed_back_args a) {
    const int64_t b = a.first + blockIdx.x, p = b / a.parts;
    const int i = ((int)(b % a.parts) * EMBED_THREADS + threadIdx.x) * 8;
    const uint32_t id = (uint32_t)(a.keys[p] >> 32);
    if (i >= a.d || id == NO_ID || (p > 0 && (uint32_t)(a.keys[p - 1] >> 32) == id)) return;
    vec8 sum = {};
    for (int64_t q = p; q < a.T && (uint32_t)(a.keys[q] >> 32) == id; ++q) {
        const vec8 v = row_load8<BF16>(row_of<BF16>(a.dy, (int64_t)(uint32_t)a.keys[q] * a.ld), i, a.d);
#pragma unroll
        for (int j = 0; j < 8; ++j) sum.v[j] += v.v[j];
    }
    void* const row = row_of<GRAD_BF16>(a.dtable, id * a.ld_grad);
    const vec8 was = a.accumulate ? row_load8<GRAD_BF16>(row, i, a.d) : vec8{};
#pragma unroll
    for (int j = 0; j < 8; ++j) sum.v[j] = fmaf(sum.v[j], a.scale, was.v[j]);
    row_store8<GRAD_BF16>(row, i, a.d, sum);
}

// blocks 0 .. n-1 in launches that a grid holds
template <class Kernel, class Args>
hipError_t launch_blocks(hipStream_t s, Kernel kernel, Args a, int64_t n) {
    for (a.first = 0; a.first < n; a.first += EMBED_MAX_GRID)
        hipLaunchKernelGGL(kernel, dim3((unsigned)(n - a.first < EMBED_MAX_GRID ? n - a.first : EMBED_MAX_GRID)), dim3(EMBED_THREADS), 0, s, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_embed(hipStream_t s, const int32_t* ids, int64_t T, const void* table, int32_t V, int32_t d, int64_t ld, int32_t dtype, float scale,
                        void* y, int64_t ld_y, int32_t out_dtype) {
    const int parts = (d + EMBED_THREADS * 8 - 1) / (EMBED_THREADS * 8);
    const embed_args a{ids, table, y, ld, ld_y, 0, V, d, parts, scale};
    if (dtype == MOE_BF16) return out_dtype == MOE_BF16 ? launch_blocks(s, embed_kernel<true, true>, a, T * parts) : launch_blocks(s, embed_kernel<true, false>, a, T * parts);
    return out_dtype == MOE_BF16 ? launch_blocks(s, embed_kernel<false, true>, a, T * parts) : launch_blocks(s, embed_kernel<false, false>, a, T * parts);
}

hipError_t launch_embed_backward(moe_ctx* c, const void* dy, const int32_t* ids, int64_t T, int32_t V, int32_t d, int64_t ld, int32_t dtype, float scale,
                                 int32_t accumulate, void* dtable, int64_t ld_grad, int32_t grad_dtype) {
    const int parts = (d + EMBED_THREADS * 8 - 1) / (EMBED_THREADS * 8);
    uint64_t* keys = static_cast<uint64_t*>(c->grad_ws);
    uint64_t* other = keys + EMBED_MAX_TOKENS;
    embed_back_args a{dy, keys, dtable, ld, ld_grad, T, 0, V, d, parts, accumulate, scale};
    hipError_t e = hipSuccess;
    if (!accumulate)
        e = grad_dtype == MOE_BF16 ? launch_blocks(c->stream, embed_zero_kernel<true>, a, (int64_t)V * parts)
                                   : launch_blocks(c->stream, embed_zero_kernel<false>, a, (int64_t)V * parts);
    if (e != hipSuccess || T == 0) return e;
    sort_tokens_kernel<<<(unsigned)((T + SORT_CHUNK - 1) / SORT_CHUNK), SORT_CHUNK, 0, c->stream>>>(ids, T, V, keys);
    for (int64_t run = SORT_CHUNK; run < T; run *= MERGE_WAYS) {
        merge_tokens_kernel<<<(unsigned)((T + EMBED_THREADS - 1) / EMBED_THREADS), EMBED_THREADS, 0, c->stream>>>(keys, T, run, other);
        uint64_t* const sorted = other;
        other = keys;
        keys = sorted;
    }
    a.keys = keys;
    if (dtype == MOE_BF16)
        return grad_dtype == MOE_BF16 ? launch_blocks(c->stream, embed_sum_kernel<true, true>, a, T * parts)
                                      : launch_blocks(c->stream, embed_sum_kernel<true, false>, a, T * parts);
    return grad_dtype == MOE_BF16 ? launch_blocks(c->stream, embed_sum_kernel<false, true>, a, T * parts)
                                  : launch_blocks(c->stream, embed_sum_kernel<false, false>, a, T * parts);
}

}  // namespace moe355
