// The norm of a list of gradients, and the list scaled down to a largest norm.
#include "grad_common.hpp"
#include "ticket.hpp"

namespace moe355 {
namespace {

constexpr int LIST_THREADS = 256, AT_ONCE = 4;
constexpr int LIST_ARGS = 128;                         // gradients that a launch takes in its arguments; longer lists are put into the workspace first
constexpr int LIST_MAX_PIECES = 1 << 22;
constexpr int LIST_PIECES = 8192;                      // of a long list, about
constexpr int64_t LEAST_CHUNK = 4096, MOST_CHUNK = 65536;
constexpr int64_t LIST_TABLE = (int64_t)32 << 20;      // where the workspace has the table of a list; in front of it the pieces' sums

struct list_entry {
    const void* grad;
    void* out;
    int64_t count;                                     // negative: of bf16 numbers, ~count of them
};
// Gradients cut into pieces of `chunk` elements, one for each block; first: a gradient's first piece
struct list_args {
    list_entry entry[LIST_ARGS];
    uint32_t first[LIST_ARGS];
};
struct list_table {
    const list_entry* entry;
    const uint32_t* first;
    int n;
    int64_t chunk;
    uint32_t pieces;
};
struct list_piece {
    const void* grad;
    void* out;
    int64_t n;
    bool bf16;
};

// The last gradient that begins at this piece or in front of it (empty ones begin where the next does): 64 looked at together
template <class First>
__device__ inline int gradient_of(uint32_t piece, int n, First first) {
    const int lane = threadIdx.x & 63;
    int at = 0;
    for (int step = (n + 63) / 64;; step = (step + 63) / 64) {
        const int k = at + lane * step;
        at += (__popcll(__ballot(k < n && first(k < n ? k : 0) <= piece)) - 1) * step;
        if (step == 1) return at;
    }
}
__device__ inline list_piece piece_of(const list_entry& e, uint32_t first, int64_t chunk, uint32_t piece) {
    const bool bf16 = e.count < 0;
    const int64_t count = bf16 ? ~e.count : e.count, begin = (int64_t)(piece - first) * chunk, bytes = begin * (bf16 ? 2 : 4);
    return list_piece{static_cast<const char*>(e.grad) + bytes, static_cast<char*>(e.out) + bytes, begin + chunk < count ? chunk : count - begin, bf16};
}
template <bool ARGS>
__device__ inline list_piece find_piece(const list_args& a, const list_table& t, uint32_t piece) {
    if (ARGS) {
        const int g = __builtin_amdgcn_readfirstlane(gradient_of(piece, t.n, [&](int k) { return a.first[k]; }));
        return piece_of(a.entry[g], a.first[g], t.chunk, piece);
    }
    const int g = __builtin_amdgcn_readfirstlane(gradient_of(piece, t.n, [&](int k) { return t.first[k]; }));
    return piece_of(t.entry[g], t.first[g], t.chunk, piece);
}

// 16 bytes at any element
template <bool BF16>
struct sixteen {
    static constexpr int N = BF16 ? 8 : 4;
    static __device__ u32x4 load(const void* p, int64_t i) { return *reinterpret_cast<const u32x4_any*>(static_cast<const char*>(p) + i * 16); }
    static __device__ float at(const u32x4& v, int j) { return BF16 ? (j & 1 ? bf16hi(v[j >> 1]) : bf16lo(v[j >> 1])) : __uint_as_float(v[j & 3]); }
};
// vector(v, i) for the vectors of a thread, one(i) for its element behind them
template <bool BF16, class Vector, class One>
__device__ inline void for_piece(const list_piece& p, Vector vector, One one) {
    typedef sixteen<BF16> S;
    const int64_t vecs = p.n / S::N;
    int64_t i = threadIdx.x;
    for (; i + (AT_ONCE - 1) * LIST_THREADS < vecs; i += AT_ONCE * LIST_THREADS) {
        u32x4 v[AT_ONCE];
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) v[u] = S::load(p.grad, i + u * LIST_THREADS);
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) vector(v[u], i + u * LIST_THREADS);
    }
    for (; i < vecs; i += LIST_THREADS) vector(S::load(p.grad, i), i);
    if (vecs * S::N + threadIdx.x < p.n) one(vecs * S::N + threadIdx.x);
}

template <bool BF16>
__device__ inline double squares(const list_piece& p) {
    double sum[2] = {};
    for_piece<BF16>(p,
                    [&](const u32x4& v, int64_t) {
#pragma unroll
                        for (int j = 0; j < sixteen<BF16>::N; ++j) {
                            const double x = sixteen<BF16>::at(v, j);
                            sum[j & 1] = fma(x, x, sum[j & 1]);
                        }
                    },
                    [&](int64_t i) {
                        const double x = load1<BF16>(p.grad, i);
                        sum[0] = fma(x, x, sum[0]);
                    });
    return sum[0] + sum[1];
}
__device__ inline double block_total(double v, double* lds) {  // in thread 0
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    for (int w = 1; w < LIST_THREADS / 64; ++w) v += threadIdx.x == 0 ? lds[w] : 0.0;
    return v;
}
// Whether this is the last piece to be summed: pieces arrive in groups, whose last ones arrive at one ticket (arrivals at one address are taken one after another)
__device__ inline bool last_piece(int32_t* tickets, uint32_t piece, uint32_t pieces) {
    const uint32_t groups = pieces < GRAD_GROUPS ? pieces : GRAD_GROUPS, g = piece % groups;
    return last_to_arrive(DeviceCount{tickets + (1 + g) * GRAD_TICKET_INTS}, (int)((pieces - g + groups - 1) / groups)) && last_to_arrive(DeviceCount{tickets}, (int)groups);
}
// Squares in fp64: no fp32 number's is out of its range, and the sum of 2^40 of them has 13 digits.  The last block adds up the pieces' sums in their order.
// Bound by the bytes: 700 gradients of 2.8 GB 460 us, 6.0 TB/s read; 60 of 0.8 MB 5.4, the load, the piece's sum and the two tickets one behind the other.
template <bool ARGS>
__global__ __launch_bounds__(LIST_THREADS) void squares_kernel(const list_args a, const list_table t, double* sums, int32_t* tickets, double* sum_sq, float* norm) {
    __shared__ double s[LIST_THREADS / 64];
    __shared__ int32_t s_last;
    const uint32_t piece = blockIdx.x;
    const list_piece p = find_piece<ARGS>(a, t, piece);
    double v = block_total(p.bf16 ? squares<true>(p) : squares<false>(p), s);
    if (threadIdx.x == 0) {
        __hip_atomic_store(sums + piece, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // the sum has reached the point where all L2 caches agree
        s_last = last_piece(tickets, piece, t.pieces);
    }
    __syncthreads();
    if (!s_last) return;
    v = 0.0;
    for (uint32_t i = threadIdx.x; i < t.pieces; i += 8 * LIST_THREADS) {
        double x[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) x[u] = __hip_atomic_load(sums + (i + u * LIST_THREADS < t.pieces ? i + u * LIST_THREADS : i), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
        for (int u = 0; u < 8; ++u) v += i + u * LIST_THREADS < t.pieces ? x[u] : 0.0;
    }
    v = block_total(v, s);
    if (threadIdx.x == 0) {
        *sum_sq = v;
        if (norm) *norm = (float)sqrt(v);
    }
}
__global__ void no_squares_kernel(double* sum_sq, float* norm) {
    *sum_sq = 0.0;
    if (norm) *norm = 0.f;
}

template <bool BF16>
__device__ inline void scale_piece(const list_piece& p, float factor) {
    for_piece<BF16>(p,
                    [&](const u32x4& v, int64_t i) {
                        u32x4 o;
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            o[j] = BF16 ? bf16_pair(sixteen<BF16>::at(v, (2 * j) % sixteen<BF16>::N) * factor, sixteen<BF16>::at(v, (2 * j + 1) % sixteen<BF16>::N) * factor)
                                        : __float_as_uint(sixteen<BF16>::at(v, j) * factor);
                        __builtin_nontemporal_store(o, reinterpret_cast<u32x4_any*>(static_cast<char*>(p.out) + i * 16));
                    },
                    [&](int64_t i) { store1<BF16>(p.out, i, load1<BF16>(p.grad, i) * factor); });
}
__device__ inline float clip_factor(double sum_sq, float max_norm) {
    const double f = (double)max_norm / sqrt(sum_sq);
    return sum_sq == 0.0 || f >= 1.0 ? 1.f : (float)f;         // (NaN stays)
}
// The pieces from the last to the first: what the norm's pass has read last is in the caches still.  Bound by the bytes: the 700 gradients into others 1059 us,
// 5.2 TB/s read and written; 60 small ones 2.4.  In two launches with the norm: the factor needs every piece's sum, and a wait inside a kernel for all blocks,
// pieces kept in registers, would hold no more than 0.1 GB of them.
template <bool ARGS>
__global__ __launch_bounds__(LIST_THREADS) void clip_kernel(const list_args a, const list_table t, const double* __restrict__ sum_sq, float max_norm) {
    const float factor = clip_factor(*sum_sq, max_norm);
    const list_piece p = find_piece<ARGS>(a, t, t.pieces - 1 - blockIdx.x);
    if (factor == 1.f && p.grad == p.out) return;
    if (p.bf16) scale_piece<true>(p, factor);
    else scale_piece<false>(p, factor);
}

// Gradients of a long list, as many as a launch takes, into the workspace's table
__global__ __launch_bounds__(LIST_ARGS) void table_kernel(const list_args a, int n, list_entry* __restrict__ entry, uint32_t* __restrict__ first) {
    const int k = threadIdx.x;
    if (k >= n) return;
    entry[k] = a.entry[k];
    first[k] = a.first[k];
}

// Pieces of a list: `chunk` elements each, a multiple of what a block has on its way
list_table cut_list(const int64_t* counts, int32_t n) {
    list_table t{};
    int64_t total = 0, pieces;
    for (int i = 0; i < n; ++i) total += counts[i];
    t.n = n;
    t.chunk = LEAST_CHUNK;
    while (t.chunk < MOST_CHUNK && t.chunk * LIST_PIECES < total) t.chunk *= 2;
    for (;; t.chunk *= 2) {
        pieces = 0;
        for (int i = 0; i < n; ++i) pieces += (counts[i] + t.chunk - 1) / t.chunk;
        if (pieces <= LIST_MAX_PIECES) break;
    }
    t.pieces = (uint32_t)pieces;
    return t;
}
// launch(arguments, table) for the whole list
template <class Launch>
hipError_t for_list(moe_ctx* c, list_table t, const void* const* grads, void* const* outs, const int64_t* counts, const int32_t* dtypes, Launch launch) {
    static_assert((size_t)LIST_MAX_PIECES * sizeof(double) <= LIST_TABLE && LIST_TABLE + (size_t)LIST_MAX_GRADS * (sizeof(list_entry) + 4) <= GRAD_WS_BYTES, "workspace");
    list_entry* const entry = reinterpret_cast<list_entry*>(static_cast<char*>(c->grad_ws) + LIST_TABLE);
    uint32_t* const first = reinterpret_cast<uint32_t*>(entry + LIST_MAX_GRADS);
    t.entry = entry;
    t.first = first;
    list_args a;
    uint32_t pieces = 0;
    for (int at = 0; at < t.n; at += LIST_ARGS) {
        const int n = t.n - at < LIST_ARGS ? t.n - at : LIST_ARGS;
        for (int i = 0; i < n; ++i) {
            const int64_t count = counts[at + i];
            a.entry[i] = list_entry{grads[at + i], outs ? outs[at + i] : const_cast<void*>(grads[at + i]), dtypes[at + i] == MOE_BF16 ? ~count : count};
            a.first[i] = pieces;
            pieces += (uint32_t)((count + t.chunk - 1) / t.chunk);
        }
        if (t.n > LIST_ARGS) table_kernel<<<1, LIST_ARGS, 0, c->stream>>>(a, n, entry + at, first + at);
    }
    launch(a, t);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_grad_norm(moe_ctx* c, const void* const* grads, const int64_t* counts, const int32_t* dtypes, int32_t n, double* sum_sq, float* norm) {
    const list_table t = cut_list(counts, n);
    if (t.pieces == 0) {
        no_squares_kernel<<<1, 1, 0, c->stream>>>(sum_sq, norm);
        return hipGetLastError();
    }
    return for_list(c, t, grads, nullptr, counts, dtypes, [&](const list_args& a, const list_table& t) {
        auto kernel = n <= LIST_ARGS ? squares_kernel<true> : squares_kernel<false>;
        kernel<<<t.pieces, LIST_THREADS, 0, c->stream>>>(a, t, static_cast<double*>(c->grad_ws), c->grad_tickets, sum_sq, norm);
    });
}

hipError_t launch_clip_grads(moe_ctx* c, const void* const* grads, const int64_t* counts, const int32_t* dtypes, int32_t n, const double* sum_sq,
                             float max_norm, void* const* outs) {
    const list_table t = cut_list(counts, n);
    if (t.pieces == 0) return hipSuccess;
    return for_list(c, t, grads, outs, counts, dtypes, [&](const list_args& a, const list_table& t) {
        auto kernel = n <= LIST_ARGS ? clip_kernel<true> : clip_kernel<false>;
        kernel<<<t.pieces, LIST_THREADS, 0, c->stream>>>(a, t, sum_sq, max_norm);
    });
}

}  // namespace moe355
