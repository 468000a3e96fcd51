// Log-probabilities of given tokens, entropy and the most likely tokens of rows of logits; and the logits' gradient from those of the first two.
#include "softmax_rows.hpp"

namespace moe355 {
namespace {

constexpr int LOGP_THREADS = 256;
constexpr int64_t LOGP_MAX_GRID = 1 << 22;

struct logp_args {
    const void* logits;
    int64_t ld, rows, first;                   // (first: of a launch)
    int V, m, n;
    const int32_t* ids;
    float inv_temp;
    float *logp, *entropy, *top_logp, *stats;
    int32_t* top_idx;
};

// (v - m) / temperature - log s to fp32's resolution: in fp64, the logits as they are
__device__ inline float logp_of(float v, const softmax_stats& st, double log_s, float inv_temp) {
    if (v <= LOWEST && st.s == st.s) return -INFINITY;
    return (float)(((double)v - (double)st.m) * (double)inv_temp - log_s);
}

// One block per row.  The alternatives one after the other, each the largest behind the one before
template <bool BF16>
__global__ __launch_bounds__(LOGP_THREADS) void logp_kernel(const logp_args a) {
    typedef row_type<BF16> T;
    constexpr int N = T::N;
    __shared__ block_scratch s_scratch;
    __shared__ float s_v[LOGP_THREADS / 64];
    __shared__ int s_i[LOGP_THREADS / 64];
    const int64_t r = a.first + blockIdx.x;
    const int tid = threadIdx.x, vecs = a.V / N, rest = a.V % N;
    const void* const z = row_of<BF16>(a.logits, r * a.ld);
    running_sums<BF16> sums(a.inv_temp * LOG2E);
    for (int i = tid; i < vecs; i += LOGP_THREADS) {
        const u32x4 v[1] = {T::load(z, i)};
        sums.add(v);
    }
    if (tid < rest) sums.add_one(load1<BF16>(z, vecs * N + tid));
    const softmax_stats st = block_join(sums.st, sums.c, s_scratch);
    const bool empty = st.m == -INFINITY && st.s == 0.f;
    const double log_s = st.s > 0.f && st.s < INFINITY ? log2_of(st.s) * LN2 : (double)logf(st.s);
    if (tid < a.m) {
        const int id = a.ids[r * a.m + tid];
        float lp = 0.f;
        if ((uint32_t)id < (uint32_t)a.V) lp = empty ? -INFINITY : logp_of(load1<BF16>(z, id), st, log_s, a.inv_temp);
        a.logp[r * a.m + tid] = lp;
    }
    if (tid == 0) {
        if (a.entropy) a.entropy[r] = empty ? 0.f : (float)(log_s - (double)(st.u / st.s) * LN2);
        if (a.stats) {
            a.stats[2 * r] = st.m;
            a.stats[2 * r + 1] = st.s;
        }
    }
    float last = INFINITY;                     // the alternative before: its logit and place
    int last_i = -1;
    for (int k = 0; k < a.n; ++k) {
        float best = LOWEST;
        int best_i = -1;
        for (int i = tid; i < a.V; i += LOGP_THREADS) {
            const float v = load1<BF16>(z, i);
            if (v > best && (v < last || (v == last && i > last_i))) best = v, best_i = i;
        }
        auto better = [&](float v, int i) {
            if (v > best || (v == best && i >= 0 && i < best_i)) best = v, best_i = i;
        };
        for (int o = 32; o > 0; o >>= 1) {
            const float v = __shfl_xor(best, o);
            better(v, __shfl_xor(best_i, o));
        }
        if ((tid & 63) == 0) s_v[tid >> 6] = best, s_i[tid >> 6] = best_i;
        __syncthreads();
        for (int w = 0; w < LOGP_THREADS / 64; ++w) better(s_v[w], s_i[w]);
        __syncthreads();
        if (tid == 0) {
            a.top_idx[r * a.n + k] = best_i;
            a.top_logp[r * a.n + k] = best_i < 0 ? -INFINITY : logp_of(best, st, log_s, a.inv_temp);
        }
        last = best;
        last_i = best_i;
    }
}

struct logp_grad_args {
    const void* logits;
    int64_t ld, ld_grad, rows, first;
    int V, m;
    const int32_t* ids;
    float inv_temp;
    const float *dlogp, *dentropy, *stats, *entropy;
    void* dlogits;
};

// dz[v] = (sum_j dlogp_j (1[v = id_j] - p_v) - dH p_v (log p_v + H)) / temperature = 2^y (a y + b), and more at the given tokens.  One block per row
template <bool BF16, bool GRAD_BF16>
__global__ __launch_bounds__(LOGP_THREADS) void logp_grad_kernel(const logp_grad_args a) {
    typedef row_type<BF16> T;
    constexpr int N = T::N;
    __shared__ float s_d[LOGP_MAX_GIVEN], s_v[LOGP_MAX_GIVEN];
    __shared__ int s_id[LOGP_MAX_GIVEN];
    const int64_t r = a.first + blockIdx.x;
    const int tid = threadIdx.x, vecs = a.V / N, rest = a.V % N;
    const void* const z = row_of<BF16>(a.logits, r * a.ld);
    void* const out = row_of<GRAD_BF16>(a.dlogits, r * a.ld_grad);
    const float m = a.stats[2 * r], s = a.stats[2 * r + 1], dH = a.dentropy ? a.dentropy[r] : 0.f;
    if (tid < a.m) {
        const int id = a.ids[r * a.m + tid];
        float v = 0.f, d = 0.f;
        if ((uint32_t)id < (uint32_t)a.V && (v = load1<BF16>(z, id), !(v <= LOWEST))) d = a.dlogp[r * a.m + tid];
        s_id[tid] = id;
        s_v[tid] = v;
        s_d[tid] = d;
    }
    const float extra = tid < rest ? load1<BF16>(z, vecs * N + tid) : 0.f;
    __syncthreads();
    float sum = 0.f;
    bool live = dH != 0.f;
    for (int j = 0; j < a.m; ++j) {
        sum += s_d[j];
        live |= s_d[j] != 0.f;
    }
    live &= !(m == -INFINITY && s == 0.f);
    const float c = a.inv_temp * LOG2E, scale = a.inv_temp / s;
    const double log_s = s > 0.f && s < INFINITY ? log2_of(s) * LN2 : (double)logf(s), H = dH != 0.f ? (double)a.entropy[r] : 0.0;
    const float ka = (float)(-(double)dH * LN2) * scale, kb = (float)((double)dH * (log_s - H) - (double)sum) * scale;
    auto of = [&](float v) {
        const float y = (v - m) * c;
        return __builtin_amdgcn_exp2f(y) * fmaf(ka, fmaxf(y, Y_LOWEST), kb);
    };
    for (int i = tid; i < vecs; i += LOGP_THREADS) {
        float g[N] = {};
        if (live) {
            const u32x4 v = T::load(z, i);
#pragma unroll
            for (int j = 0; j < N; ++j) g[j] = of(T::at(v, j));
        }
        store_grad<GRAD_BF16, N>(out, i, g);
    }
    if (tid < rest) store1<GRAD_BF16>(out, vecs * N + tid, live ? of(extra) : 0.f);
    if (!live) return;
    // the given tokens, by the threads that have written their places: one with several gradients receives their sum as often
    for (int j = 0; j < a.m; ++j) {
        const int id = s_id[j];
        if ((uint32_t)id >= (uint32_t)a.V || (id < vecs * N ? (id / N) % LOGP_THREADS : id - vecs * N) != tid || s_v[j] <= LOWEST) continue;
        float d = 0.f;
        for (int k = 0; k < a.m; ++k) d += s_id[k] == id ? s_d[k] : 0.f;
        store1<GRAD_BF16>(out, id, fmaf(d, a.inv_temp, of(s_v[j])));
    }
}

template <class Kernel, class Args>
hipError_t launch_rows(hipStream_t s, Kernel kernel, Args a) {
    for (a.first = 0; a.first < a.rows; a.first += LOGP_MAX_GRID)
        hipLaunchKernelGGL(kernel, dim3((unsigned)(a.rows - a.first < LOGP_MAX_GRID ? a.rows - a.first : LOGP_MAX_GRID)), dim3(LOGP_THREADS), 0, s, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_token_logp(moe_ctx* c, const void* logits, int64_t ld, int32_t dtype, int64_t rows, int32_t V, const int32_t* ids, int32_t m,
                             float temperature, float* logp, float* entropy, int32_t n, int32_t* top_idx, float* top_logp, float* stats) {
    const logp_args a{logits, ld, rows, 0, V, m, n, ids, 1.0f / temperature, logp, entropy, top_logp, stats, top_idx};
    return dtype == MOE_BF16 ? launch_rows(c->stream, logp_kernel<true>, a) : launch_rows(c->stream, logp_kernel<false>, a);
}

hipError_t launch_token_logp_backward(hipStream_t s, const void* logits, int64_t ld, int32_t dtype, int64_t rows, int32_t V, const int32_t* ids, int32_t m,
                                      float temperature, const float* dlogp, const float* dentropy, const float* stats, const float* entropy,
                                      void* dlogits, int64_t ld_grad, int32_t grad_dtype) {
    const logp_grad_args a{logits, ld, ld_grad, rows, 0, V, m, ids, 1.0f / temperature, dlogp, dentropy, stats, entropy, dlogits};
    if (dtype == MOE_BF16) return grad_dtype == MOE_BF16 ? launch_rows(s, logp_grad_kernel<true, true>, a) : launch_rows(s, logp_grad_kernel<true, false>, a);
    return grad_dtype == MOE_BF16 ? launch_rows(s, logp_grad_kernel<false, true>, a) : launch_rows(s, logp_grad_kernel<false, false>, a);
}

}  // namespace moe355
