// Clipped policy loss on logits: log-probabilities, entropy, loss and the logits' gradient.
#include "grad_common.hpp"
#include "ticket.hpp"

namespace moe355 {
namespace {

constexpr int LOSS_MAX_THREADS = 1024, LOSS_MAX_WAVES = LOSS_MAX_THREADS / 64;
constexpr int LOSS_HELD = 16;                  // vectors of 16 bytes of a row that a thread holds in registers
constexpr float LOWEST = -1e30f;               // logits not above it are masked; and in place of -inf in y it makes 2^y y = 0
constexpr float LOG2E = 1.44269504088896340736f;
constexpr double LN2 = 0.69314718055994530942;

struct loss_args {
    const void* logits;
    int64_t ld, rows;
    int V;
    const int32_t* target;
    const float *old_logp, *ref_logp, *advantage, *weight, *clip_rows;
    float clip_low, clip_high, kl_coef, entropy_coef, inv_temp;
    float *logp, *entropy, *row_loss, *loss;
    void* dlogits;
    int64_t ld_grad;
    int32_t* ticket;
};

// Sums over logits in units of log 2, y = z log2 e - m: s = sum 2^y, u = sum y 2^y, which log-sum-exp and entropy are made of.  m is the whole
// number next to the largest z log2 e: so y is one fused multiply-add of the logit, rounded once, and sums over different m are
// brought together by exact powers of two.  m = -inf: nothing but masked logits so far (or NaN, which the sums hold)
struct softmax_stats {
    float m, s, u;
};
__device__ inline void rebase(softmax_stats& t, float to) {
    if (t.m == to) return;
    const float d = fmaxf(t.m - to, LOWEST), f = __builtin_amdgcn_exp2f(d);
    t.u = f * fmaf(t.s, d, t.u);
    t.s *= f;
    t.m = to;
}
__device__ inline softmax_stats join(softmax_stats a, softmax_stats b) {
    const float to = fmaxf(a.m, b.m);
    if (to > -INFINITY) {
        rebase(a, to);
        rebase(b, to);
    }
    return softmax_stats{to, a.s + b.s, a.u + b.u};
}
// joined over the block, in every thread; lds: one for each wave
__device__ inline softmax_stats block_join(softmax_stats t, softmax_stats* lds) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) t = join(t, softmax_stats{__shfl_xor(t.m, o), __shfl_xor(t.s, o), __shfl_xor(t.u, o)});
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = t;
    __syncthreads();
    t = lds[0];
    for (int w = 1; w < (int)(blockDim.x >> 6); ++w) t = join(t, lds[w]);
    return t;
}

// 16 bytes of a row, at any element: rows of odd length start at odd places
typedef u32x4 __attribute__((aligned(2))) u32x4_any;
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

__device__ inline uint32_t bf16_pair(float a, float b) {       // round to nearest even
    typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, v2bf{(__bf16)a, (__bf16)b});
}
// vector i of N gradients
template <bool BF16, int N>
__device__ inline void store_grad(void* row, int64_t i, const float (&g)[N]) {
    char* const p = static_cast<char*>(row) + i * N * (BF16 ? 2 : 4);
    if (BF16 && N == 8) *reinterpret_cast<u32x4_any*>(p) = u32x4{bf16_pair(g[0], g[1]), bf16_pair(g[2], g[3]), bf16_pair(g[4], g[5]), bf16_pair(g[6], g[7])};
    else if (BF16) *reinterpret_cast<u32x2_any*>(p) = u32x2{bf16_pair(g[0], g[1]), bf16_pair(g[2], g[3])};
    else
#pragma unroll
        for (int h = 0; h < N; h += 4)
            *reinterpret_cast<u32x4_any*>(p + h * 4) = u32x4{__float_as_uint(g[h]), __float_as_uint(g[h + 1]), __float_as_uint(g[h + 2]), __float_as_uint(g[h + 3])};
}

// A row's gradient: 2^y (a y + b), and `target` more at the target
struct row_result {
    float m, a, b, target;
    int live;
};

struct row_inputs {
    int target;
    double z_target;
    float old_logp, ref_logp, A, w, low, high;
};
template <bool BF16>
__device__ inline row_inputs inputs_of(const loss_args& a, int64_t r) {
    row_inputs n;
    n.target = a.target[r];
    n.z_target = 0.0;
    if (n.target >= 0 && n.target < a.V) {
        const float v = load1<BF16>(row_of<BF16>(a.logits, r * a.ld), n.target);
        n.z_target = v <= LOWEST ? -INFINITY : (double)v * (double)a.inv_temp;
    }
    n.old_logp = a.old_logp[r];
    n.ref_logp = a.ref_logp ? a.ref_logp[r] : 0.f;
    n.A = a.advantage[r];
    n.w = a.weight[r];
    n.low = a.clip_rows ? a.clip_rows[r] : a.clip_low;
    n.high = a.clip_rows ? a.clip_rows[r] : a.clip_high;
    return n;
}

// One thread.  In fp64 from the row's sums on: a loss near zero is the difference of terms that are not
__device__ inline row_result finish_row(const loss_args& a, int64_t r, const softmax_stats& st, const row_inputs& n) {
    const bool known = n.target >= 0 && n.target < a.V;
    const bool empty = st.m == -INFINITY && st.s == 0.f;
    const double log_s = log((double)st.s), H = empty ? 0.0 : log_s - (double)st.u / (double)st.s * LN2;
    const double logp = !known ? 0.0 : empty ? -INFINITY : n.z_target - (double)st.m * LN2 - log_s;
    const bool live = known && !empty && n.w != 0.f;
    double loss = 0.0, slope = 0.0;
    if (live) {
        const double A = n.A;
        if (A != 0.0) {
            const double rho = exp(logp - (double)n.old_logp);
            const double free = rho * A, held = fmin(fmax(rho, 1.0 - (double)n.low), 1.0 + (double)n.high) * A;
            loss = -fmin(free, held);
            if (!(free > held)) slope = -free;
            if (free != free) loss = slope = free;             // NaN is not lost in the comparisons
        }
        if (a.ref_logp && a.kl_coef != 0.f) {
            const double x = (double)n.ref_logp - logp, e = expm1(x);
            loss += (double)a.kl_coef * (e - x);
            slope -= (double)a.kl_coef * e;
        }
        loss = (double)n.w * (loss - (double)a.entropy_coef * H);
        slope *= (double)n.w;
    }
    a.logp[r] = (float)logp;
    a.entropy[r] = (float)H;
    __hip_atomic_store(a.row_loss + r, (float)loss, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);   // the last block reads it
    if (!live) return row_result{0.f, 0.f, 0.f, 0.f, 0};
    const double scale = (double)a.inv_temp / (double)st.s, bonus = (double)n.w * (double)a.entropy_coef;
    return row_result{st.m, (float)(bonus * LN2 * scale), (float)((bonus * (H - log_s) - slope) * scale),
                      (float)(slope * (double)a.inv_temp), 1};
}

// Sum of all rows' losses, by the block that found itself the last one
__device__ inline void total_loss(const loss_args& a, double* lds) {
    double sum = 0.0;
    for (int64_t i = threadIdx.x; i < a.rows; i += blockDim.x) sum += (double)__hip_atomic_load(a.row_loss + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < (int)(blockDim.x >> 6); ++w) sum += lds[w];
        a.loss[0] = (float)sum;
    }
}

// The vectors stay as they were loaded: without this the compiler keeps the unpacked values of one pass for the next, twice the registers
__device__ inline void keep_packed(u32x4 (&v)[LOSS_HELD]) {
#pragma unroll
    for (int n = 0; n < LOSS_HELD; ++n) asm volatile("" : "+v"(v[n]));
}

// One block per row.  HELD: the row stays in registers between the two passes that its maximum and its sum ask for and the pass
// that writes its gradient, so it is read once; otherwise it is read again for each of them.
template <bool BF16, bool GRAD_BF16, bool HELD>
__global__ __launch_bounds__(LOSS_MAX_THREADS) void loss_kernel(const loss_args a) {
    typedef row_type<BF16> T;
    constexpr int N = T::N;
    __shared__ softmax_stats s_stats[LOSS_MAX_WAVES];
    __shared__ row_result s_row;
    __shared__ int32_t s_last;
    __shared__ double s_sum[LOSS_MAX_WAVES];
    const int64_t r = blockIdx.x;
    const int tid = threadIdx.x, threads = blockDim.x;
    const void* const z = row_of<BF16>(a.logits, r * a.ld);
    const int vecs = a.V / N, rest = a.V % N;                  // thread t < rest has element t behind the vectors as well
    const row_inputs in = inputs_of<BF16>(a, r);
    const float c = a.inv_temp * LOG2E;
    u32x4 held[LOSS_HELD];
    const float extra = tid < rest ? load1<BF16>(z, vecs * N + tid) : -INFINITY;
    softmax_stats st{-INFINITY, 0.f, 0.f};
    auto whole = [&](float v) { return v > LOWEST ? rintf(v * c) : -INFINITY; };
    auto sums = [&](const u32x4& v, float base) {              // base = -m
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const float y = fmaf(T::at(v, j), c, base), e = __builtin_amdgcn_exp2f(y);
            st.s += e;
            st.u = fmaf(e, fmaxf(y, LOWEST), st.u);
        }
    };
    auto sums_extra = [&](float base) {
        if (tid >= rest) return;
        const float y = fmaf(extra, c, base), e = __builtin_amdgcn_exp2f(y);
        st.s += e;
        st.u = fmaf(e, fmaxf(y, LOWEST), st.u);
    };
    float top = extra;
    if (HELD) {
#pragma unroll
        for (int n = 0; n < LOSS_HELD; ++n) {
            const int i = tid + n * threads;
            held[n] = i < vecs ? T::load(z, i) : T::none();
        }
#pragma unroll
        for (int n = 0; n < LOSS_HELD; ++n)
#pragma unroll
            for (int j = 0; j < N; ++j) top = fmaxf(top, T::at(held[n], j));
        // (a thread's own maximum serves its sums; a thread with nothing but masked logits has empty sums, unless one of them is NaN)
        st.m = whole(top);
        const float base = st.m > -INFINITY ? -st.m : 0.f;
        keep_packed(held);
#pragma unroll
        for (int n = 0; n < LOSS_HELD; ++n) sums(held[n], base);
        sums_extra(base);
        keep_packed(held);
    } else {
        for (int i = tid; i < vecs; i += threads) {
            const u32x4 v = T::load(z, i);
            float m = T::at(v, 0);
#pragma unroll
            for (int j = 1; j < N; ++j) m = fmaxf(m, T::at(v, j));
            if (whole(m) > st.m) rebase(st, whole(m));
            sums(v, st.m > -INFINITY ? -st.m : 0.f);
        }
        if (tid < rest) {
            if (whole(extra) > st.m) rebase(st, whole(extra));
            sums_extra(st.m > -INFINITY ? -st.m : 0.f);
        }
    }
    st = block_join(st, s_stats);
    if (tid == 0) {
        s_row = finish_row(a, r, st, in);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // the row's loss has reached the point where all L2 caches agree
        s_last = last_to_arrive(DeviceCount{a.ticket}, (int)gridDim.x);
    }
    __syncthreads();
    if (a.dlogits) {
        void* const out = row_of<GRAD_BF16>(a.dlogits, r * a.ld_grad);
        const row_result f = s_row;
        if (!f.live) {
            const float none[N] = {};
            for (int i = tid; i < vecs; i += threads) store_grad<GRAD_BF16, N>(out, i, none);
            if (tid < rest) store1<GRAD_BF16>(out, vecs * N + tid, 0.f);
        } else {
            auto grad = [&](float v) {
                const float y = fmaf(v, c, -f.m);
                return __builtin_amdgcn_exp2f(y) * fmaf(f.a, fmaxf(y, LOWEST), f.b);
            };
            const int at = in.target / N;
            auto put = [&](const u32x4& v, int i) {
                float g[N];
#pragma unroll
                for (int j = 0; j < N; ++j) g[j] = grad(T::at(v, j));
                if (at == i) {
#pragma unroll
                    for (int j = 0; j < N; ++j) g[j] += in.target % N == j ? f.target : 0.f;
                }
                store_grad<GRAD_BF16, N>(out, i, g);
            };
            if (HELD) {
#pragma unroll
                for (int n = 0; n < LOSS_HELD; ++n) {
                    const int i = tid + n * threads;
                    if (i < vecs) put(held[n], i);
                }
            } else {
                for (int i = tid; i < vecs; i += threads) put(T::load(z, i), i);
            }
            if (tid < rest) {
                const int i = vecs * N + tid;
                store1<GRAD_BF16>(out, i, grad(extra) + (in.target == i ? f.target : 0.f));
            }
        }
    }
    if (s_last) total_loss(a, s_sum);
}

}  // namespace

hipError_t launch_policy_loss(moe_ctx* c, const void* logits, int64_t ld, int32_t dtype, int64_t rows, int32_t V, const int32_t* target,
                              const float* old_logp, const float* ref_logp, const float* advantage, const float* weight,
                              const float* clip_rows, float clip_low, float clip_high, float kl_coef, float entropy_coef, float temperature,
                              float* logp, float* entropy, float* row_loss, float* loss, void* dlogits, int64_t ld_grad, int32_t grad_dtype) {
    const loss_args a{logits,     ld,      rows,     V,          target,       old_logp,           ref_logp, advantage, weight, clip_rows, clip_low,
                      clip_high,  kl_coef, entropy_coef, 1.0f / temperature, logp, entropy, row_loss, loss,  dlogits,   ld_grad, c->grad_ticket};
    if (rows == 0) return launch_fill_i32(c->stream, reinterpret_cast<int32_t*>(loss), 1, 0);
    const int vecs = V / (dtype == MOE_BF16 ? 8 : 4);
    const bool held = vecs <= LOSS_MAX_THREADS * LOSS_HELD;
    int threads = held ? (vecs / LOSS_HELD + 63) / 64 * 64 : LOSS_MAX_THREADS;
    if (threads < 64) threads = 64;
    if (held && threads * LOSS_HELD < vecs) threads += 64;
    auto launch = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)rows), dim3(threads), 0, c->stream, a);
        return hipGetLastError();
    };
    if (dtype == MOE_BF16) {
        if (grad_dtype == MOE_BF16) return held ? launch(loss_kernel<true, true, true>) : launch(loss_kernel<true, true, false>);
        return held ? launch(loss_kernel<true, false, true>) : launch(loss_kernel<true, false, false>);
    }
    if (grad_dtype == MOE_BF16) return held ? launch(loss_kernel<false, true, true>) : launch(loss_kernel<false, true, false>);
    return held ? launch(loss_kernel<false, false, true>) : launch(loss_kernel<false, false, false>);
}

}  // namespace moe355
