// Clipped policy loss on logits: log-probabilities, entropy, loss and the logits' gradient.
#include "grad_common.hpp"
#include "ticket.hpp"

namespace moe355 {
namespace {

constexpr int LOSS_THREADS = 512, LOSS_WAVES = LOSS_THREADS / 64;
constexpr float LOWEST = -1e30f;               // stands for -inf in z - max: its exponential is 0 and 0 times it is 0

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

// Running maximum m of z, s = sum e^(z-m), u = sum e^(z-m) (z-m): what log-sum-exp and entropy are made of
struct softmax_stats {
    float m, s, u;
    // the sums as if over a maximum of `to` >= m
    __device__ void rebase(float to) {
        if (m == to) return;
        const float d = fmaxf(m - to, LOWEST), f = __expf(d);
        u = f * fmaf(s, d, u);
        s *= f;
        m = to;
    }
    __device__ void add(float z) {             // m is a maximum that includes z, and not -inf
        const float d = fmaxf(z - m, LOWEST), e = __expf(z - m);
        s += e;
        u = fmaf(e, d, u);
    }
    __device__ void join(softmax_stats o) {
        const float to = fmaxf(m, o.m);
        if (to == -INFINITY) {                 // nothing but masked logits (or NaN, which the sums hold)
            s += o.s;
            u += o.u;
            return;
        }
        rebase(to);
        o.rebase(to);
        s += o.s;
        u += o.u;
    }
};

// a row's numbers, and its gradient e^(z-m) * (grad_a*(z-m) + grad_b), plus grad_target at the target
struct row_result {
    float m, grad_a, grad_b, grad_target;
};

__device__ inline row_result finish_row(const loss_args& a, int64_t r, const softmax_stats& st, float z_target, int target) {
    const bool known = target >= 0 && target < a.V;
    const bool empty = st.m == -INFINITY && st.s == 0.f;
    const float log_s = logf(st.s);
    const float H = empty ? 0.f : log_s - st.u / st.s;
    const float logp = !known ? 0.f : empty ? -INFINITY : (z_target - st.m) - log_s;
    const float w = a.weight[r];
    const bool live = known && !empty && w != 0.f;
    float loss = 0.f, slope = 0.f, bonus = 0.f;
    if (live) {
        const float A = a.advantage[r];
        const float low = a.clip_rows ? a.clip_rows[r] : a.clip_low, high = a.clip_rows ? a.clip_rows[r] : a.clip_high;
        if (A != 0.f) {
            const float rho = expf(logp - a.old_logp[r]);
            const float free = rho * A, held = fminf(fmaxf(rho, 1.f - low), 1.f + high) * A;
            loss = -fminf(free, held);
            if (!(free > held)) slope = -free;
            if (free != free) loss = slope = free;             // NaN is not lost in the comparisons
        }
        if (a.ref_logp && a.kl_coef != 0.f) {
            const float x = a.ref_logp[r] - logp, e = expm1f(x);
            loss = fmaf(a.kl_coef, e - x, loss);
            slope = fmaf(-a.kl_coef, e, slope);
        }
        loss = w * (loss - a.entropy_coef * H);
        slope *= w;
        bonus = w * a.entropy_coef;
    }
    a.logp[r] = logp;
    a.entropy[r] = H;
    __hip_atomic_store(a.row_loss + r, loss, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);   // the last block reads it
    if (!live) return row_result{0.f, 0.f, 0.f, 0.f};
    const float scale = a.inv_temp / st.s;
    return row_result{st.m, bonus * scale, (bonus * (H - log_s) - slope) * scale, slope * a.inv_temp};
}

// One block per row; the row is read for its sums and read again for its gradient.
template <bool BF16, bool GRAD_BF16>
__global__ __launch_bounds__(LOSS_THREADS) void loss_kernel(const loss_args a) {
    __shared__ softmax_stats s_stats[LOSS_WAVES];
    __shared__ row_result s_row;
    __shared__ int32_t s_last;
    __shared__ double s_sum[LOSS_WAVES];
    const int64_t r = blockIdx.x;
    const void* const z = row_of<BF16>(a.logits, r * a.ld);
    const int target = a.target[r];
    softmax_stats st{-INFINITY, 0.f, 0.f};
    for (int i = threadIdx.x; i < a.V; i += LOSS_THREADS) {
        const float v = load1<BF16>(z, i) * a.inv_temp;
        if (v > st.m) st.rebase(v);
        if (st.m > -INFINITY) st.add(v);
        else if (v != v) st.s = v;
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) st.join(softmax_stats{__shfl_xor(st.m, o), __shfl_xor(st.s, o), __shfl_xor(st.u, o)});
    if ((threadIdx.x & 63) == 0) s_stats[threadIdx.x >> 6] = st;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < LOSS_WAVES; ++w) st.join(s_stats[w]);
        s_row = finish_row(a, r, st, target >= 0 && target < a.V ? load1<BF16>(z, target) * a.inv_temp : 0.f, target);
    }
    __syncthreads();
    if (a.dlogits) {
        void* const out = row_of<GRAD_BF16>(a.dlogits, r * a.ld_grad);
        const row_result f = s_row;
        for (int i = threadIdx.x; i < a.V; i += LOSS_THREADS) {
            const float x = load1<BF16>(z, i) * a.inv_temp - f.m;
            float g = f.grad_a == 0.f && f.grad_b == 0.f ? 0.f : __expf(x) * fmaf(f.grad_a, fmaxf(x, LOWEST), f.grad_b);
            if (i == target) g += f.grad_target;
            store1<GRAD_BF16>(out, i, g);
        }
    }
    if (!last_block(a.ticket, gridDim.x, s_last)) return;
    double sum = 0.0;
    for (int64_t i = threadIdx.x; i < a.rows; i += LOSS_THREADS)
        sum += (double)__hip_atomic_load(a.row_loss + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
    if ((threadIdx.x & 63) == 0) s_sum[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < LOSS_WAVES; ++w) sum += s_sum[w];
        a.loss[0] = (float)sum;
    }
}

}  // namespace

hipError_t launch_policy_loss(moe_ctx* c, const void* logits, int64_t ld, int32_t dtype, int64_t rows, int32_t V, const int32_t* target,
                              const float* old_logp, const float* ref_logp, const float* advantage, const float* weight,
                              const float* clip_rows, float clip_low, float clip_high, float kl_coef, float entropy_coef, float temperature,
                              float* logp, float* entropy, float* row_loss, float* loss, void* dlogits, int64_t ld_grad, int32_t grad_dtype) {
    const loss_args a{logits,     ld,      rows,     V,          target,       old_logp,           ref_logp, advantage, weight, clip_rows, clip_low,
                      clip_high,  kl_coef, entropy_coef, 1.0f / temperature, logp, entropy, row_loss, loss,  dlogits,   ld_grad, c->grad_ticket};
    if (rows == 0) return launch_fill_i32(c->stream, reinterpret_cast<int32_t*>(loss), 1, 0);
    const auto kernel = dtype == MOE_BF16 ? (grad_dtype == MOE_BF16 ? loss_kernel<true, true> : loss_kernel<true, false>)
                                          : (grad_dtype == MOE_BF16 ? loss_kernel<false, true> : loss_kernel<false, false>);
    hipLaunchKernelGGL(kernel, dim3((unsigned)rows), dim3(LOSS_THREADS), 0, c->stream, a);
    return hipGetLastError();
}

}  // namespace moe355
