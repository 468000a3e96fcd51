// Clipped policy loss on logits: log-probabilities, entropy, loss and the logits' gradient.
#include "softmax_rows.hpp"
#include "ticket.hpp"

namespace moe355 {
namespace {

constexpr int LOSS_MAX_THREADS = 1024, LOSS_MAX_WAVES = LOSS_MAX_THREADS / 64;
constexpr int PART_THREADS = 256, MAX_PARTS = 64;   // rows in parts: a block's threads, parts of a row at most
constexpr int LOSS_HELD = 16;                  // vectors of 16 bytes of a row that a thread holds in registers

struct loss_args {
    const void* logits;
    int64_t ld, rows, first;                   // (first: of a launch)
    int V;
    const int32_t* target;
    const float *old_logp, *ref_logp, *advantage, *weight, *clip_rows;
    float clip_low, clip_high, kl_coef, entropy_coef, inv_temp;
    float *logp, *entropy, *row_loss, *loss;
    void* dlogits;
    int64_t ld_grad;
    int32_t* tickets;
    // rows in parts (few rows): their number and length in vectors, the parts' sums, the rows' tickets and results
    int parts, part_vecs;
    float* part_sums;                          // [rows][parts][3]
    struct row_result* results;                // [rows]
};

// A row's gradient: 2^y (a y + b), and `target` more at the target
struct row_result {
    float m, a, b, target;
    int live;
};

struct row_inputs {
    int target;
    float v_target;
    float old_logp, ref_logp, A, w, low, high;
};
template <bool BF16>
__device__ inline row_inputs inputs_of(const loss_args& a, int64_t r) {
    row_inputs n;
    n.target = a.target[r];
    n.v_target = 0.f;
    if (n.target >= 0 && n.target < a.V) {
        n.v_target = load1<BF16>(row_of<BF16>(a.logits, r * a.ld), n.target);
        if (n.v_target <= LOWEST) n.v_target = -INFINITY;
    }
    n.old_logp = a.old_logp[r];
    n.ref_logp = a.ref_logp ? a.ref_logp[r] : 0.f;
    n.A = a.advantage[r];
    n.w = a.weight[r];
    n.low = a.clip_rows ? a.clip_rows[r] : a.clip_low;
    n.high = a.clip_rows ? a.clip_rows[r] : a.clip_high;
    return n;
}

// e^x - 1 and, in `above`, e^x - 1 - x
__device__ inline double exp_minus_one(double x, double& above) {
    if (!(x > -0.5 && x < 0.5)) {
        const double e = exp2_of(x * (1.0 / LN2)) - 1.0;
        above = e - x;                         // (x = -inf: the slope e stays -1 where the term is infinite)
        return e;
    }
    const float t = (float)x;
    float p = 1.f / 362880.f;
    for (const float c : {1.f / 40320.f, 1.f / 5040.f, 1.f / 720.f, 1.f / 120.f, 1.f / 24.f, 1.f / 6.f, 0.5f}) p = fmaf(p, t, c);
    above = (double)p * x * x;
    return above + x;
}

// One thread.  Sums and products in fp64: a loss near zero is the difference of terms that are not
__device__ inline row_result finish_row(const loss_args& a, int64_t r, const softmax_stats& st, const row_inputs& n) {
    const bool known = n.target >= 0 && n.target < a.V;
    const bool empty = st.m == -INFINITY && st.s == 0.f;
    const double log_s = st.s > 0.f && st.s < INFINITY ? log2_of(st.s) * LN2 : (double)logf(st.s);
    const float mean = st.u / st.s;            // (of y: a rounding of H at most)
    const double H = empty ? 0.0 : log_s - (double)mean * LN2;
    const double logp = !known ? 0.0 : empty ? -INFINITY : ((double)n.v_target - (double)st.m) * (double)a.inv_temp - log_s;
    // (a masked target: the ratio is zero and the KL term infinite, with gradients that are 0 * inf.  Nothing can be learnt from a token that the policy
    // excludes)
    const bool live = known && !empty && n.w != 0.f && n.v_target != -INFINITY;
    double loss = 0.0, slope = 0.0;
    if (live) {
        const double A = n.A;
        if (A != 0.0) {
            const double rho = exp2_of((logp - (double)n.old_logp) * (1.0 / LN2));
            const double free = rho * A, held = fmin(fmax(rho, 1.0 - (double)n.low), 1.0 + (double)n.high) * A;
            loss = -fmin(free, held);
            if (!(free > held)) slope = -free;
            if (free != free) loss = slope = free;             // NaN is not lost in the comparisons
        }
        if (a.ref_logp && a.kl_coef != 0.f) {
            double above;
            const double e = exp_minus_one((double)n.ref_logp - logp, above);
            loss += (double)a.kl_coef * above;
            slope -= (double)a.kl_coef * e;
        }
        loss = (double)n.w * (loss - (double)a.entropy_coef * H);
        slope *= (double)n.w;
    }
    a.logp[r] = (float)logp;
    a.entropy[r] = (float)H;
    __hip_atomic_store(a.row_loss + r, (float)loss, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);   // the last block reads it
    if (!live) return row_result{0.f, 0.f, 0.f, 0.f, 0};
    const float scale = a.inv_temp / st.s;
    const double bonus = (double)n.w * (double)a.entropy_coef;
    return row_result{st.m, (float)(bonus * LN2) * scale, (float)(bonus * (H - log_s) - slope) * scale, (float)(slope * (double)a.inv_temp), 1};
}

// Whether row r is the last to be finished: rows arrive in groups and the groups' last ones at the launch's ticket, because arrivals at
// one address are taken one after another (15 ns each: 8192 rows of 4001 logits 135 us).  One thread, whose loss has reached the point
// where all L2 caches agree.
__device__ inline bool last_row(const loss_args& a, int64_t r) {
    const int groups = (int)(a.rows < GRAD_GROUPS ? a.rows : GRAD_GROUPS), g = (int)(r % groups);
    const int of_group = (int)((a.rows - g + groups - 1) / groups);
    return last_to_arrive(DeviceCount{a.tickets + (1 + g) * GRAD_TICKET_INTS}, of_group) && last_to_arrive(DeviceCount{a.tickets}, groups);
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

// A row's gradient, written vector by vector
template <bool BF16, bool GRAD_BF16>
struct row_grad {
    static constexpr int N = row_type<BF16>::N;
    const row_result f;
    void* const out;
    const float c;
    const int target, at;
    __device__ row_grad(const loss_args& a, int64_t r, const row_result& f_, int target_)
        : f(f_), out(row_of<GRAD_BF16>(a.dlogits, r * a.ld_grad)), c(a.inv_temp * LOG2E), target(target_), at(target_ / N) {}
    __device__ float of(float v) const {
        const float y = (v - f.m) * c;
        return __builtin_amdgcn_exp2f(y) * fmaf(f.a, fmaxf(y, Y_LOWEST), f.b);
    }
    __device__ void put(const u32x4& v, int i) const {
        float g[N] = {};
        if (f.live) {                          // (the same for the whole block)
#pragma unroll
            for (int j = 0; j < N; ++j) g[j] = of(row_type<BF16>::at(v, j));
            if (at == i) {
#pragma unroll
                for (int j = 0; j < N; ++j) g[j] += target % N == j ? f.target : 0.f;
            }
        }
        store_grad<GRAD_BF16, N>(out, i, g);
    }
    __device__ void put_one(float v, int i) const { store1<GRAD_BF16>(out, i, f.live ? of(v) + (target == i ? f.target : 0.f) : 0.f); }
};

// dz[v] = (dlogp (1[v = target] - p_v) + w entropy_coef p_v (log p_v + H)) / temperature, which is 2^y (a y + b) for numbers a, b of the row.
// Bound by the bytes, logits once and gradients once, and by the vector ALU: with one row to a CU its copies, sums and gradient follow one another, and an
// instruction for each logit is 14 us of 4096 x 131072 bf16, 476 us = 4.5 TB/s (a copy: 4.87; v c - m c in one instruction each, which large logits do not
// allow, 456).  333 x 50001 f32 32 us where a copy takes 20.5: a row is held by the registers of one CU, and 77 of the rows have a second round.
// One block per row.  HELD: the row stays in registers between the two passes that its maximum and its sum ask for and the pass
// that writes its gradient, so it is read once; otherwise it is read again for the gradient.
template <bool BF16, bool GRAD_BF16, bool HELD>
__global__ __launch_bounds__(LOSS_MAX_THREADS) void loss_kernel(const loss_args a) {
    typedef row_type<BF16> T;
    constexpr int N = T::N;
    __shared__ block_scratch s_scratch;
    __shared__ row_result s_row;
    __shared__ int32_t s_last;
    __shared__ double s_sum[LOSS_MAX_WAVES];
    const int64_t r = a.first + blockIdx.x;
    const int tid = threadIdx.x, threads = blockDim.x;
    const void* const z = row_of<BF16>(a.logits, r * a.ld);
    const int vecs = a.V / N, rest = a.V % N;                  // thread t < rest has element t behind the vectors as well
    running_sums<BF16> sums(a.inv_temp * LOG2E);
    u32x4 held[LOSS_HELD];
    if (HELD) {
#pragma unroll
        for (int n = 0; n < LOSS_HELD; ++n) {
            const int i = tid + n * threads;
            held[n] = i < vecs ? T::load(z, i) : T::none();
        }
    }
    const float extra = tid < rest ? load1<BF16>(z, vecs * N + tid) : -INFINITY;
    const row_inputs in = inputs_of<BF16>(a, r);
    softmax_stats st;
    if (HELD) {
        sums.take(block_largest(fmaxf(extra, sums.largest(held)), s_scratch));
        keep_packed(held);
        sums.sum(held);
        keep_packed(held);
        sums.one(extra, sums.base());
        st = block_sums(sums.st, s_scratch);
    } else {
        int i = tid;
        for (; i + 3 * threads < vecs; i += 4 * threads) {     // four in flight
            u32x4 v[4];
#pragma unroll
            for (int n = 0; n < 4; ++n) v[n] = T::load(z, i + n * threads);
            sums.add(v);
        }
        for (; i < vecs; i += threads) {
            const u32x4 v[1] = {T::load(z, i)};
            sums.add(v);
        }
        if (tid < rest) sums.add_one(extra);
        st = block_join(sums.st, sums.c, s_scratch);
    }
    if (tid == 0) {
        s_row = finish_row(a, r, st, in);
        s_last = 0;
        if (a.rows <= GRAD_MAX_SPLIT_ROWS) {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // the row's loss has reached the point where all L2 caches agree
            s_last = last_row(a, r);
        }
    }
    __syncthreads();
    if (a.dlogits) {
        const row_grad<BF16, GRAD_BF16> grad(a, r, s_row, in.target);
        if (!grad.f.live) {                    // (apart from the loops below, so that they have no branch for each vector)
            const float none[N] = {};
            for (int i = tid; i < vecs; i += threads) store_grad<GRAD_BF16, N>(grad.out, i, none);
        } else if (HELD) {
#pragma unroll
            for (int n = 0; n < LOSS_HELD; ++n) {
                const int i = tid + n * threads;
                if (i < vecs) grad.put(held[n], i);
            }
        } else {
            int i = tid;
            for (; i + 3 * threads < vecs; i += 4 * threads) {
                u32x4 v[4];
#pragma unroll
                for (int n = 0; n < 4; ++n) v[n] = T::load(z, i + n * threads);
#pragma unroll
                for (int n = 0; n < 4; ++n) grad.put(v[n], i + n * threads);
            }
            for (; i < vecs; i += threads) grad.put(T::load(z, i), i);
        }
        if (tid < rest) grad.put_one(extra, vecs * N + tid);
    }
    if (s_last) total_loss(a, s_sum);
}

// The total of many rows, in a launch of its own: their blocks need not wait for a ticket each
__global__ __launch_bounds__(LOSS_MAX_THREADS) void loss_total_kernel(const loss_args a) {
    __shared__ double s_sum[LOSS_MAX_WAVES];
    total_loss(a, s_sum);
}

// Few rows, in parts: a block has the sums of one part, the last block of a row joins them in the parts' order and finishes the row.
template <bool BF16>
__global__ __launch_bounds__(PART_THREADS) void loss_part_kernel(const loss_args a) {
    typedef row_type<BF16> T;
    constexpr int N = T::N;
    __shared__ block_scratch s_scratch;
    __shared__ int32_t s_last;
    __shared__ double s_sum[LOSS_MAX_WAVES];
    const int64_t r = blockIdx.x / a.parts;
    const int part = blockIdx.x % a.parts, tid = threadIdx.x;
    const void* const z = row_of<BF16>(a.logits, r * a.ld);
    const int vecs = a.V / N, first = part * a.part_vecs, end = min(first + a.part_vecs, vecs);
    const float c = a.inv_temp * LOG2E;
    const row_inputs in = inputs_of<BF16>(a, r);
    running_sums<BF16> sums(c);
    int i = first + tid;
    for (; i + 3 * PART_THREADS < end; i += 4 * PART_THREADS) {  // four in flight
        u32x4 v[4];
#pragma unroll
        for (int n = 0; n < 4; ++n) v[n] = T::load(z, i + n * PART_THREADS);
        sums.add(v);
    }
    for (; i < end; i += PART_THREADS) {
        const u32x4 v[1] = {T::load(z, i)};
        sums.add(v);
    }
    if (part == 0 && tid < a.V % N) sums.add_one(load1<BF16>(z, vecs * N + tid));
    softmax_stats st = block_join(sums.st, sums.c, s_scratch);
    float* const mine = a.part_sums + (r * a.parts + part) * 3;
    if (tid == 0) {
        __hip_atomic_store(mine, st.m, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __hip_atomic_store(mine + 1, st.s, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __hip_atomic_store(mine + 2, st.u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    if (!last_block(a.tickets + (1 + GRAD_GROUPS + r) * GRAD_TICKET_INTS, a.parts, s_last)) return;
    const float* const all = a.part_sums + r * a.parts * 3;
    if (tid < 64) {                            // (at most 64 parts: a lane has one)
        st = softmax_stats{-INFINITY, 0.f, 0.f};
        if (tid < a.parts)
            st = softmax_stats{__hip_atomic_load(all + tid * 3, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT),
                               __hip_atomic_load(all + tid * 3 + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT),
                               __hip_atomic_load(all + tid * 3 + 2, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)};
        const float m = wave_largest(st.m);
        if (m > -INFINITY) rebase(st, m, c);
        st = softmax_stats{m, wave_total(st.s), wave_total(st.u)};
    }
    if (tid == 0) {
        a.results[r] = finish_row(a, r, st, in);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        s_last = last_row(a, r);
    }
    __syncthreads();
    if (s_last) total_loss(a, s_sum);
}

template <bool BF16, bool GRAD_BF16>
__global__ __launch_bounds__(PART_THREADS) void loss_part_grad_kernel(const loss_args a) {
    typedef row_type<BF16> T;
    constexpr int N = T::N;
    const int64_t r = blockIdx.x / a.parts;
    const int part = blockIdx.x % a.parts, tid = threadIdx.x;
    const void* const z = row_of<BF16>(a.logits, r * a.ld);
    const int vecs = a.V / N, rest = a.V % N, first = part * a.part_vecs, end = min(first + a.part_vecs, vecs);
    const row_grad<BF16, GRAD_BF16> grad(a, r, a.results[r], a.target[r]);
    const float extra = part == 0 && tid < rest ? load1<BF16>(z, vecs * N + tid) : 0.f;
    int i = first + tid;
    for (; i + 3 * PART_THREADS < end; i += 4 * PART_THREADS) {
        u32x4 v[4];
#pragma unroll
        for (int n = 0; n < 4; ++n) v[n] = T::load(z, i + n * PART_THREADS);
#pragma unroll
        for (int n = 0; n < 4; ++n) grad.put(v[n], i + n * PART_THREADS);
    }
    for (; i < end; i += PART_THREADS) grad.put(T::load(z, i), i);
    if (part == 0 && tid < rest) grad.put_one(extra, vecs * N + tid);
}

// Parts of a row: long rows that alone leave much of the chip idle.  With a gradient that makes two launches of one and the row is read
// twice: 64 x 131072 bf16 25 -> 18 us, 128 28.5 -> 22.5, but 192 31 -> 34 and 100 x 64000 15.4 -> 16.3; f32 rows of the same 16-byte vectors lose a little:
// 64 x 32768 10.5 -> 12.4, 128 x 60000 17.4 -> 19.6, 128 x 131072 31.2 -> 33.3, 200 x 60000 20 -> 27.  Without: 8 x 60000 f32 10 -> 8, 500 x 60000 f32
// 32 -> 27.5, 512 x 131072 bf16 46.5 -> 33, f32 level, 500 x 32768 f32 15.4 -> 16.7.  GRAD_MAX_SPLIT_ROWS is how many rows have a ticket, no measured bound
// (600 x 131072 bf16 in one block each: 60 us).
int loss_parts(int64_t rows, int vecs, bool gradient) {
    if (vecs < 8192 || rows > (gradient ? 128 : GRAD_MAX_SPLIT_ROWS)) return 1;
    const int64_t parts = 1024 / rows < vecs / 512 ? 1024 / rows : vecs / 512;
    return parts > MAX_PARTS ? MAX_PARTS : (int)parts;
}

constexpr int64_t LOSS_MAX_GRID = 1 << 21;     // blocks of a launch: a grid has fewer than 2^32 threads

}  // namespace

hipError_t launch_policy_loss(moe_ctx* c, const void* logits, int64_t ld, int32_t dtype, int64_t rows, int32_t V, const int32_t* target,
                              const float* old_logp, const float* ref_logp, const float* advantage, const float* weight,
                              const float* clip_rows, float clip_low, float clip_high, float kl_coef, float entropy_coef, float temperature,
                              float* logp, float* entropy, float* row_loss, float* loss, void* dlogits, int64_t ld_grad, int32_t grad_dtype) {
    loss_args a{logits,    ld,        rows,    0,            V,                  target, old_logp, ref_logp, advantage, weight,  clip_rows,
                clip_low,  clip_high, kl_coef, entropy_coef, 1.0f / temperature, logp,   entropy,  row_loss, loss,      dlogits, ld_grad,
                c->grad_tickets};
    if (rows == 0) return launch_fill_i32(c->stream, reinterpret_cast<int32_t*>(loss), 1, 0);
    const int vecs = V / (dtype == MOE_BF16 ? 8 : 4);
    const int parts = loss_parts(rows, vecs, dlogits != nullptr);
    if (parts > 1) {
        a.parts = parts;
        a.part_vecs = (vecs + parts - 1) / parts;
        a.part_sums = static_cast<float*>(c->grad_ws);
        a.results = reinterpret_cast<row_result*>(a.part_sums + (int64_t)GRAD_MAX_SPLIT_ROWS * MAX_PARTS * 3);
        const unsigned grid = (unsigned)(rows * parts);
        if (dtype == MOE_BF16) loss_part_kernel<true><<<grid, PART_THREADS, 0, c->stream>>>(a);
        else loss_part_kernel<false><<<grid, PART_THREADS, 0, c->stream>>>(a);
        if (dlogits) {
            if (dtype == MOE_BF16) {
                if (grad_dtype == MOE_BF16) loss_part_grad_kernel<true, true><<<grid, PART_THREADS, 0, c->stream>>>(a);
                else loss_part_grad_kernel<true, false><<<grid, PART_THREADS, 0, c->stream>>>(a);
            } else if (grad_dtype == MOE_BF16) loss_part_grad_kernel<false, true><<<grid, PART_THREADS, 0, c->stream>>>(a);
            else loss_part_grad_kernel<false, false><<<grid, PART_THREADS, 0, c->stream>>>(a);
        }
        return hipGetLastError();
    }
    const bool held = vecs <= LOSS_MAX_THREADS * LOSS_HELD;
    int threads = held ? (vecs / LOSS_HELD + 63) / 64 * 64 : LOSS_MAX_THREADS;
    if (threads < 64) threads = 64;
    if (held && threads * LOSS_HELD < vecs) threads += 64;
    auto launch = [&](auto kernel) {
        for (; a.first < rows; a.first += LOSS_MAX_GRID)
            hipLaunchKernelGGL(kernel, dim3((unsigned)(rows - a.first < LOSS_MAX_GRID ? rows - a.first : LOSS_MAX_GRID)), dim3(threads), 0, c->stream, a);
        if (rows > GRAD_MAX_SPLIT_ROWS) loss_total_kernel<<<1, LOSS_MAX_THREADS, 0, c->stream>>>(a);
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
