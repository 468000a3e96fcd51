// Residual addition, root-mean-square norm and e4m3 coding in one pass over a row, and the norm's gradient.
#include "grad_common.hpp"
#include "grad_rules.hpp"
#include "lanes.hpp"

namespace moe355 {
namespace {

constexpr int NORM_MAX_THREADS = 1024;
constexpr int NORM_VECTORS = 4;                // vectors of eight elements that a thread holds at most

struct norm_args {
    const void *x, *residual;
    const float* gain;
    int64_t rows, first, ld_x, ld_res;         // (first: of a launch)
    int cols;
    float eps;
    void *sum, *y;
    uint8_t* q;
    float *scales, *rstd;
};

// h = x + residual (rounded to its type), r = 1 / sqrt(mean h^2 + eps), y = h r gain, q = e4m3(y / s) with s = max|y| / 448 of 128 columns.
// Rows in vectors of eight elements and what is left over, one to a thread; `per_block` neighbouring rows to a block, each in registers while the
// next is on its way, so that a row is read once and its results leave as it is done: bound by those bytes.  32768 x 7168 bf16 with residual, sum and
// codes 326 us = 5.1 TB/s (a copy: 4.87); one row of 4096 4.2 us, 8 with the call.  Thread t of a block of n holds vectors t, t+n, ...; sixteen
// neighbouring threads hold a group of 128 columns.  Scales leave in runs of NORM_ROWS words: as single words each would be a part of a cache line
// of its own.
template <bool BF16, int NV, bool REST>         // REST: cols is no multiple of eight (an instance of its own, it takes registers)
__global__ __launch_bounds__(NORM_MAX_THREADS) void norm_kernel(const norm_args a, int per_block) {
    __shared__ float lds[2][16];
    extern __shared__ float s_scales[];        // [cols / 128][NORM_ROWS]
    const int vecs = a.cols / 8, waves = blockDim.x >> 6, tid = threadIdx.x, lane = tid & 63;
    const int rest = REST ? a.cols & 7 : 0, last = vecs * 8 + tid;        // thread t < rest has column `last` as well
    const int64_t r0 = a.first + (int64_t)blockIdx.x * per_block;
    const int rows = (int)(a.rows - r0 < per_block ? a.rows - r0 : per_block);
    raw8<BF16, REST && NV < 4> x[NV], res[NV];
    float x1 = 0.f, res1 = 0.f;
    auto request = [&](int64_t r) {
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            const int i = tid + n * blockDim.x;
            if (i >= vecs) continue;
            x[n].load(row_of<BF16>(a.x, r * a.ld_x), (int64_t)i * 8);
            if (a.residual) res[n].load(row_of<BF16>(a.residual, r * a.ld_res), (int64_t)i * 8);
        }
        if (REST && tid < rest) {
            x1 = load1<BF16>(a.x, r * a.ld_x + last);
            if (a.residual) res1 = load1<BF16>(a.residual, r * a.ld_res + last);
        }
    };
    request(r0);
    for (int k = 0; k < rows; ++k) {
        const int64_t r = r0 + k;
        vec8 h[NV];
        float square = 0.f;
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            if (tid + n * (int)blockDim.x >= vecs) continue;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                h[n].v[j] = a.residual ? rounded<BF16>(x[n].at(j) + res[n].at(j)) : x[n].at(j);
                square = fmaf(h[n].v[j], h[n].v[j], square);
            }
        }
        const float h1 = REST && a.residual ? rounded<BF16>(x1 + res1) : x1;   // (zero for a thread without)
        if (REST) square = fmaf(h1, h1, square);
        if (k + 1 < rows) request(r + 1);
        square = wave_total(square);
        if (waves > 1) {
            if (lane == 0) lds[k & 1][tid >> 6] = square;
            __syncthreads();
            square = wave_total(lane < waves ? lds[k & 1][lane] : 0.f);
        }
        const float inv = 1.0f / sqrtf(square / (float)a.cols + a.eps);
        if (a.rstd && tid == 0) a.rstd[r] = inv;
        if (REST && tid < rest) {
            if (a.sum) store1<BF16>(a.sum, r * a.cols + last, h1);
            if (a.y) store1<BF16>(a.y, r * a.cols + last, h1 * inv * a.gain[last]);
        }
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            const int i = tid + n * blockDim.x;
            if (i >= vecs) continue;           // (with codes: whole groups of sixteen threads)
            if (a.sum) store8_any<BF16>(row_of<BF16>(a.sum, r * a.cols), (int64_t)i * 8, h[n]);
            if (!a.y && !a.q) continue;
            const vec8 g = load8_any(a.gain, (int64_t)i * 8);
            vec8 y;
#pragma unroll
            for (int j = 0; j < 8; ++j) y.v[j] = h[n].v[j] * inv * g.v[j];
            if (a.y) store8_any<BF16>(row_of<BF16>(a.y, r * a.cols), (int64_t)i * 8, y);
            if (a.q) {
                float amax = 0.f;              // (NaN stays NaN)
#pragma unroll
                for (int j = 0; j < 8; ++j) amax = __builtin_elementwise_maximum(amax, fabsf(y.v[j]));
#pragma unroll
                for (int o = 1; o < 16; o <<= 1) amax = __builtin_elementwise_maximum(amax, __shfl_xor(amax, o));
                const float scale = amax / 448.0f;
                const E4m3Coder coder(scale == 0.f ? 1.0f : scale, true);                      // (zero up to a maximum of 448 * 2^-150)
                u32x2 c;
                c[0] = coder.pack4<true>(y.v[0], y.v[1], y.v[2], y.v[3]);
                c[1] = coder.pack4<true>(y.v[4], y.v[5], y.v[6], y.v[7]);
                __builtin_nontemporal_store(c, reinterpret_cast<u32x2*>(a.q + r * a.cols + (int64_t)i * 8));
                if ((tid & 15) == 0) {
                    if (per_block == 1) a.scales[(int64_t)(i >> 4) * a.rows + r] = coder.s;
                    else s_scales[(i >> 4) * NORM_ROWS + k] = coder.s;
                }
            }
        }
    }
    if (a.q && per_block > 1) {
        __syncthreads();
        for (int i = tid; i < a.cols / QBLOCK * NORM_ROWS; i += blockDim.x)
            if (i % NORM_ROWS < rows) a.scales[(int64_t)(i / NORM_ROWS) * a.rows + r0 + i % NORM_ROWS] = s_scales[i];
    }
}

// Rows too wide for a block's registers: element by element, the row read twice.  No codes.  2000 x 65536 bf16 with residual and sum 747 us = 1.4 TB/s
// (2000 x 32768, in vectors: 114 us = 4.6 TB/s).
template <bool BF16>
__global__ __launch_bounds__(256) void norm_any_kernel(const norm_args a) {
    __shared__ float lds[4];
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const void* const x = row_of<BF16>(a.x, r * a.ld_x);
        const void* const res = a.residual ? row_of<BF16>(a.residual, r * a.ld_res) : nullptr;
        auto h_at = [&](int i) {
            const float v = load1<BF16>(x, i);
            return res ? rounded<BF16>(v + load1<BF16>(res, i)) : v;
        };
        float square = 0.f;
        for (int i = threadIdx.x; i < a.cols; i += 256) {
            const float h = h_at(i);
            square = fmaf(h, h, square);
        }
        const float inv = 1.0f / sqrtf(block_sum(square, lds, 4) / (float)a.cols + a.eps);
        if (a.rstd && threadIdx.x == 0) a.rstd[r] = inv;
        for (int i = threadIdx.x; i < a.cols; i += 256) {
            const float h = h_at(i);           // (before the sum is stored: it may take the place of x or the residual)
            if (a.sum) store1<BF16>(a.sum, r * a.cols + i, h);
            if (a.y) store1<BF16>(a.y, r * a.cols + i, h * inv * a.gain[i]);
        }
    }
}

struct norm_back_args {
    const void *dy, *h, *dh;
    const float *rstd, *gain;
    int64_t rows;
    int cols;
    void* dx;
    float* partial;                            // [gridDim.x][cols]: each block's part of dgain
};

// dx = u - h r^2 (u . h) / cols + dh with u = r gain dy; dgain = sum over rows of dy h r.
// Rows of block b: b, b + gridDim.x, ..., each requested while the one before is worked on; a thread keeps its columns' part of dgain in registers
// over all of them.  Bound by the bytes of dy, h, dh and dx, each once: 4096 x 5120 bf16 34.2 us = 4.9 TB/s, and 5.6 for the blocks' parts of dgain, which
// leave them as one row a block (a fixed order of the sums, no atomics).
template <bool BF16, int NV, int THREADS, bool REST>
__global__ __launch_bounds__(THREADS) void norm_back_kernel(const norm_back_args a) {
    __shared__ float lds[2][16];
    const int vecs = a.cols / 8, waves = blockDim.x >> 6, tid = threadIdx.x, lane = tid & 63;
    vec8 dg[NV];
#pragma unroll
    for (int n = 0; n < NV; ++n) dg[n] = vec8{};
    raw8<BF16> dy[NV], h[NV], dh[NV];
    const int rest = REST ? a.cols & 7 : 0, last = vecs * 8 + tid;        // thread t < rest has column `last` as well
    float dy1 = 0.f, h1 = 0.f, dh1 = 0.f, dg1 = 0.f;
    const float g1 = REST && tid < rest ? a.gain[last] : 0.f;
    auto request = [&](int64_t r) {
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            const int i = tid + n * blockDim.x;
            if (i >= vecs) continue;
            dy[n].load(a.dy, r * a.cols + (int64_t)i * 8);
            h[n].load(a.h, r * a.cols + (int64_t)i * 8);
            if (a.dh) dh[n].load(a.dh, r * a.cols + (int64_t)i * 8);
        }
        if (REST && tid < rest) {
            dy1 = load1<BF16>(a.dy, r * a.cols + last);
            h1 = load1<BF16>(a.h, r * a.cols + last);
            if (a.dh) dh1 = load1<BF16>(a.dh, r * a.cols + last);
        }
    };
    request(blockIdx.x);
    int turn = 0;
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x, turn ^= 1) {
        const int64_t row = r * a.cols;
        const float inv = a.rstd[r];
        vec8 d[NV], f[NV];                     // inv * gain * dy (+ dh), and h
        float dot = 0.f;
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            const int i = tid + n * blockDim.x;
            if (i >= vecs) continue;
            const vec8 g = load8_any(a.gain, (int64_t)i * 8);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                f[n].v[j] = h[n].at(j);
                const float u = dy[n].at(j) * inv;
                dg[n].v[j] = fmaf(u, f[n].v[j], dg[n].v[j]);
                const float t = u * g.v[j];
                dot = fmaf(t, f[n].v[j], dot);
                d[n].v[j] = a.dh ? t + dh[n].at(j) : t;
            }
        }
        const float f1 = h1, u1 = dy1 * inv;
        if (REST) {
            dg1 = fmaf(u1, f1, dg1);
            dot = fmaf(u1 * g1, f1, dot);
        }
        const float d1 = u1 * g1 + dh1;
        if (r + gridDim.x < a.rows) request(r + gridDim.x);
        dot = wave_total(dot);
        if (waves > 1) {
            if (lane == 0) lds[turn][tid >> 6] = dot;
            __syncthreads();
            dot = wave_total(lane < waves ? lds[turn][lane] : 0.f);
        }
        const float along = dot / (float)a.cols * inv * inv;
        if (REST && tid < rest) store1<BF16>(a.dx, row + last, fmaf(-along, f1, d1));
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            const int i = tid + n * blockDim.x;
            if (i >= vecs) continue;
#pragma unroll
            for (int j = 0; j < 8; ++j) d[n].v[j] = fmaf(-along, f[n].v[j], d[n].v[j]);
            store8_any<BF16>(a.dx, row + (int64_t)i * 8, d[n]);
        }
    }
#pragma unroll
    for (int n = 0; n < NV; ++n) {
        const int i = tid + n * blockDim.x;
        if (i >= vecs) continue;
        f32x4_any* const p = reinterpret_cast<f32x4_any*>(a.partial + (int64_t)blockIdx.x * a.cols + (int64_t)i * 8);
        p[0] = f32x4{dg[n].v[0], dg[n].v[1], dg[n].v[2], dg[n].v[3]};
        p[1] = f32x4{dg[n].v[4], dg[n].v[5], dg[n].v[6], dg[n].v[7]};
    }
    if (REST && tid < rest) a.partial[(int64_t)blockIdx.x * a.cols + last] = dg1;
}

// Rows too wide for a block's registers.  A thread's columns of dgain are added up in the block's row of `partial`, which it alone touches: a read and a write
// of memory for each element, 2000 x 65536 bf16 2930 us = 0.36 TB/s (2000 x 32768 in registers, one block of 1024 threads to a CU: 319).
template <bool BF16>
__global__ __launch_bounds__(256) void norm_back_any_kernel(const norm_back_args a) {
    __shared__ float lds[4];
    float* const part = a.partial + (int64_t)blockIdx.x * a.cols;
    for (int i = threadIdx.x; i < a.cols; i += 256) part[i] = 0.f;
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const int64_t row = r * a.cols;
        const float inv = a.rstd[r];
        float dot = 0.f;
        for (int i = threadIdx.x; i < a.cols; i += 256) {
            const float dy = load1<BF16>(a.dy, row + i), h = load1<BF16>(a.h, row + i);
            part[i] = fmaf(dy * inv, h, part[i]);
            dot = fmaf(dy * a.gain[i], h, dot);
        }
        const float f = block_sum(dot, lds, 4) / (float)a.cols * inv * inv * inv;
        for (int i = threadIdx.x; i < a.cols; i += 256) {
            float d = fmaf(-f, load1<BF16>(a.h, row + i), inv * (load1<BF16>(a.dy, row + i) * a.gain[i]));
            if (a.dh) d += load1<BF16>(a.dh, row + i);
            store1<BF16>(a.dx, row + i, d);
        }
    }
}

// dgain[c] = sum of the blocks' parts: 16 columns a block, 64 chains of parts joined at the end
__global__ __launch_bounds__(1024) void norm_gain_kernel(const float* __restrict__ partial, int parts, int cols, float* __restrict__ dgain) {
    __shared__ float lds[64][17];
    const int lc = threadIdx.x & 15, c = blockIdx.x * 16 + lc, chain = threadIdx.x >> 4;
    float s = 0.f;
    if (c < cols) {
#pragma unroll 4
        for (int p = chain; p < parts; p += 64) s += partial[(int64_t)p * cols + c];
    }
    lds[chain][lc] = s;
    __syncthreads();
    const int col = threadIdx.x >> 6, lane = threadIdx.x & 63;                 // a wave for each column
    s = wave_total(lds[lane][col]);
    if (lane == 0 && blockIdx.x * 16 + col < (unsigned)cols) dgain[blockIdx.x * 16 + col] = s;
}

// threads of a block that holds a row in vectors; 0: it does not fit
int row_threads(int cols, int& vectors) {
    const int vecs = cols < 8 ? 1 : cols / 8;
    vectors = vecs <= 256 ? 1 : vecs <= 2 * NORM_MAX_THREADS ? 2 : NORM_VECTORS;
    const int threads = ((vecs + vectors - 1) / vectors + 63) / 64 * 64;
    return threads <= NORM_MAX_THREADS ? threads : 0;
}

constexpr int64_t NORM_MAX_GRID = 1 << 20;

template <bool BF16>
hipError_t norm_forward(hipStream_t s, norm_args a) {
    int vectors;
    const int threads = row_threads(a.cols, vectors);
    if (!threads) {
        if (a.q) return hipErrorInvalidValue;  // (the entry point has refused it)
        norm_any_kernel<BF16><<<(unsigned)(a.rows < NORM_MAX_GRID ? a.rows : NORM_MAX_GRID), 256, 0, s>>>(a);
        return hipGetLastError();
    }
    const int per_block = norm_rows_per_block(a.rows, a.cols, threads, a.q != nullptr);
    const size_t lds = a.q && per_block > 1 ? (size_t)a.cols / QBLOCK * NORM_ROWS * sizeof(float) : 0;
    const bool rest = a.cols % 8 != 0;
    const auto kernel = vectors == 1   ? (rest ? norm_kernel<BF16, 1, true> : norm_kernel<BF16, 1, false>)
                        : vectors == 2 ? (rest ? norm_kernel<BF16, 2, true> : norm_kernel<BF16, 2, false>)
                                       : (rest ? norm_kernel<BF16, NORM_VECTORS, true> : norm_kernel<BF16, NORM_VECTORS, false>);
    for (int64_t blocks; a.first < a.rows; a.first += blocks * per_block) {
        blocks = norm_blocks(a.rows - a.first, threads, per_block);
        kernel<<<(unsigned)blocks, threads, lds, s>>>(a, per_block);
    }
    return hipGetLastError();
}

template <bool BF16>
hipError_t norm_backward(hipStream_t s, norm_back_args a, float* dgain) {
    int vectors;
    const int threads = row_threads(a.cols, vectors);
    // two blocks to a CU, more of narrow ones, all with about the same number of rows (4096 x 5120: 512 blocks of 8 rows 40 us, 716 of 5 or 6 48;
    // 8192 x 1024: 512 blocks 31 us, 1024 23.5, 1792 22)
    int blocks = threads > 192 || !threads ? 512 : threads > 128 ? 1024 : 1536;
    if (blocks > (int)(GRAD_WS_BYTES / sizeof(float) / a.cols)) blocks = (int)(GRAD_WS_BYTES / sizeof(float) / a.cols);
    const int64_t each = (a.rows + blocks - 1) / blocks;
    blocks = each ? (int)((a.rows + each - 1) / each) : 0;
    const bool rest = a.cols % 8 != 0;
    const auto kernel = !threads         ? norm_back_any_kernel<BF16>
                        : vectors == 1   ? (rest ? norm_back_kernel<BF16, 1, 512, true> : norm_back_kernel<BF16, 1, 512, false>)
                        : threads <= 512 ? (rest ? norm_back_kernel<BF16, 2, 512, true> : norm_back_kernel<BF16, 2, 512, false>)
                        : vectors == 2   ? (rest ? norm_back_kernel<BF16, 2, NORM_MAX_THREADS, true> : norm_back_kernel<BF16, 2, NORM_MAX_THREADS, false>)
                                         : (rest ? norm_back_kernel<BF16, NORM_VECTORS, NORM_MAX_THREADS, true>
                                                 : norm_back_kernel<BF16, NORM_VECTORS, NORM_MAX_THREADS, false>);
    if (blocks > 0) kernel<<<blocks, threads ? threads : 256, 0, s>>>(a);
    norm_gain_kernel<<<(a.cols + 15) / 16, 1024, 0, s>>>(a.partial, blocks, a.cols, dgain);
    return hipGetLastError();
}

}  // namespace

// a wide row's codes need the row in registers
bool norm_codes_fit(int32_t cols) {
    int vectors;
    return row_threads(cols, vectors) != 0;
}

hipError_t launch_norm(hipStream_t s, const void* x, const void* residual, const float* gain, int64_t rows, int32_t cols, int64_t ld_x,
                       int64_t ld_res, int32_t dtype, float eps, void* sum, void* y, uint8_t* q, float* scales, float* rstd) {
    const norm_args a{x, residual, gain, rows, 0, ld_x, residual ? ld_res : 0, cols, eps, sum, y, q, scales, rstd};
    return dtype == MOE_BF16 ? norm_forward<true>(s, a) : norm_forward<false>(s, a);
}

hipError_t launch_norm_backward(moe_ctx* c, const void* dy, const void* h, const float* rstd, const float* gain, const void* dh, int64_t rows,
                                int32_t cols, int32_t dtype, void* dx, float* dgain) {
    const norm_back_args a{dy, h, dh, rstd, gain, rows, cols, dx, static_cast<float*>(c->grad_ws)};
    return dtype == MOE_BF16 ? norm_backward<true>(c->stream, a, dgain) : norm_backward<false>(c->stream, a, dgain);
}

}  // namespace moe355
