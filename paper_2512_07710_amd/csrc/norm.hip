// Residual addition, root-mean-square norm and e4m3 coding in one pass over a row, and the norm's gradient.
#include "grad_common.hpp"

namespace moe355 {
namespace {

constexpr int NORM_MAX_THREADS = 1024;
constexpr int NORM_VECTORS = 4;                // vectors of eight elements that a thread holds at most

struct norm_args {
    const void *x, *residual;
    const float* gain;
    int64_t rows, ld_x, ld_res;
    int cols;
    float eps;
    void *sum, *y;
    uint8_t* q;
    float *scales, *rstd;
};

// One block per row, the row in registers.  VEC: rows of whole aligned vectors, thread t of TPR holds vectors t, t+TPR, ...; sixteen
// neighbouring threads hold a group of 128 columns.  Otherwise single elements, read again for the output.
template <bool BF16, int NV>
__global__ __launch_bounds__(NORM_MAX_THREADS) void norm_kernel(const norm_args a) {
    __shared__ float lds[16];
    const int vecs = a.cols / 8, waves = blockDim.x >> 6;
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const void* const x = row_of<BF16>(a.x, r * a.ld_x);
        const void* const res = a.residual ? row_of<BF16>(a.residual, r * a.ld_res) : nullptr;
        vec8 h[NV];
        float square = 0.f;
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            const int i = threadIdx.x + n * blockDim.x;
            if (i >= vecs) {
                h[n] = vec8{};
                continue;
            }
            h[n] = load8<BF16>(x, (int64_t)i * 8);
            if (res) {
                const vec8 v = load8<BF16>(res, (int64_t)i * 8);
#pragma unroll
                for (int j = 0; j < 8; ++j) h[n].v[j] = rounded<BF16>(h[n].v[j] + v.v[j]);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) square = fmaf(h[n].v[j], h[n].v[j], square);
        }
        const float inv = 1.0f / sqrtf(block_sum(square, lds, waves) / (float)a.cols + a.eps);
        if (a.rstd && threadIdx.x == 0) a.rstd[r] = inv;
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            const int i = threadIdx.x + n * blockDim.x;
            if (i >= vecs) continue;           // (whole groups of sixteen threads)
            if (a.sum) store8<BF16>(row_of<BF16>(a.sum, r * a.cols), (int64_t)i * 8, h[n]);
            const vec8 g = load8<false>(a.gain, (int64_t)i * 8);
            vec8 y;
#pragma unroll
            for (int j = 0; j < 8; ++j) y.v[j] = h[n].v[j] * inv * g.v[j];
            if (a.y) store8<BF16>(row_of<BF16>(a.y, r * a.cols), (int64_t)i * 8, y);
            if (a.q) {
                float amax = 0.f;
#pragma unroll
                for (int j = 0; j < 8; ++j) amax = fmaxf(amax, fabsf(y.v[j]));
#pragma unroll
                for (int o = 1; o < 16; o <<= 1) amax = fmaxf(amax, __shfl_xor(amax, o));
                const E4m3Coder coder(amax == 0.f ? 1.0f : amax / 448.0f);
                u32x2 c;
                c[0] = coder.pack4(y.v[0], y.v[1], y.v[2], y.v[3]);
                c[1] = coder.pack4(y.v[4], y.v[5], y.v[6], y.v[7]);
                *reinterpret_cast<u32x2*>(a.q + r * a.cols + (int64_t)i * 8) = c;
                if ((threadIdx.x & 15) == 0) a.scales[(int64_t)(i >> 4) * a.rows + r] = coder.s;
            }
        }
    }
}

// Any width, stride and alignment: element by element, the row read twice.  No codes.
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

// Rows of block b: b, b + gridDim.x, ...; a thread keeps its columns' part of dgain in registers over all of them.
template <bool BF16, int NV>
__global__ __launch_bounds__(NORM_MAX_THREADS) void norm_back_kernel(const norm_back_args a) {
    __shared__ float lds[16];
    const int vecs = a.cols / 8, waves = blockDim.x >> 6;
    vec8 dg[NV];
#pragma unroll
    for (int n = 0; n < NV; ++n) dg[n] = vec8{};
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const int64_t row = r * a.cols;
        const float inv = a.rstd[r];
        vec8 u[NV], h[NV];
        float dot = 0.f;
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            const int i = threadIdx.x + n * blockDim.x;
            if (i >= vecs) {
                u[n] = h[n] = vec8{};
                continue;
            }
            u[n] = load8<BF16>(a.dy, row + (int64_t)i * 8);
            h[n] = load8<BF16>(a.h, row + (int64_t)i * 8);
            const vec8 g = load8<false>(a.gain, (int64_t)i * 8);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                dg[n].v[j] = fmaf(u[n].v[j] * inv, h[n].v[j], dg[n].v[j]);
                u[n].v[j] *= g.v[j];
                dot = fmaf(u[n].v[j], h[n].v[j], dot);
            }
        }
        const float f = block_sum(dot, lds, waves) / (float)a.cols * inv * inv * inv;
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            const int i = threadIdx.x + n * blockDim.x;
            if (i >= vecs) continue;
            vec8 d;
#pragma unroll
            for (int j = 0; j < 8; ++j) d.v[j] = fmaf(-f, h[n].v[j], inv * u[n].v[j]);
            if (a.dh) {
                const vec8 e = load8<BF16>(a.dh, row + (int64_t)i * 8);
#pragma unroll
                for (int j = 0; j < 8; ++j) d.v[j] += e.v[j];
            }
            store8<BF16>(a.dx, row + (int64_t)i * 8, d);
        }
    }
#pragma unroll
    for (int n = 0; n < NV; ++n) {
        const int i = threadIdx.x + n * blockDim.x;
        if (i < vecs) store8<false>(a.partial, (int64_t)blockIdx.x * a.cols + (int64_t)i * 8, dg[n]);
    }
}

// Any width and alignment.  A thread's columns of dgain are added up in the block's row of `partial`, which it alone touches.
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

// dgain[c] = sum of the blocks' parts: 32 columns a block, eight chains of rows joined at the end
__global__ __launch_bounds__(256) void norm_gain_kernel(const float* __restrict__ partial, int parts, int cols, float* __restrict__ dgain) {
    __shared__ float lds[8][32];
    const int c = blockIdx.x * 32 + (threadIdx.x & 31), chain = threadIdx.x >> 5;
    float s = 0.f;
    if (c < cols)
        for (int p = chain; p < parts; p += 8) s += partial[(int64_t)p * cols + c];
    lds[chain][threadIdx.x & 31] = s;
    __syncthreads();
    if (chain == 0 && c < cols) {
        for (int w = 1; w < 8; ++w) s += lds[w][threadIdx.x];
        dgain[c] = s;
    }
}

// threads of a block that holds a row in vectors; 0: it does not fit
int row_threads(int cols, int& vectors) {
    const int vecs = cols / 8;
    vectors = vecs <= 256 ? 1 : vecs <= 1024 ? 2 : NORM_VECTORS;
    const int threads = ((vecs + vectors - 1) / vectors + 63) / 64 * 64;
    return threads <= NORM_MAX_THREADS ? threads : 0;
}

constexpr int64_t NORM_MAX_GRID = 1 << 20;

template <bool BF16>
hipError_t norm_forward(hipStream_t s, const norm_args& a) {
    int vectors;
    const int threads = row_threads(a.cols, vectors), eight = BF16 ? 8 : 4;
    const unsigned grid = (unsigned)(a.rows < NORM_MAX_GRID ? a.rows : NORM_MAX_GRID);
    const bool whole = threads && a.cols % 8 == 0 && a.ld_x % eight == 0 && a.ld_res % eight == 0 && aligned16(a.x) && aligned16(a.residual) &&
                       aligned16(a.gain) && aligned16(a.sum) && aligned16(a.y) && ((uintptr_t)a.q & 7) == 0;
    if (!whole) {
        if (a.q) return hipErrorInvalidValue;  // (the entry point has refused it)
        norm_any_kernel<BF16><<<grid, 256, 0, s>>>(a);
    } else if (vectors == 1) {
        norm_kernel<BF16, 1><<<grid, threads, 0, s>>>(a);
    } else if (vectors == 2) {
        norm_kernel<BF16, 2><<<grid, threads, 0, s>>>(a);
    } else {
        norm_kernel<BF16, NORM_VECTORS><<<grid, threads, 0, s>>>(a);
    }
    return hipGetLastError();
}

constexpr int NORM_BACK_BLOCKS = 512;           // at most, and as many as the workspace has rows for

template <bool BF16>
hipError_t norm_backward(hipStream_t s, norm_back_args a, float* dgain) {
    int vectors;
    const int threads = row_threads(a.cols, vectors);
    int blocks = (int)(GRAD_WS_BYTES / sizeof(float) / a.cols);
    if (blocks > NORM_BACK_BLOCKS) blocks = NORM_BACK_BLOCKS;
    if (blocks > a.rows) blocks = (int)a.rows;
    const bool whole = threads && a.cols % 8 == 0 && aligned16(a.dy) && aligned16(a.h) && aligned16(a.dh) && aligned16(a.gain) && aligned16(a.dx);
    if (blocks == 0) {
    } else if (!whole) {
        norm_back_any_kernel<BF16><<<blocks, 256, 0, s>>>(a);
    } else if (vectors == 1) {
        norm_back_kernel<BF16, 1><<<blocks, threads, 0, s>>>(a);
    } else if (vectors == 2) {
        norm_back_kernel<BF16, 2><<<blocks, threads, 0, s>>>(a);
    } else {
        norm_back_kernel<BF16, NORM_VECTORS><<<blocks, threads, 0, s>>>(a);
    }
    norm_gain_kernel<<<(a.cols + 31) / 32, 256, 0, s>>>(a.partial, blocks, a.cols, dgain);
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
    const norm_args a{x, residual, gain, rows, ld_x, residual ? ld_res : 0, cols, eps, sum, y, q, scales, rstd};
    return dtype == MOE_BF16 ? norm_forward<true>(s, a) : norm_forward<false>(s, a);
}

hipError_t launch_norm_backward(moe_ctx* c, const void* dy, const void* h, const float* rstd, const float* gain, const void* dh, int64_t rows,
                                int32_t cols, int32_t dtype, void* dx, float* dgain) {
    const norm_back_args a{dy, h, dh, rstd, gain, rows, cols, dx, static_cast<float*>(c->grad_ws)};
    return dtype == MOE_BF16 ? norm_backward<true>(c->stream, a, dgain) : norm_backward<false>(c->stream, a, dgain);
}

}  // namespace moe355
