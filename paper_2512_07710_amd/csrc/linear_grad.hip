// Gradients of the block-scaled FP8 linear, dense or grouped by expert: products of bf16 gradients with e4m3 codes on the bf16 matrix cores.
//
// Both have a matrix of codes [k][c] whose rows run along the sum:
//   dgrad   dx[p,c] = sum_n dy[p,n] * ws[n/128,c/128] Wq[n,c]     k = n: dy's rows run along the sum as well, the codes do not
//   wgrad   dW[n,c] = sum_p dy[p,n] * xs[c/128,p] xq[p,c]         k = p: neither does
// What does not run along the sum is transposed on its way from LDS to the registers by the transposing LDS reads.
#include "ffn_common.hpp"
#include "grad_common.hpp"

#include <type_traits>

namespace moe355 {
namespace {

template <int N>
using step = std::integral_constant<int, N>;

typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef short v8s __attribute__((ext_vector_type(8)));
typedef int v2i __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) v2i* lds_v2i_ptr;
typedef __attribute__((address_space(3))) v4s* lds_v4s_ptr;
typedef __attribute__((address_space(3))) const v8s* lds_v8s_ptr;
typedef __attribute__((address_space(3))) const v4f* lds_v4f_ptr;

constexpr int GM = 128, GN = 256;              // tile of the result: rows (along dy) and columns (along the codes)
constexpr int GK = 64;                         // steps of the sum that are staged at a time
constexpr int G_THREADS = 256;                 // four waves, each all 128 rows of the tile and 64 of its columns
constexpr int DY_STAGE = GM * GK * 2, CODE_STAGE = GN * GK, SCALE_STAGE = 4 * GK * 4, G_STAGE = DY_STAGE + CODE_STAGE + SCALE_STAGE;
constexpr int G_LDS = 2 * G_STAGE;             // two blocks to a CU

struct grad_args {
    const uint16_t* dy;
    const uint8_t* codes;                      // Wq or xq
    const float* scales;                       // ws or xs
    const int32_t* offsets;                    // or null: one expert with all rows
    int64_t rows;
    int E, NOUT, K;
    int accumulate;
    void* out;
};

// expert e's rows
__device__ inline void segment(const grad_args& a, int e, int& lo, int& hi) {
    if (!a.offsets) {
        lo = 0;
        hi = (int)a.rows;
        return;
    }
    lo = min(max(a.offsets[e], 0), (int)a.rows);
    hi = min(max(a.offsets[e + 1], lo), (int)a.rows);
}

// codes as bf16, times the power of two that `pow2` is
__device__ inline v8bf codes_bf16(v2i c, float pow2) {
    const v2bf a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[0], pow2, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[0], pow2, true);
    const v2bf d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[1], pow2, false), e = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[1], pow2, true);
    return v8bf{a[0], a[1], b[0], b[1], d[0], d[1], e[0], e[1]};
}

// what a wave reads from LDS for 16 steps of the sum, and its codes as operands
template <int PLANES>
struct operands {
    v8s d[4];                                  // dy: 4 x 32 rows of the tile
    v2i q[2];                                  // codes: 2 x 32 columns
    v4f s[2];                                  // (wgrad) the scales of a lane's eight steps
    v8bf c[2][PLANES];
};

// W: the weights' gradient; PLANES: bf16 planes of its scaled operand; F32: type of the result
template <bool W, int PLANES, bool F32>
__global__ __launch_bounds__(G_THREADS, 2) void grad_kernel(const grad_args a) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ int s_unit[4], s_waves[4];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int ctiles = (a.K + GN - 1) / GN;
    // ---- which tile
    int e, lo, hi, row0;                       // row0: first row of the result's tile
    const int c0 = (int)(blockIdx.x % ctiles) * GN;
    if (W) {
        const int ntiles = a.NOUT / GM, u = blockIdx.x / ctiles;
        e = u / ntiles;
        row0 = u % ntiles * GM;
        segment(a, e, lo, hi);
    } else if (!a.offsets) {
        e = 0;
        lo = 0;
        hi = (int)a.rows;
        row0 = (int)(blockIdx.x / ctiles) * GM;
    } else {                                   // the experts' row tiles in order: thread e counts those of expert e
        int l = 0, h = 0;
        if (tid < a.E) segment(a, tid, l, h);
        const int tiles = (h - l + GM - 1) / GM, upto = wave_scan(tiles);
        if (lane == 63) s_waves[wave] = upto;
        if (tid == 0) s_unit[0] = -1;
        __syncthreads();
        int first = upto - tiles;
        for (int w = 0; w < wave; ++w) first += s_waves[w];
        const int u = blockIdx.x / ctiles;
        if (u >= first && u < first + tiles) {
            s_unit[0] = tid;
            s_unit[1] = l;
            s_unit[2] = h;
            s_unit[3] = l + (u - first) * GM;
        }
        __syncthreads();
        e = s_unit[0];
        if (e < 0) return;
        lo = s_unit[1];
        hi = s_unit[2];
        row0 = s_unit[3];
    }
    e = __builtin_amdgcn_readfirstlane(e);
    lo = __builtin_amdgcn_readfirstlane(lo);
    hi = __builtin_amdgcn_readfirstlane(hi);
    row0 = __builtin_amdgcn_readfirstlane(row0);
    const int nk = W ? (hi - lo + GK - 1) / GK : a.NOUT / GK;
    const int cmask = a.K - c0 >= GN ? 15 : 7;                 // 16-byte chunks of codes in a row of the tile
    const size_t mat = (size_t)a.NOUT * a.K;
    const uint8_t* const codes = W ? a.codes + (size_t)lo * a.K + c0 : a.codes + (size_t)e * mat + c0;
    const uint16_t* const dy = W ? a.dy + (size_t)lo * a.NOUT + row0 : a.dy + (size_t)row0 * a.NOUT;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;

    // ---- copies of stage kb into its half of the ring; rows behind the segment repeat its last
    const int r4 = lane >> 4, r8 = lane >> 3;
    const uint32_t code_chunk = ((lane & 15) ^ ((r4 & 3) << 1)) & cmask, code_chunk4 = ((lane & 15) ^ ((r4 + 4) << 1)) & cmask;
    auto copy = [&](int kb) {
        const uint32_t at = lds0 + (uint32_t)(kb & 1) * G_STAGE;
        const int last = W ? hi - lo - 1 - kb * GK : GK - 1;
        if (W) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int row = wave * 16 + i * 4 + r4, chunk = (lane & 15) ^ (r4 << 2);
                dma16(at + (wave * 4 + i) * 1024, (uint32_t)min(row, last) * (uint32_t)(a.NOUT * 2) + chunk * 16, dy + (size_t)kb * GK * a.NOUT);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int row = wave * 32 + i * 8 + r8, chunk = (lane & 7) ^ r8 ^ (i & 1);
                dma16(at + (wave * 4 + i) * 1024, (uint32_t)min(row, hi - 1 - row0) * (uint32_t)(a.NOUT * 2) + chunk * 16, dy + kb * GK);
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = wave * 16 + i * 4 + r4;
            dma16(at + DY_STAGE + (wave * 4 + i) * 1024, (uint32_t)min(row, last) * (uint32_t)a.K + (i & 1 ? code_chunk4 : code_chunk) * 16,
                  codes + (size_t)kb * GK * a.K);
        }
        if (W) {                               // wave w brings the scales of 128-column block w&1 of the tile (those of waves 0 and 1 are read)
            const int cb = min(c0 / QBLOCK + (wave & 1), a.K / QBLOCK - 1);
            dma4(at + DY_STAGE + CODE_STAGE + wave * 256, (uint32_t)min(lane, last) * 4, a.scales + (size_t)cb * a.rows + lo + kb * GK);
        }
    };
    constexpr int COPIES = W ? 9 : 8;
    // (wgrad) what repeats the last row is no part of the sum: zeros in its place
    auto clear_behind = [&](int kb) {
        const int left = hi - lo - kb * GK;
        if (left >= GK) return;
        char* const at = lds + (kb & 1) * G_STAGE;
        const u32x4 zero = {0u, 0u, 0u, 0u};
        for (int i = left * 16 + tid; i < GK * 16; i += G_THREADS) {
            *reinterpret_cast<u32x4*>(at + i * 16) = zero;
            *reinterpret_cast<u32x4*>(at + DY_STAGE + i * 16) = zero;
        }
        if (lane >= left) *reinterpret_cast<float*>(at + DY_STAGE + CODE_STAGE + tid * 4) = 0.f;
        __syncthreads();
    };

    // ---- this wave's part: 128 rows x 64 columns of the tile
    const int cols0 = c0 + wave * 64;
    const bool mine = cols0 < a.K;
    uint32_t dy_at[4], code_at[2];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (W) {
            const int chunk = (i * 4 + (lane >> 4 & 1) * 2 + (lane >> 1 & 1)) ^ ((lane >> 2 & 3) << 2);
            dy_at[i] = lds0 + ((lane >> 5) * 8 + (lane >> 2 & 3)) * 256 + chunk * 16 + (lane & 1) * 8;
        } else {                               // i: sixteen steps of the sum
            const int row = lane & 31;
            dy_at[i] = lds0 + row * 128 + (((i * 2 + (lane >> 5)) ^ (row & 7) ^ (row >> 3 & 1)) << 4);
        }
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int chunk = (wave * 4 + j * 2 + (lane >> 4 & 1)) ^ ((lane >> 1 & 7) << 1);
        code_at[j] = lds0 + DY_STAGE + ((lane >> 5) * 8 + (lane >> 1 & 7)) * 256 + chunk * 16 + (lane & 1) * 8;
    }
    const uint32_t scale_at = lds0 + DY_STAGE + CODE_STAGE + (wave >> 1) * 256 + (lane >> 5) * 32;
    auto fetch = [&](operands<PLANES>& o, uint32_t at, auto kk_) {     // at: the stage's offset
        constexpr int kk = decltype(kk_)::value;
#pragma unroll
        for (int j = 0; j < 2; ++j) o.q[j] = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_v2i_ptr)(uintptr_t)(code_at[j] + at + kk * 4096));
        if (W) {
            o.s[0] = *(lds_v4f_ptr)(uintptr_t)(scale_at + at + kk * 64);
            o.s[1] = *(lds_v4f_ptr)(uintptr_t)(scale_at + at + kk * 64 + 16);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (W) {
                const v4s p = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s_ptr)(uintptr_t)(dy_at[i] + at + kk * 4096));
                const v4s q = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s_ptr)(uintptr_t)(dy_at[i] + at + kk * 4096 + 1024));
                o.d[i] = __builtin_shufflevector(p, q, 0, 1, 2, 3, 4, 5, 6, 7);
            } else {
                o.d[i] = *(lds_v8s_ptr)(uintptr_t)(dy_at[kk] + at + i * 4096);
            }
        }
    };

    v16f acc[4][2];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;
    // (dgrad) acc is held in units of the present block's scale without its power of two, which the codes carry: a factor of less than
    // two either way from block to block, whatever the scales are.  (In the constant address space, so that they come as scalar loads:
    // a vector load's wait would include the copies)
    const __attribute__((address_space(4))) float* const block_scales = (const __attribute__((address_space(4))) float*)(uintptr_t)(
        a.scales + (size_t)e * (a.NOUT / QBLOCK) * (a.K / QBLOCK) + min(cols0, a.K - 1) / QBLOCK);
    float unit = 1.f, pow2 = 1.f;
    int block_mask = -1;
    auto next_block = [&](int kb) {            // the factor on acc
        const float s = block_scales[(size_t)(kb / 2) * (a.K / QBLOCK)];
        const uint32_t exponent = __float_as_uint(s) & 0x7F800000u;
        const bool live = exponent != 0, finite = exponent != 0x7F800000u;
        block_mask = live ? -1 : 0;            // a zero scale (or one below the normal range): the block adds nothing
        const float to = !live ? unit : finite ? __uint_as_float((__float_as_uint(s) & 0x807FFFFFu) | 0x3F800000u) : s;
        pow2 = live && finite ? __uint_as_float(exponent) : 1.f;
        const float ratio = unit / to;
        unit = to;
        return ratio;
    };
    auto convert = [&](operands<PLANES>& o) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            if (!W) {
                o.c[j][0] = codes_bf16(o.q[j] & block_mask, pow2);
                continue;
            }
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                const v2f x = h & 1 ? __builtin_amdgcn_cvt_pk_f32_fp8(o.q[j][h >> 1], true) : __builtin_amdgcn_cvt_pk_f32_fp8(o.q[j][h >> 1], false);
#pragma unroll
                for (int v = 0; v < 2; ++v) {
                    float y = x[v] * o.s[h >> 1][(h & 1) * 2 + v];
#pragma unroll
                    for (int p = 0; p < PLANES; ++p) {
                        o.c[j][p][h * 2 + v] = (__bf16)y;
                        if (p + 1 < PLANES) {
                            y -= (float)o.c[j][p][h * 2 + v];
                            if (y != y) y = 0.f;               // (the first plane has the infinity)
                        }
                    }
                }
            }
        }
    };
    auto product = [&](const operands<PLANES>& o, int i, int p) {
#pragma unroll
        for (int j = 0; j < 2; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(o.c[j][p], __builtin_bit_cast(v8bf, o.d[i]), acc[i][j], 0, 0, 0);
    };
    // The products of `o`, while the operands of the next group (if there is one) come from LDS behind the first of them and are converted
    // behind the others: in this order, which the compiler would not keep by itself
    auto group = [&](operands<PLANES>& o, operands<PLANES>* next, auto rescale_, float ratio) {
        constexpr bool rescale = decltype(rescale_)::value;
        if (rescale) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                acc[i][0] *= ratio;
                acc[i][1] *= ratio;
                product(o, i, 0);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) product(o, i, 0);
        }
        if (PLANES > 1) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {      // an infinite gradient counts in the first plane, the others have both signs and zeros
#pragma unroll
                for (int v = 0; v < 8; ++v) o.d[i][v] = (o.d[i][v] & 0x7F80) == 0x7F80 ? (short)0 : o.d[i][v];
            }
#pragma unroll
            for (int p = 1; p < PLANES; ++p)
#pragma unroll
                for (int i = 0; i < 4; ++i) product(o, i, p);
        }
        if (next) convert(*next);
        if (PLANES == 1) {
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                __builtin_amdgcn_sched_group_barrier(0x100, W ? 3 : 2, 0);     // LDS reads
                if (rescale) __builtin_amdgcn_sched_group_barrier(0x2, 16, 0);
                __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);               // a product
            }
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                __builtin_amdgcn_sched_group_barrier(0x2, rescale ? 18 : W ? 8 : 2, 0);
                __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    };

    // ---- the sum.  Operands are fetched one group of products ahead; the barrier that hands over the stages stands before a stage's last group,
    // so that the first operands of the next come during its products
    if (nk > 0) {
        copy(0);
        if (nk > 1) {
            copy(1);
            asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(COPIES) : "memory");
        } else {
            asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
        }
        if (W) clear_behind(0);
        operands<PLANES> f, g;
        fetch(f, 0, step<0>{});
        auto stage = [&](int kb, auto first_) {
            constexpr bool first = decltype(first_)::value;    // (dgrad) of a block of scales
            const uint32_t at = (uint32_t)(kb & 1) * G_STAGE;
            const float ratio = first ? next_block(kb) : 1.f;
            if (!W && first) convert(f);
            fetch(g, at, step<1>{});
            group(f, &g, first_, ratio);
            fetch(f, at, step<2>{});
            group(g, &f, std::false_type{}, 1.f);
            fetch(g, at, step<3>{});
            group(f, &g, std::false_type{}, 1.f);
            if (kb + 1 < nk) {
                asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");   // stage kb+1 is there, and this one has been read
                if (kb + 2 < nk) copy(kb + 2);
                if (W) clear_behind(kb + 1);
            }
            fetch(f, G_STAGE - at, step<0>{});                 // (behind the last stage: of no use, and not used)
            group(g, W || first ? &f : nullptr, std::false_type{}, 1.f);
        };
        if (W) {
            convert(f);
            for (int kb = 0; kb < nk; ++kb) stage(kb, std::false_type{});
        } else {
            for (int kb = 0; kb < nk; kb += 2) {               // two stages to a block of scales
                stage(kb, std::true_type{});
                stage(kb + 1, std::false_type{});
            }
        }
    }

    // ---- a lane holds one row of the result, four neighbouring columns at a time
    if (!mine) return;
    const int end = W ? a.NOUT : hi;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = row0 + i * 32 + (lane & 31);
        if (row >= end) continue;
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const size_t o = (W ? (size_t)e * mat : 0) + (size_t)row * a.K + cols0 + j * 32 + g * 8 + (lane >> 5) * 4;
                f32x4 r = {acc[i][j][g * 4], acc[i][j][g * 4 + 1], acc[i][j][g * 4 + 2], acc[i][j][g * 4 + 3]};
                if (!W) r *= unit;
                if (F32) {
                    f32x4* const p = reinterpret_cast<f32x4*>(static_cast<float*>(a.out) + o);
                    if (a.accumulate) r += *p;
                    *p = r;
                } else {
                    u32x2* const p = reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.out) + o);
                    if (a.accumulate) {
                        const u32x2 was = *p;
                        r += f32x4{bf16lo(was[0]), bf16hi(was[0]), bf16lo(was[1]), bf16hi(was[1])};
                    }
                    *p = u32x2{bf16_bits(r[0]) | bf16_bits(r[1]) << 16, bf16_bits(r[2]) | bf16_bits(r[3]) << 16};
                }
            }
    }
}

}  // namespace

hipError_t set_grad_lds_limits() {
    for (const void* f : {(const void*)grad_kernel<false, 1, false>, (const void*)grad_kernel<true, 1, false>, (const void*)grad_kernel<true, 3, true>})
        if (const hipError_t e = hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, G_LDS); e != hipSuccess) return e;
    return hipSuccess;
}

hipError_t launch_linear_dgrad(moe_ctx* c, const uint16_t* dy, int64_t rows, int32_t NOUT, const uint8_t* Wq, const float* ws, int32_t K,
                               const int32_t* offsets, int32_t E, uint16_t* dx) {
    const grad_args a{dy, Wq, ws, offsets, rows, E, NOUT, K, 0, dx};
    const int64_t tiles = offsets ? rows / GM + E : (rows + GM - 1) / GM;
    grad_kernel<false, 1, false><<<(unsigned)(tiles * ((K + GN - 1) / GN)), G_THREADS, G_LDS, c->stream>>>(a);
    return hipGetLastError();
}

hipError_t launch_linear_wgrad(moe_ctx* c, const uint16_t* dy, int64_t rows, int32_t NOUT, const uint8_t* xq, const float* xs, int32_t K,
                               const int32_t* offsets, int32_t E, int32_t accumulate, int32_t dtype, void* dW) {
    const grad_args a{dy, xq, xs, offsets, rows, E, NOUT, K, accumulate, dW};
    const unsigned grid = (unsigned)((int64_t)E * (NOUT / GM) * ((K + GN - 1) / GN));
    if (dtype == MOE_BF16) grad_kernel<true, 1, false><<<grid, G_THREADS, G_LDS, c->stream>>>(a);
    else grad_kernel<true, 3, true><<<grid, G_THREADS, G_LDS, c->stream>>>(a);
    return hipGetLastError();
}

}  // namespace moe355
