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
constexpr int G_MIN_PART = 4;                  // stages of a part of a sum at least

struct grad_args {
    const uint16_t* dy;
    const uint8_t* codes;                      // Wq or xq
    const float* scales;                       // ws or xs
    const int32_t* offsets;                    // or null: one expert with all rows
    int64_t rows;
    int E, NOUT, K;
    int accumulate;
    void* out;
    float* parts;                              // [units][4][8][256] f32x4: a thread's sums, in its own order
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

// Tiles are dealt to the XCDs (blockIdx % 8) in runs, and run through a band of eight tile rows column by column, so that the 64 tiles that an XCD
// works on at a time share their operands in its L2.  Tiles that do not fill a round of the chip are cut along the sum: parts
// go to the workspace and a second launch adds them up.
constexpr int G_SLOTS = 512, G_BAND = 8;       // blocks that run at a time
struct split_plan {
    int whole, cut, parts;                     // tiles done at once; tiles in parts, and how many parts
};
__host__ __device__ inline split_plan plan_of(int tiles, int stages) {
    split_plan p{tiles, 0, 1};
    const int rest = tiles % G_SLOTS;
    if (rest == 0) return p;
    int parts = G_SLOTS / rest;
    if (parts > stages / G_MIN_PART) parts = stages / G_MIN_PART;
    if (parts < (tiles < G_SLOTS ? 2 : 3)) return p;
    // (in stages) what is saved against what the parts' way through memory costs
    if (tiles >= G_SLOTS && stages * (0.55f - 1.0f / parts) < 24.f) return p;
    return split_plan{tiles - rest, rest, parts};
}

struct find_scratch {
    int waves[G_THREADS / 64], found[4];
};
struct unit {
    int e, lo, hi;                             // expert and its rows
    int row0, c0;                              // first row and column of the tile
    int part, parts, slot;                     // part of the sum; its place in the workspace
};
// The unit of block b; JOIN: of the launch that adds up, four blocks to a tile.  False: none.  Called by the whole block.
template <bool W, bool JOIN = false>
__device__ inline bool unit_of(const grad_args& a, int b, find_scratch& s, unit& u) {
    const int ctiles = (a.K + GN - 1) / GN, tid = threadIdx.x;
    int row_tiles = W ? a.E * (a.NOUT / GM) : (int)((a.rows + GM - 1) / GM);
    int first = 0, tiles = 0, l = 0, h = 0;    // (grouped dgrad) thread e: expert e's row tiles
    const bool search = !W && a.offsets;
    if (search) {
        if (tid < a.E) segment(a, tid, l, h);
        tiles = (h - l + GM - 1) / GM;
        const int upto = wave_scan(tiles);
        if ((tid & 63) == 63) s.waves[tid >> 6] = upto;
        __syncthreads();
        first = upto - tiles;
        row_tiles = 0;
        for (int w = 0; w < G_THREADS / 64; ++w) {
            if (w < tid >> 6) first += s.waves[w];
            row_tiles += s.waves[w];
        }
    }
    const int total = row_tiles * ctiles;
    const split_plan p = W && a.offsets ? split_plan{total, 0, 1} : plan_of(total, W ? (int)((a.rows + GK - 1) / GK) : a.NOUT / GK);
    int t;
    u.part = 0;
    u.parts = 1;
    u.slot = 0;
    if (JOIN) {
        if (b >= p.cut) return false;
        t = p.whole + b;
        u.parts = p.parts;
        u.slot = b * p.parts;
    } else {
        const int units = p.whole + p.cut * p.parts, x = b & 7, at = b >> 3;
        int n;
        if (W && a.offsets) {                  // experts' sums have different lengths: runs of 64 tiles, taken in turns
            n = (at / 64 * 8 + x) * 64 + at % 64;
            if (n >= units) return false;
        } else if (p.whole > 0) {              // whole tiles in eight runs, then the parts
            const int from = (int)((int64_t)p.whole * x / 8), count = (int)((int64_t)p.whole * (x + 1) / 8) - from;
            const int pfrom = (int)((int64_t)(units - p.whole) * x / 8), pcount = (int)((int64_t)(units - p.whole) * (x + 1) / 8) - pfrom;
            if (at >= count + pcount) return false;
            n = at < count ? from + at : p.whole + pfrom + (at - count);
        } else {
            const int from = (int)((int64_t)units * x / 8), count = (int)((int64_t)units * (x + 1) / 8) - from;
            if (at >= count) return false;
            n = from + at;
        }
        t = n;
        if (n >= p.whole) {
            u.slot = n - p.whole;
            t = p.whole + u.slot / p.parts;
            u.part = u.slot % p.parts;
            u.parts = p.parts;
        }
    }
    const int band = t / (G_BAND * ctiles), in_band = t - band * G_BAND * ctiles, height = min(G_BAND, row_tiles - band * G_BAND);
    const int row_tile = band * G_BAND + in_band % height;
    u.c0 = in_band / height * GN;
    if (W) {
        u.e = row_tile / (a.NOUT / GM);
        u.row0 = row_tile % (a.NOUT / GM) * GM;
        segment(a, u.e, u.lo, u.hi);
    } else if (!search) {
        u.e = 0;
        u.lo = 0;
        u.hi = (int)a.rows;
        u.row0 = row_tile * GM;
    } else {
        if (row_tile >= first && row_tile < first + tiles) {
            s.found[0] = tid;
            s.found[1] = l;
            s.found[2] = h;
            s.found[3] = l + (row_tile - first) * GM;
        }
        __syncthreads();
        u.e = s.found[0];
        u.lo = s.found[1];
        u.hi = s.found[2];
        u.row0 = s.found[3];
    }
    // (the same for the whole block: scalars)
    u.e = __builtin_amdgcn_readfirstlane(u.e);
    u.lo = __builtin_amdgcn_readfirstlane(u.lo);
    u.hi = __builtin_amdgcn_readfirstlane(u.hi);
    u.row0 = __builtin_amdgcn_readfirstlane(u.row0);
    return true;
}

// A wave's 32 x 64 values of the result, a lane's four neighbouring columns of row lane%32 at a time, go through LDS to be stored as whole
// lines.  buffer: the wave's own place.
constexpr int OUT_LD = 68;                     // floats of a row there
template <bool F32>
__device__ inline void store_rows(const grad_args& a, float* buffer, const f32x4 (&r)[2][4], size_t at, int rows) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            *reinterpret_cast<f32x4*>(buffer + (lane & 31) * OUT_LD + j * 32 + g * 8 + (lane >> 5) * 4) = r[j][g];
    __builtin_amdgcn_wave_barrier();
    constexpr int PER_ROW = F32 ? 16 : 8, STEP = 64 / PER_ROW, N = 64 / PER_ROW;               // lanes of a row, rows at a time, a lane's columns
#pragma unroll
    for (int i = 0; i < 32; i += STEP) {
        const int row = i + lane / PER_ROW, c = lane % PER_ROW * N;
        if (row >= rows) continue;
        float v[N];
#pragma unroll
        for (int n = 0; n < N; n += 4) *reinterpret_cast<f32x4*>(v + n) = *reinterpret_cast<const f32x4*>(buffer + row * OUT_LD + c + n);
        const size_t o = at + (size_t)row * a.K + c;
        if (F32) {
            f32x4* const p = reinterpret_cast<f32x4*>(static_cast<float*>(a.out) + o);
            f32x4 w = {v[0], v[1], v[2], v[3]};
            if (a.accumulate) w += *p;
            *p = w;
        } else {
            uint16_t* const p = static_cast<uint16_t*>(a.out) + o;
            vec8 w;
#pragma unroll
            for (int n = 0; n < 8; ++n) w.v[n] = v[n % N];
            if (a.accumulate) {
                const vec8 was = load8<true>(p, 0);
#pragma unroll
                for (int n = 0; n < 8; ++n) w.v[n] += was.v[n];
            }
            store8<true>(p, 0, w);
        }
    }
    __builtin_amdgcn_wave_barrier();
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
    __shared__ find_scratch s_find;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    unit u;
    if (!unit_of<W>(a, blockIdx.x, s_find, u)) return;
    const int e = u.e, lo = u.lo, hi = u.hi, row0 = u.row0, c0 = u.c0;
    // this block's stages of the sum: all, or a part
    const int all_stages = W ? (hi - lo + GK - 1) / GK : a.NOUT / GK, pair = W ? 1 : 2;        // (dgrad: two to a block of scales)
    const int k0 = all_stages / pair * u.part / u.parts * pair, nk = all_stages / pair * (u.part + 1) / u.parts * pair;
    const int cmask = a.K - c0 >= GN ? 15 : 7;                 // 16-byte chunks of codes in a row of the tile
    const size_t mat = (size_t)a.NOUT * a.K;
    const uint8_t* const codes = W ? a.codes + (size_t)lo * a.K + c0 : a.codes + (size_t)e * mat + c0;
    const uint16_t* const dy = W ? a.dy + (size_t)lo * a.NOUT + row0 : a.dy + (size_t)row0 * a.NOUT;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;

    // ---- copies of stage kb into its half of the ring; rows behind the segment repeat its last
    const int r4 = lane >> 4, r8 = lane >> 3;
    const uint32_t code_chunk = ((lane & 15) ^ ((r4 & 3) << 1)) & cmask, code_chunk4 = ((lane & 15) ^ ((r4 + 4) << 1)) & cmask;
    auto copy = [&](int kb) {
        const uint32_t at = lds0 + (uint32_t)((kb - k0) & 1) * G_STAGE;
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
        char* const at = lds + ((kb - k0) & 1) * G_STAGE;
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
    float unit_scale = 1.f, pow2 = 1.f;
    int block_mask = -1;
    auto next_block = [&](int kb) {            // the factor on acc
        const float s = block_scales[(size_t)(kb / 2) * (a.K / QBLOCK)];
        const uint32_t exponent = __float_as_uint(s) & 0x7F800000u;
        const bool live = exponent != 0, finite = exponent != 0x7F800000u;
        block_mask = live ? -1 : 0;            // a zero scale (or one below the normal range): the block adds nothing
        const float to = !live ? unit_scale : finite ? __uint_as_float((__float_as_uint(s) & 0x807FFFFFu) | 0x3F800000u) : s;
        pow2 = live && finite ? __uint_as_float(exponent) : 1.f;
        const float ratio = unit_scale / to;
        unit_scale = to;
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
    if (nk > k0) {
        copy(k0);
        if (nk > k0 + 1) {
            copy(k0 + 1);
            asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(COPIES) : "memory");
        } else {
            asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
        }
        if (W) clear_behind(k0);
        operands<PLANES> f, g;
        fetch(f, 0, step<0>{});
        auto stage = [&](int kb, auto first_) {
            constexpr bool first = decltype(first_)::value;    // (dgrad) of a block of scales
            const uint32_t at = (uint32_t)((kb - k0) & 1) * G_STAGE;
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
            for (int kb = k0; kb < nk; ++kb) stage(kb, std::false_type{});
        } else {
            for (int kb = k0; kb < nk; kb += 2) {              // two stages to a block of scales
                stage(kb, std::true_type{});
                stage(kb + 1, std::false_type{});
            }
        }
    }

    // ---- a lane holds one row of the result, four neighbouring columns at a time
    if (u.parts > 1) {
        f32x4* const out = reinterpret_cast<f32x4*>(a.parts) + (size_t)u.slot * 4 * 8 * G_THREADS + tid;
        if (mine)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        f32x4 r = {acc[i][j][g * 4], acc[i][j][g * 4 + 1], acc[i][j][g * 4 + 2], acc[i][j][g * 4 + 3]};
                        if (!W) r *= unit_scale;
                        out[((i * 2 + j) * 4 + g) * G_THREADS] = r;
                    }
        return;
    }
    __syncthreads();                           // (the last stage has been read)
    if (!mine) return;
    float* const buffer = reinterpret_cast<float*>(lds) + wave * 32 * OUT_LD;
    const int end = W ? a.NOUT : hi;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f32x4 r[2][4];
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                r[j][g] = f32x4{acc[i][j][g * 4], acc[i][j][g * 4 + 1], acc[i][j][g * 4 + 2], acc[i][j][g * 4 + 3]};
                if (!W) r[j][g] *= unit_scale;
            }
        const int row = row0 + i * 32;
        if (row < end) store_rows<F32>(a, buffer, r, (W ? (size_t)e * mat : 0) + (size_t)row * a.K + cols0, end - row);
    }
}

// Adds up the parts of the tiles that were cut, in their order.  Four blocks to a tile, 32 rows each.
template <bool W, bool F32>
__global__ __launch_bounds__(G_THREADS) void grad_join_kernel(const grad_args a) {
    __shared__ find_scratch s_find;
    __shared__ __attribute__((aligned(16))) float s_out[4 * 32 * OUT_LD];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i = blockIdx.x & 3;
    unit u;
    if (!unit_of<W, true>(a, blockIdx.x >> 2, s_find, u)) return;
    const int cols0 = u.c0 + wave * 64, row = u.row0 + i * 32, end = W ? a.NOUT : u.hi;
    if (cols0 >= a.K || row >= end) return;
    f32x4 r[2][4] = {};
    const f32x4* in = reinterpret_cast<const f32x4*>(a.parts) + ((size_t)u.slot * 4 + i) * 8 * G_THREADS + tid;
    for (int p = 0; p < u.parts; ++p, in += 4 * 8 * G_THREADS)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int g = 0; g < 4; ++g) r[j][g] += in[(j * 4 + g) * G_THREADS];
    store_rows<F32>(a, s_out + wave * 32 * OUT_LD, r, (W ? (size_t)u.e * a.NOUT * a.K : 0) + (size_t)row * a.K + cols0, end - row);
}

}  // namespace

hipError_t set_grad_lds_limits() {
    for (const void* f : {(const void*)grad_kernel<false, 1, false>, (const void*)grad_kernel<true, 1, false>, (const void*)grad_kernel<true, 3, true>})
        if (const hipError_t e = hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, G_LDS); e != hipSuccess) return e;
    return hipSuccess;
}

namespace {

static_assert((size_t)G_SLOTS * GM * GN * sizeof(float) <= GRAD_WS_BYTES, "the parts of a round fit the workspace");

// tiles: as many as there can be; stages: of a whole sum
template <bool W, int PLANES, bool F32>
hipError_t launch(moe_ctx* c, const grad_args& a, int64_t tiles, int stages) {
    const bool known = !a.offsets;             // how many tiles there are
    const split_plan p = W && !known ? split_plan{(int)tiles, 0, 1} : plan_of((int)tiles, stages);
    int64_t units = p.whole + (int64_t)p.cut * p.parts;
    if (!known) units = W ? (tiles + 511) / 512 * 512 : tiles + G_SLOTS;
    grad_kernel<W, PLANES, F32><<<(unsigned)((units + 7) / 8 * 8 + 8), G_THREADS, G_LDS, c->stream>>>(a);
    const int cut = known ? p.cut : W ? 0 : G_SLOTS / 2;
    if (cut) grad_join_kernel<W, F32><<<(unsigned)(cut * 4), G_THREADS, 0, c->stream>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_linear_dgrad(moe_ctx* c, const uint16_t* dy, int64_t rows, int32_t NOUT, const uint8_t* Wq, const float* ws, int32_t K,
                               const int32_t* offsets, int32_t E, uint16_t* dx) {
    const grad_args a{dy, Wq, ws, offsets, rows, E, NOUT, K, 0, dx, static_cast<float*>(c->grad_ws)};
    return launch<false, 1, false>(c, a, (offsets ? rows / GM + E : (rows + GM - 1) / GM) * ((K + GN - 1) / GN), NOUT / GK);
}

hipError_t launch_linear_wgrad(moe_ctx* c, const uint16_t* dy, int64_t rows, int32_t NOUT, const uint8_t* xq, const float* xs, int32_t K,
                               const int32_t* offsets, int32_t E, int32_t accumulate, int32_t dtype, void* dW) {
    const grad_args a{dy, xq, xs, offsets, rows, E, NOUT, K, accumulate, dW, static_cast<float*>(c->grad_ws)};
    const int64_t tiles = (int64_t)E * (NOUT / GM) * ((K + GN - 1) / GN);
    const int stages = (int)((rows + GK - 1) / GK);
    return dtype == MOE_BF16 ? launch<true, 1, false>(c, a, tiles, stages) : launch<true, 3, true>(c, a, tiles, stages);
}

}  // namespace moe355
