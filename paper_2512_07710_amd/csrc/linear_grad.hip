// Gradients of the block-scaled FP8 linear, dense or grouped by expert: products of bf16 gradients with e4m3 codes on the bf16 matrix cores.
//
// Both have a matrix of codes [k][c] whose rows run along the sum:
//   dgrad   dx[p,c] = sum_n dy[p,n] * ws[n/128,c/128] Wq[n,c]     k = n: dy's rows run along the sum as well, the codes do not
//   wgrad   dW[n,c] = sum_p dy[p,n] * xs[c/128,p] xq[p,c]         k = p: neither does
// What does not run along the sum is transposed on its way from LDS to the registers by the transposing LDS reads.
//
// Bound by the bf16 matrix cores at the chip's power cap where there are many rows: a loop of 16x16x32 products from registers alone runs at 2.06
// PFLOP/s (32x32x16: 1.88), the library's bf16 products of these sizes at 1.32 to 1.53.  A tile is 128 x 256, two blocks to a CU: a wave's 128 x 64
// take 10 KiB of LDS for 0.5 million operations, and one block's products cover the other's waits.  dgrad 8192 x 8192 x
// 8192 827 us = 1.33 PFLOP/s, 4096 x 32768 x 5120 1145 = 1.20; wgrad 897 = 1.23 and 1165 = 1.18, with three planes for fp32 results 4096 x 4096 x 4096
// 324 = 0.42 (three times the products: 1.27); cards differ by 3 %.  With accumulate, dW is read just before it is written, 8 or 16 bytes of a row at a
// time: 128 experts of 5120 x 1536 under 32768 rows 811 -> 1432 us, 32768 x 5120 under 4096 rows 1222 -> 1287.  Fewer rows: the codes (dgrad) or the results (wgrad) at the memory's rate: 128 rows on 128 experts of
// 5120 x 1536 176 us = 5.7 TB/s read, wgrad 331 = 6.1 TB/s written.
#include "ffn_common.hpp"
#include "grad_common.hpp"
#include "grad_rules.hpp"

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

constexpr int G_THREADS = 256;                 // four waves, each all 128 rows of the tile and 64 of its columns
constexpr int DY_STAGE = GM * GK * 2, CODE_STAGE = GN * GK, SCALE_STAGE = 4 * GK * 4, G_STAGE = DY_STAGE + CODE_STAGE + SCALE_STAGE;
constexpr int OUT_PITCH = 64 * 2 + 16, OUT_BYTES = 16 * OUT_PITCH;             // a wave's 16 x 64 results on their way out
constexpr int G_LDS = 2 * G_STAGE + G_THREADS / 64 * OUT_BYTES;                // two blocks to a CU

struct grad_args {
    const uint16_t* dy;
    const uint8_t* codes;                      // Wq or xq
    const float* scales;                       // ws or xs
    const int32_t* offsets;                    // or null: one expert with all rows
    int64_t rows;
    int E, NOUT, K;
    int accumulate;
    int weight;                                // of a stage, for plan_of
    int cuts;                                  // whether tiles may be cut along the sum
    void* out;
    float* parts;                              // [units][rows / 32][2][4][256] f32x4: a thread's sums, in its own order
};

// expert e's rows (in the constant address space, so that they come as scalar loads where e is the same for all: the wait for a vector load would
// include the copies and stores that are under way)
__device__ inline void segment(const grad_args& a, int e, int& lo, int& hi) {
    if (!a.offsets) {
        lo = 0;
        hi = (int)a.rows;
        return;
    }
    const __attribute__((address_space(4))) int32_t* const at = (const __attribute__((address_space(4))) int32_t*)(uintptr_t)a.offsets + e;
    lo = min(max(at[0], 0), (int)a.rows);
    hi = min(max(at[1], lo), (int)a.rows);
}

struct find_scratch {
    int waves[G_THREADS / 64], found[4];
};
struct unit_place {
    int e, lo, hi;                             // expert and its rows
    int row0, c0;                              // first row and column of the tile
    int part, parts, slot;                     // part of the sum; its place in the workspace
};
// The unit of block b; JOIN: of the launch that adds up, a tile that was cut.  False: none.  Called by the whole block.
template <bool W, bool JOIN = false>
__device__ inline bool unit_of(const grad_args& a, int b, find_scratch& s, unit_place& u) {
    const int ctiles = (a.K + GN - 1) / GN, tid = threadIdx.x;
    int row_tiles = W ? a.E * (a.NOUT / GM) : (int)((a.rows + GM - 1) / GM);
    int first = 0, tiles = 0, l = 0, h = 0;    // (grouped dgrad) thread e: expert e's row tiles
    const bool search = !W && a.offsets;
    if (search) {
        if (tid < a.E) {
            l = min(max(a.offsets[tid], 0), (int)a.rows);
            h = min(max(a.offsets[tid + 1], l), (int)a.rows);
        }
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
    const split_plan p = !a.cuts ? split_plan{total, 0, 1} : plan_of(total, W ? (int)((a.rows + GK - 1) / GK) : a.NOUT / GK, a.weight, W ? 100 : fill_of(a.rows, row_tiles));
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
        const int n = unit_of_block(p, W && a.offsets, b);
        if (n < 0) return false;
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

// A wave's 32 x 64 values of the result, four neighbouring columns of row lane%16 of a lane's at a time, go through LDS to be stored as whole
// lines.  buffer: the wave's own place.
constexpr int OUT_LD = 68;                     // floats of a row there
template <bool F32>
__device__ inline void store_rows(const grad_args& a, float* buffer, const f32x4 (&r)[2][4], size_t at, int rows) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int j = 0; j < 4; ++j) *reinterpret_cast<f32x4*>(buffer + (h * 16 + (lane & 15)) * OUT_LD + j * 16 + (lane >> 4) * 4) = r[h][j];
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

// (dgrad) Sums are held in units of the present block's scale without its power of two, which the codes carry: a factor of less than two either way
// from block to block.  That power of two stays where every code, 2^-9 to 448, is a normal bf16 number; what a scale has beyond is left in the unit, which
// then is up to 2^10 or down to 2^-32 (a scale below the normal range).
struct block_scale {
    static constexpr uint32_t LEAST = (127 - 117) << 23, MOST = (127 + 118) << 23;             // 2^-117 and 2^118
    float scale = 1.f, pow2 = 1.f;
    int mask = -1;                             // on the codes
    __device__ float next(float s) {           // the factor on the sums
        const uint32_t bits = __float_as_uint(s) & 0x7FFFFFFFu, exponent = min(max(bits & 0x7F800000u, LEAST), MOST);
        const bool live = bits != 0, finite = bits < 0x7F800000u;
        mask = live ? -1 : 0;                  // a zero scale: the block adds nothing
        pow2 = live && finite ? __uint_as_float(exponent) : 1.f;
        const float to = !live ? scale : finite ? s * __uint_as_float((254u << 23) - exponent) : s;
        const float ratio = scale / to;
        scale = to;
        return ratio;
    }
};

// W: the weights' gradient; PLANES: bf16 planes of its scaled operand; F32: type of the result
template <bool W, int PLANES, bool F32>
__global__ __launch_bounds__(G_THREADS, 2) void grad_kernel(const grad_args a) {
    extern __shared__ __attribute__((aligned(1024))) char lds[];   // (the places of chunks are exchanged inside 256 bytes)
    __shared__ find_scratch s_find;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    unit_place u;
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

    // ---- copies of stage kb into its half of the ring; rows behind the segment repeat its last.  16-byte chunks of a row change places by
    // the row's number, so that each transposing or plain read of a wave meets every LDS bank once
    const int r4 = lane >> 4, r8 = lane >> 3, c16 = lane & 15;
    const uint32_t dy_pitch = (uint32_t)a.NOUT * 2, code_pitch = (uint32_t)a.K;
    // offsets of a lane from the first row that its wave's copy brings
    const uint32_t code_row = (uint32_t)r4 * code_pitch, code_chunk = (uint32_t)((c16 ^ r4) & 15) * 16, code_mask = (uint32_t)cmask * 16;
    uint32_t dy_off[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (W) dy_off[i] = (uint32_t)r4 * dy_pitch + (c16 ^ ((r4 | (i >> 1) << 2) << 1)) * 16;           // (rows 4 i on; only two of them differ)
        else dy_off[i] = (uint32_t)min(wave * 32 + i * 8 + r8, hi - 1 - row0) * dy_pitch + ((lane & 7) ^ ((i & 1) * 4 + (r8 >> 1))) * 16;
    auto copy = [&](int kb) {
        const uint32_t at = lds0 + (uint32_t)((kb - k0) & 1) * G_STAGE;
        const int last = W ? hi - lo - 1 - kb * GK : GK - 1;
        const char* const dy_base = reinterpret_cast<const char*>(W ? dy + (size_t)kb * GK * a.NOUT : dy + kb * GK);
        const uint8_t* const code_base = codes + (size_t)kb * GK * a.K;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t to = at + (wave * 4 + i) * 1024;
            const int row = wave * 16 + i * 4;                 // of the sum
            const uint32_t chunk = (code_chunk ^ i * 64) & code_mask;
            if (!W) {
                dma16(to, dy_off[i], dy_base);
                dma16(to + DY_STAGE, code_row + chunk, code_base + (size_t)row * code_pitch);
            } else if (last >= GK - 1) {
                dma16(to, dy_off[i], dy_base + (size_t)row * dy_pitch);
                dma16(to + DY_STAGE, code_row + chunk, code_base + (size_t)row * code_pitch);
            } else {
                const uint32_t r = (uint32_t)min(row + r4, last);
                dma16(to, r * dy_pitch + (dy_off[i] - (uint32_t)r4 * dy_pitch), dy_base);
                dma16(to + DY_STAGE, r * code_pitch + chunk, code_base);
            }
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
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");      // (the copies that are under way are not waited for)
    };

    // ---- this wave's part: 128 rows x 64 columns of the tile, in products of 16 x 16 over 32 steps of the sum, a stage is two groups of them.
    // A lane has eight steps: from 8 (lane/16) on
    const int cols0 = c0 + wave * 64;
    const bool mine = cols0 < a.K;
    uint32_t dy_at[2], code_at;
    if (W) {                                   // row of the sum 8 (lane/16) + (lane%16)/4, and 4 more; [0]: rows 0 to 15 of the tile
        const int f = (lane >> 2 & 3) | (r4 & 1) << 2;
        dy_at[0] = dy_at[1] = lds0 + (r4 * 8 + (lane >> 2 & 3)) * 256 + (((lane >> 1 & 1) ^ f << 1) << 4) + (lane & 1) * 8;
    } else {                                   // [g]: group g
#pragma unroll
        for (int g = 0; g < 2; ++g) dy_at[g] = lds0 + c16 * 128 + (((g * 4 + r4) ^ (c16 >> 1)) << 4);
    }
    code_at = lds0 + DY_STAGE + (r4 * 8 + (c16 >> 1)) * 256 + (((wave * 4) ^ ((r4 & 1) * 8 + (c16 >> 1))) << 4) + (lane & 1) * 8;
    const uint32_t scale_at = lds0 + DY_STAGE + CODE_STAGE + (wave >> 1) * 256 + r4 * 32;

    v4f acc[8][4];                             // [rows / 16][columns / 16]
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = v4f{0.f, 0.f, 0.f, 0.f};
    v8s d[8];                                  // dy: of the present group, replaced by the next one's as soon as they have been used
    v2i q[2][4];                               // codes of 4 x 16 columns, [of group 0 or 1]
    v4f sc[2][2];                              // (wgrad) the scales of a lane's eight steps, [of group 0 or 1]
    constexpr int NJ = PLANES == 1 ? 2 : 1, PARTS = 4 / NJ;    // a group's products in parts of 16 NJ columns
    u32x4 c[2][NJ][PLANES];                    // codes as operands: of the present and of the next part
    auto fetch_codes = [&](uint32_t at, int g) {               // at: the stage's offset
#pragma unroll
        for (int j = 0; j < 4; ++j) q[g][j] = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_v2i_ptr)(uintptr_t)((code_at ^ j * 16) + at + g * 8192));
        if (W) {
            sc[g][0] = *(lds_v4f_ptr)(uintptr_t)(scale_at + at + g * 128);
            sc[g][1] = *(lds_v4f_ptr)(uintptr_t)(scale_at + at + g * 128 + 16);
        }
    };
    auto fetch_dy = [&](uint32_t at, int g, int i) {
        if (W) {
            const uint32_t p = (dy_at[0] ^ i * 32) + at + g * 8192;
            const v4s x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s_ptr)(uintptr_t)p);
            const v4s y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s_ptr)(uintptr_t)(p + 1024));
            d[i] = __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
        } else {
            d[i] = *(lds_v8s_ptr)(uintptr_t)(dy_at[g] + at + i * 2048);
        }
    };
    // (In the constant address space, so that they come as scalar loads: a vector load's wait would include the copies)
    const __attribute__((address_space(4))) float* const block_scales = (const __attribute__((address_space(4))) float*)(uintptr_t)(
        a.scales + (size_t)e * (a.NOUT / QBLOCK) * (a.K / QBLOCK) + min(cols0, a.K - 1) / QBLOCK);
    block_scale unit;                          // (dgrad) of acc
    // A quarter of the codes of 16 columns: two steps of the sum.  (The empty asm keeps the instructions where they are asked for; they would
    // be moved down to where the operand is used)
    auto convert = [&](u32x4 (&o)[PLANES], const v2i& codes_, const v4f (&scale)[2], int h) {
        if (!W) {
            const int w = codes_[h >> 1] & unit.mask;
            const v2bf x = h & 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, unit.pow2, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, unit.pow2, false);
            uint32_t r = __builtin_bit_cast(uint32_t, x);
            asm volatile("" : "+v"(r));
            o[0][h] = r;
            return;
        }
        const v2f x = h & 1 ? __builtin_amdgcn_cvt_pk_f32_fp8(codes_[h >> 1], true) : __builtin_amdgcn_cvt_pk_f32_fp8(codes_[h >> 1], false);
        const float y[2] = {x[0] * scale[h >> 1][(h & 1) * 2], x[1] * scale[h >> 1][(h & 1) * 2 + 1]};
        if (PLANES == 1) {
            const v2bf z = {(__bf16)y[0], (__bf16)y[1]};
            uint32_t r = __builtin_bit_cast(uint32_t, z);
            asm volatile("" : "+v"(r));
            o[0][h] = r;
            return;
        }
        // 24 bits in three times eight, cut off, so that all planes have the sign of y and none is zero unless y is: an infinite gradient times
        // each of them is the infinity that it is times y (an infinite or NaN y is whole in the first plane)
        float rest[2] = {y[0], y[1]};
#pragma unroll
        for (int p = 0; p < PLANES; ++p) {
            uint32_t r = __builtin_amdgcn_perm(__float_as_uint(rest[1]), __float_as_uint(rest[0]), 0x07060302u);
            asm volatile("" : "+v"(r));
            o[p][h] = r;
            if (p + 1 < PLANES)
#pragma unroll
                for (int v = 0; v < 2; ++v) {
                    rest[v] -= __uint_as_float(__float_as_uint(rest[v]) & 0xFFFF0000u);
                    rest[v] = copysignf(fmaxf(fabsf(rest[v]), fminf(fabsf(y[v]), 0x1p-126f)), y[v]);
                }
        }
    };
    // Part P of a group's products: all rows, columns 16 NJ P and on.  Between them, piece by piece, what comes behind needs: the codes of the next
    // part are converted, those of the next group (at `at`, group G) come from LDS in the first part, and in the last dy of the next group takes
    // the place of what has been used.  The compiler would gather these and wait for them.
    auto part = [&](auto I_, auto P_, uint32_t at, auto G_) {
        constexpr int I = decltype(I_)::value, P = decltype(P_)::value, G = decltype(G_)::value, NP = (P + 1) % PARTS, NG = P + 1 < PARTS ? 1 - G : G;
        if (P == 0) fetch_codes(at, G);
#pragma unroll
        for (int i = 0; i < I; ++i) {
#pragma unroll
            for (int p = 0; p < PLANES; ++p)
#pragma unroll
                for (int jj = 0; jj < NJ; ++jj) {
                    const int j = i & 1 ? NJ - 1 - jj : jj;    // (neighbouring products share an operand)
                    v4f& r = acc[i][P * NJ + j];
                    r = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, c[P & 1][j][p]), __builtin_bit_cast(v8bf, d[i]), r, 0, 0, 0);
                }
            __builtin_amdgcn_sched_barrier(0);
            if (P == PARTS - 1) fetch_dy(at, G, i);
#pragma unroll
            for (int n = i * 8 / I; n < (i + 1) * 8 / I; ++n)
                if (NJ == 2 || n % 2 == 0) convert(c[NP & 1][NJ == 2 ? n >> 2 : 0], q[NG][NP * NJ + (NJ == 2 ? n >> 2 : 0)], sc[NG], NJ == 2 ? n & 3 : n / 2);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    auto group = [&](auto I_, uint32_t at, auto G_) {
        part(I_, step<0>{}, at, G_);
        part(I_, step<1>{}, at, G_);
        if (PARTS > 2) {
            part(I_, step<(PARTS > 2 ? 2 : 0)>{}, at, G_);
            part(I_, step<(PARTS > 2 ? 3 : 1)>{}, at, G_);
        }
    };

    // ---- the sum.  The barrier that hands over the stages stands between the two groups of a stage: the second's operands have been
    // read by then, and those of the next stage come during its products
    auto sum = [&](auto I_) {
        constexpr int I = decltype(I_)::value;
        copy(k0);
        if (nk > k0 + 1) {
            copy(k0 + 1);
            asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(COPIES) : "memory");
        } else {
            asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
        }
        if (W) clear_behind(k0);
        auto next_block = [&](int kb) { return unit.next(block_scales[(size_t)(kb / 2) * (a.K / QBLOCK)]); };
        float ratio = W ? 1.f : next_block(k0);
        fetch_codes(0, 0);
#pragma unroll
        for (int i = 0; i < I; ++i) fetch_dy(0, 0, i);
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int h = 0; h < 4; ++h) convert(c[0][j], q[0][j], sc[0], h);
        for (int kb = k0; kb < nk; ++kb) {
            const uint32_t at = (uint32_t)((kb - k0) & 1) * G_STAGE;
            if (!W && (kb & 1) == 0) {         // of a block of scales the first stage
#pragma unroll
                for (int i = 0; i < I; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[i][j] *= ratio;
            }
            group(I_, at, step<1>{});
            if (kb + 1 < nk) {
                asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");   // stage kb+1 is there, and this one has been read
                if (kb + 2 < nk) copy(kb + 2);
                if (W) clear_behind(kb + 1);
            }
            // (behind the last stage what is fetched is of no use, and not used)
            part(I_, step<0>{}, G_STAGE - at, step<0>{});
            if (!W && (kb & 1) && kb + 1 < nk) ratio = next_block(kb + 1);
            part(I_, step<1>{}, G_STAGE - at, step<0>{});
            if (PARTS > 2) {
                part(I_, step<(PARTS > 2 ? 2 : 0)>{}, G_STAGE - at, step<0>{});
                part(I_, step<(PARTS > 2 ? 3 : 1)>{}, G_STAGE - at, step<0>{});
            }
        }
    };
    // An expert's last tile: the products of the quarters of its rows that there are (experts 32768 x 5120 x 1536 zipf, all eight row tiles 644 us, halves
    // 608, quarters 599; 128 rows on 128 experts 206, 181, 176)
    if (nk > k0) {
        const int there = W ? GM : hi - row0;
        if (W || there > GM / 4 * 3) sum(step<8>{});
        else if (there > GM / 2) sum(step<W ? 8 : 6>{});
        else if (there > GM / 4) sum(step<W ? 8 : 4>{});
        else sum(step<W ? 8 : 2>{});
    }

    // ---- the result: a lane holds rows lane%16 of its tiles of 16 x 16, four neighbouring columns of each
    if (!mine) return;
    const int rows = W ? GM : min(hi - row0, GM);
    if (u.parts > 1) {
        char* const out = reinterpret_cast<char*>(a.parts) + ((size_t)u.slot * 4 * 8 * G_THREADS + wave * 64) * sizeof(f32x4);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i * 32 < rows)                 // (those that there are)
#pragma unroll
                for (int n = 0; n < 8; ++n) {
                    const v4f r = acc[i * 2 + (n >> 2)][n & 3];
                    __builtin_nontemporal_store(W ? r : r * unit.scale, reinterpret_cast<f32x4*>(out + (i * 8 + n) * G_THREADS * sizeof(f32x4) + (uint32_t)lane * 16));
                }
        return;
    }
    // bf16 goes through LDS, a wave's own part of it, to be stored as whole lines of 128 bytes, past the caches (1 to 4 % faster at all sizes tried).
    // fp32 has 64 bytes of a row of each column tile in four lanes; rows and column tiles change places by pairs of lanes for whole lines, which go past the
    // caches too (8000 rows on 32 experts of 2048 x 4096, zipf 491 -> 469 us, 200 x 4096 x 2048 22.8 -> 21.5, 40 x 6144 x 4096 level; the 64 bytes alone
    // past the caches 26 -> 33)
    constexpr int BYTES = F32 ? 4 : 2;
    char* const out_lds = lds + 2 * G_STAGE + wave * OUT_BYTES;
    char* base = static_cast<char*>(a.out) + ((W ? (size_t)e * mat : 0) + (size_t)row0 * a.K + cols0) * BYTES;
    const uint32_t own = F32 ? ((c16 & 7) * (uint32_t)a.K + (c16 >> 3) * 16 + r4 * 4) * BYTES : (c16 * (uint32_t)a.K + r4 * 4) * BYTES, line = (r8 * (uint32_t)a.K + (lane & 7) * 8) * BYTES;
#pragma unroll
    for (int i = 0; i < 8; ++i, base += (size_t)16 * a.K * BYTES) {
        if (i * 16 >= rows) break;
        if (F32) {
#pragma unroll
            for (int j = 0; j < 4; j += 2) {
                const bool high = c16 >= 8;
                v4f there = high ? acc[i][j] : acc[i][j + 1];
#pragma unroll
                for (int n = 0; n < 4; ++n) there[n] = __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(there[n]), 0x128, 0xf, 0xf, false));
                v4f up = high ? there : acc[i][j], down = high ? acc[i][j + 1] : there;
                f32x4* const p = reinterpret_cast<f32x4*>(base + j * 64 + own);
                f32x4* const q = reinterpret_cast<f32x4*>(base + (size_t)8 * a.K * BYTES + j * 64 + own);
                if (a.accumulate) {
                    up += *p;
                    down += *q;
                }
                __builtin_nontemporal_store(up, p);
                __builtin_nontemporal_store(down, q);
            }
            continue;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v4f r = acc[i][j];
            if (!W) r *= unit.scale;
            if (W && a.accumulate) {
                const u32x2 was = *reinterpret_cast<const u32x2*>(base + j * 32 + own);
                r += v4f{bf16lo(was[0]), bf16hi(was[0]), bf16lo(was[1]), bf16hi(was[1])};
            }
            *reinterpret_cast<u32x2*>(out_lds + c16 * OUT_PITCH + j * 32 + r4 * 8) = u32x2{bf16_pair(r[0], r[1]), bf16_pair(r[2], r[3])};
        }
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const u32x4 v = *reinterpret_cast<const u32x4*>(out_lds + (h * 8 + r8) * OUT_PITCH + (lane & 7) * 16);
            if (i * 16 + h * 8 + r8 < rows) __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(base + (size_t)h * 8 * a.K * BYTES + line));
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// Adds up the parts of the tiles that were cut.  A block has 32 rows x 64 columns of a tile; each of its waves adds every fourth part, and the first
// adds those sums, in their order: short chains, the parts come from other XCDs.
template <bool W, bool F32>
__global__ __launch_bounds__(G_THREADS) void grad_join_kernel(const grad_args a) {
    constexpr int WAVES = G_THREADS / 64;
    __shared__ find_scratch s_find;
    __shared__ __attribute__((aligned(16))) f32x4 s_sums[WAVES - 1][8][64];
    __shared__ __attribute__((aligned(16))) float s_out[32 * OUT_LD];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = blockIdx.x >> 2 & 3, column = blockIdx.x & 3;
    unit_place u;
    if (!unit_of<W, true>(a, blockIdx.x >> 4, s_find, u)) return;
    const int cols0 = u.c0 + column * 64, row = u.row0 + i * 32, end = W ? a.NOUT : u.hi;
    if (cols0 >= a.K || row >= end) return;
    f32x4 r[2][4] = {};
    const f32x4* const in = reinterpret_cast<const f32x4*>(a.parts) + ((size_t)u.slot * 4 + i) * 8 * G_THREADS + column * 64 + lane;
#pragma unroll 3
    for (int p = wave; p < u.parts; p += WAVES)
#pragma unroll
        for (int n = 0; n < 8; ++n) r[n >> 2][n & 3] += __builtin_nontemporal_load(in + ((size_t)p * 4 * 8 + n) * G_THREADS);
    if (wave > 0)
#pragma unroll
        for (int n = 0; n < 8; ++n) s_sums[wave - 1][n][lane] = r[n >> 2][n & 3];
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int w = 0; w < WAVES - 1; ++w)
#pragma unroll
        for (int n = 0; n < 8; ++n) r[n >> 2][n & 3] += s_sums[w][n][lane];
    store_rows<F32>(a, s_out, r, (W ? (size_t)u.e * a.NOUT * a.K : 0) + (size_t)row * a.K + cols0, end - row);
}

// dgrad of few rows of one matrix, where all that counts is that the codes come at the rate of the memory.  A tile is up to 64 rows and 64 or 128
// columns; each wave of a block has a part of the sum of its own, two or three stages of which it asks for at a time (no barriers), and the waves' sums
// meet in LDS: a fourth of the parts that would go through memory otherwise.  1 x 6144 x 4096 8.6 us (25 MB of codes: 5.2 at a copy's rate, the rest is
// the second launch, which adds the parts up), 40 rows 13.3, 16 x 25600 x 7168 37.9 us = 4.84 TB/s.
template <int RT, int JT>                      // rows and columns in tiles of 16
__global__ __launch_bounds__(GF_WAVES * 64, 2) void few_dgrad_kernel(const grad_args a, int parts, int tile_rows, int row_tiles) {
    constexpr int COLS = JT * 16, BATCH = JT == 4 ? 3 : 2, STAGE = GK * COLS;
    constexpr int SUMS = RT * 16 * 64 * 4, EACH = SUMS > BATCH * STAGE ? SUMS : BATCH * STAGE;
    __shared__ __attribute__((aligned(1024))) char lds[GF_WAVES * EACH];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r4 = lane >> 4, c16 = lane & 15;
    const int tiles = a.K / COLS * row_tiles, units = tiles * parts, x = blockIdx.x & 7, at = blockIdx.x >> 3;
    const int from = (int)((int64_t)units * x / 8), n = from + at;         // (an XCD has neighbouring columns)
    if (n >= (int)((int64_t)units * (x + 1) / 8)) return;
    const int part = n / tiles, c0 = n % tiles / row_tiles * COLS, row0 = n % row_tiles * tile_rows, rows = min((int)a.rows - row0, tile_rows);
    const int stages = a.NOUT / GK, own = part * GF_WAVES + wave, all = parts * GF_WAVES;
    const int k0 = (int)((int64_t)stages * own / all), nk = (int)((int64_t)stages * (own + 1) / all);
    char* const mine = lds + wave * EACH;
    const uint32_t mine0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)mine;
    // the 16-byte chunks of a row change places by the row's number over 256 / COLS: a transposing read meets each bank as often as the others
    constexpr int AT_ONCE = 1024 / COLS;       // rows that a copy brings
    const int chunk = JT == 4 ? (lane & 3) ^ r4 : (lane & 7) ^ r4;         // (JT == 8: and ^ 4 in every other copy)
    const uint32_t row_off = (uint32_t)(lane / JT) * (uint32_t)a.K;
    const uint32_t code_at = mine0 + (r4 * 8 + (c16 >> 1)) * COLS + (lane & 1) * 8;
    const int swap = JT == 4 ? (r4 * 2 + (c16 >> 3)) & 3 : (r4 * 4 + (c16 >> 2)) & 7;
    const uint16_t* dy_row[RT];
#pragma unroll
    for (int i = 0; i < RT; ++i) dy_row[i] = a.dy + (size_t)(row0 + min(i * 16 + c16, rows - 1)) * a.NOUT + r4 * 8;
    const __attribute__((address_space(4))) float* const block_scales =
        (const __attribute__((address_space(4))) float*)(uintptr_t)(a.scales + c0 / QBLOCK);
    v4f acc[RT][JT];
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int j = 0; j < JT; ++j) acc[i][j] = v4f{0.f, 0.f, 0.f, 0.f};
    block_scale unit;
    for (int kb = k0; kb < nk; kb += BATCH) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // the batch before has been read
#pragma unroll
        for (int b = 0; b < BATCH; ++b)
            if (kb + b < nk)
#pragma unroll
                for (int i = 0; i < GK / AT_ONCE; ++i)
                    dma16(mine0 + b * STAGE + i * 1024, row_off + (JT == 8 && i & 1 ? chunk ^ 4 : chunk) * 16,
                          a.codes + (size_t)((kb + b) * GK + i * AT_ONCE) * a.K + c0);
        v8s d[BATCH][2][RT];
#pragma unroll
        for (int b = 0; b < BATCH; ++b)
            if (kb + b < nk)
#pragma unroll
                for (int g = 0; g < 2; ++g)
#pragma unroll
                    for (int i = 0; i < RT; ++i) d[b][g][i] = *reinterpret_cast<const v8s*>(dy_row[i] + (size_t)(kb + b) * GK + g * 32);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
        for (int b = 0; b < BATCH; ++b) {
            if (kb + b >= nk) continue;
            const float ratio = unit.next(block_scales[(size_t)((kb + b) / 2) * (a.K / QBLOCK)]);
#pragma unroll
            for (int i = 0; i < RT; ++i)
#pragma unroll
                for (int j = 0; j < JT; ++j) acc[i][j] *= ratio;
#pragma unroll
            for (int g = 0; g < 2; ++g)
#pragma unroll
                for (int j = 0; j < JT; ++j) {
                    v2i q = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_v2i_ptr)(uintptr_t)(code_at + b * STAGE + g * 32 * COLS + ((j ^ swap) << 4)));
                    q[0] &= unit.mask;
                    q[1] &= unit.mask;
                    const v8bf c = codes_bf16(q, unit.pow2);
#pragma unroll
                    for (int i = 0; i < RT; ++i)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(c, __builtin_bit_cast(v8bf, d[b][g][i]), acc[i][j], 0, 0, 0);
                }
        }
    }
    f32x4* const sums = reinterpret_cast<f32x4*>(lds);         // [wave][row tile][column tile][lane] of 64 columns
#pragma unroll
    for (int h = 0; h < JT; h += 4) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) sums[((wave * RT + i) * 4 + j) * 64 + lane] = acc[i][h + j] * unit.scale;
        __syncthreads();
        for (int i = 0; i < RT; ++i) {         // wave w: column tile w
            f32x4 r = sums[(i * 4 + wave) * 64 + lane];
#pragma unroll
            for (int w = 1; w < GF_WAVES; ++w) r += sums[((w * RT + i) * 4 + wave) * 64 + lane];
            const int row = i * 16 + c16;
            if (row >= rows) continue;
            const size_t o = (size_t)(row0 + row) * a.K + c0 + (h + wave) * 16 + r4 * 4;
            if (parts > 1) __builtin_nontemporal_store(r, reinterpret_cast<f32x4*>(a.parts + (size_t)part * a.rows * a.K + o));
            else *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.out) + o) = u32x2{bf16_pair(r[0], r[1]), bf16_pair(r[2], r[3])};
        }
    }
}

// Adds up the parts, in their order; a thread has four columns
__global__ __launch_bounds__(G_THREADS) void few_join_kernel(const grad_args a, int parts) {
    const size_t n = (size_t)a.rows * a.K / 4, i = (size_t)blockIdx.x * G_THREADS + threadIdx.x;
    if (i >= n) return;
    const f32x4* const in = reinterpret_cast<const f32x4*>(a.parts) + i;
    f32x4 r = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int p = 0; p < parts; ++p) r += __builtin_nontemporal_load(in + p * n);
    reinterpret_cast<u32x2*>(a.out)[i] = u32x2{bf16_pair(r[0], r[1]), bf16_pair(r[2], r[3])};
}

}  // namespace

hipError_t set_grad_lds_limits() {
    for (const void* f : {(const void*)grad_kernel<false, 1, false>, (const void*)grad_kernel<true, 1, false>, (const void*)grad_kernel<true, 3, true>})
        if (const hipError_t e = hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, G_LDS); e != hipSuccess) return e;
    return hipSuccess;
}

namespace {

static_assert((size_t)512 * GF_ROWS * 128 * sizeof(float) <= GRAD_WS_BYTES, "the parts of few rows fit the workspace");
static_assert((size_t)G_SLOTS * GM * GN * sizeof(float) <= GRAD_WS_BYTES, "the parts of a round fit the workspace");

// tiles: as many as there can be; stages: of a whole sum
template <bool W, int PLANES, bool F32>
hipError_t launch(moe_ctx* c, grad_args a, int64_t tiles, int stages) {
    // Grouped, the device alone knows how many tiles there are: they are cut only where they are sure to be less than a round (the second launch
    // costs 5 us whether there is something to add up or not), and in the weights' gradient, where sums differ in length, not at all
    const bool known = !a.offsets;
    a.cuts = known || (!W && tiles <= G_SLOTS);
    const split_plan p = known ? plan_of((int)tiles, stages, a.weight, W ? 100 : fill_of(a.rows, (int)((a.rows + GM - 1) / GM))) : split_plan{(int)tiles, 0, 1};
    const int64_t units = known ? (int64_t)p.whole + (int64_t)p.cut * p.parts : a.cuts ? G_SLOTS : tiles;
    grad_kernel<W, PLANES, F32><<<(unsigned)blocks_of(units, W && !known), G_THREADS, G_LDS, c->stream>>>(a);
    const int cut = known ? p.cut : a.cuts ? (int)(tiles < G_SLOTS / 2 ? tiles : G_SLOTS / 2) : 0;
    if (cut) grad_join_kernel<W, F32><<<(unsigned)(cut * 16), G_THREADS, 0, c->stream>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_linear_dgrad(moe_ctx* c, const uint16_t* dy, int64_t rows, int32_t NOUT, const uint8_t* Wq, const float* ws, int32_t K,
                               const int32_t* offsets, int32_t E, uint16_t* dx) {
    const grad_args a{dy, Wq, ws, offsets, rows, E, NOUT, K, 0, 10, 0, dx, static_cast<float*>(c->grad_ws)};
    if (!offsets && few_rows(rows, NOUT, K)) {
        const int row_tiles = ((int)rows + GF_ROWS - 1) / GF_ROWS, rt = (((int)rows + row_tiles - 1) / row_tiles + 15) / 16;
        const int cols = gf_cols(rt * 16, NOUT, K), parts = gf_parts(rt * 16, row_tiles, NOUT, K);
        const auto kernel = cols == 64 ? (rt == 1 ? few_dgrad_kernel<1, 4> : rt == 2 ? few_dgrad_kernel<2, 4> : rt == 3 ? few_dgrad_kernel<3, 4> : few_dgrad_kernel<4, 4>)
                                       : (rt == 1 ? few_dgrad_kernel<1, 8> : rt == 2 ? few_dgrad_kernel<2, 8> : rt == 3 ? few_dgrad_kernel<3, 8> : few_dgrad_kernel<4, 8>);
        kernel<<<(unsigned)((K / cols * row_tiles * parts + 7) / 8 * 8), GF_WAVES * 64, 0, c->stream>>>(a, parts, rt * 16, row_tiles);
        if (parts > 1) few_join_kernel<<<(unsigned)((rows * K / 4 + G_THREADS - 1) / G_THREADS), G_THREADS, 0, c->stream>>>(a, parts);
        return hipGetLastError();
    }
    return launch<false, 1, false>(c, a, (offsets ? rows / GM + E : (rows + GM - 1) / GM) * ((K + GN - 1) / GN), NOUT / GK);
}

hipError_t launch_linear_wgrad(moe_ctx* c, const uint16_t* dy, int64_t rows, int32_t NOUT, const uint8_t* xq, const float* xs, int32_t K,
                               const int32_t* offsets, int32_t E, int32_t accumulate, int32_t dtype, void* dW) {
    const grad_args a{dy, xq, xs, offsets, rows, E, NOUT, K, accumulate, dtype == MOE_BF16 ? 10 : 25, 0, dW, static_cast<float*>(c->grad_ws)};
    const int64_t tiles = (int64_t)E * (NOUT / GM) * ((K + GN - 1) / GN);
    const int stages = (int)((rows + GK - 1) / GK);
    return dtype == MOE_BF16 ? launch<true, 1, false>(c, a, tiles, stages) : launch<true, 3, true>(c, a, tiles, stages);
}

}  // namespace moe355
