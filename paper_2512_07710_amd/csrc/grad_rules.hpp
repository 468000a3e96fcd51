// How the products of linear_grad.hip are cut into units and dealt to blocks, and norm.hip's rows to blocks and launches.  Host and device.
#pragma once
#include <cstdint>

namespace moe355 {

constexpr int GM = 128, GN = 256;              // tile of the result: rows (along dy) and columns (along the codes)
constexpr int GK = 64;                         // steps of the sum that are staged at a time
constexpr int G_MIN_PART = 4;                  // stages of a part of a sum at least

// Tiles are dealt to the XCDs (blockIdx % 8) in runs, and run through a band of eight tile rows column by column, so that the 64 tiles that an XCD
// works on at a time share their operands in its L2 (dgrad 8192 x 8192 x 8192 with bands of 4 | 8 | 16: 858 | 851 | 870 us, experts 32768 x 5120 x 1536
// zipf 587 | 598 | 624, 2600 x 8192 x 8192 304 | 308 | 314; wgrad 4096 x 32768 x 5120 1199 | 1182 | 1205).  Tiles that do not fill a round
// of the chip are cut along the sum: parts go to the workspace and a second launch adds them up.
constexpr int G_SLOTS = 512;                   // blocks that run at a time
constexpr int G_BAND = 8, G_RUN = 16;
constexpr int G_PART = 18;                     // parts that go through memory in the time of a stage
struct split_plan {
    int whole, cut, parts;                     // tiles done at once; tiles in parts, and how many parts
};
// The host launches by this plan and each block works out its own: whole numbers throughout, so that both come to the same one.
// weight: time of a stage, in tenths of a bf16 one; fill: how much of the tiles' rows there is, in percent
__host__ __device__ inline split_plan plan_of(int tiles, int stages, int weight, int fill) {
    const split_plan none{tiles, 0, 1};
    const int rest = tiles % G_SLOTS;
    if (rest == 0) return none;
    const int most = G_SLOTS / rest < stages / G_MIN_PART ? G_SLOTS / rest : stages / G_MIN_PART;
    // the rest of many: what is saved against what the parts' way through memory costs (dgrad 4096 x 32768 x 5120 not cut 1324 us, cut 1160; 4096 x
    // 8192 x 5120 325, 295; 2600 x 8192 x 8192 341, 305; but 4096 x 2048 x 5120 85.8, 96.2 and 4096 x 4096 x 5120 166, 163)
    if (tiles >= G_SLOTS) {
        if (most < 3 || (int64_t)stages * (11 * most - 20) < (int64_t)480 * most) return none;     // stages (0.55 - 1 / most) < 24
        return split_plan{tiles - rest, rest, most};
    }
    // p parts take stages / p, and 4 for the second launch with 1 for every 18 full parts that go through memory: the best p is the last that
    // p (p-1) rest / 18 <= stages holds for.  (Measured with 18 | 26 | 38 and with as many parts as fit, us: dgrad 200 x 6144 x 4096 31.4 | 34.8 | 33.8 |
    // 34.3, 500 x 4096 x 4096 35.8 | 38.7 | 38.2 | 39.3, 8000 x 1024 x 1024 21.6 | 21.5 | 21.7 | 45; wgrad 700 x 2048 x 3584 17.5 | 17.5 | 17.5 | 38,
    // 1000 x 2048 x 2048 22.6 | 22.6 | 22.6 | 35)
    const int64_t sum = (int64_t)stages * weight * G_PART * 10;
    int p = 1;
    while (p < most && (int64_t)p * (p + 1) * rest * fill <= sum) ++p;
    if (sum * (p - 1) < p * ((int64_t)400 * G_PART + (int64_t)rest * p * fill)) return none;
    return split_plan{tiles - rest, rest, p};
}

__host__ __device__ inline int fill_of(int64_t rows, int row_tiles) {
    const int64_t room = (int64_t)row_tiles * GM;
    return rows >= room ? 100 : (int)(rows * 100 / room);
}

// The unit of block b, or -1.  Units 0 .. whole-1 are whole tiles, the others the cut ones' parts.  turns: runs of 16 units, taken in turns (experts'
// weights' gradients: sums differ in length, and an expert's tiles go to several XCDs); otherwise one run for each XCD.  Runs of 64 | 32 | 16 | 8,
// us: 16384 rows, 64 experts of 2048 x 1024, zipf 164 | 121 | 107 | 110, 32768, 128 of 5120 x 1536, zipf 868 | 796 | 804 | 820, uniform 809 | 833 |
// 830 | 847, 32768, 32 of 4096 x 4096 1163 | 1134 | 1144 | 1147.
__host__ __device__ inline int unit_of_block(const split_plan& p, bool turns, int b) {
    const int units = p.whole + p.cut * p.parts, x = b & 7, at = b >> 3;
    if (turns) {
        const int n = (at / G_RUN * 8 + x) * G_RUN + at % G_RUN;
        return n < units ? n : -1;
    }
    // whole tiles in eight runs, then the parts
    const int from = (int)((int64_t)p.whole * x / 8), count = (int)((int64_t)p.whole * (x + 1) / 8) - from;
    const int parts = units - p.whole, pfrom = (int)((int64_t)parts * x / 8), pcount = (int)((int64_t)parts * (x + 1) / 8) - pfrom;
    if (at >= count + pcount) return -1;
    return at < count ? from + at : p.whole + pfrom + (at - count);
}
// Few rows (dgrad of one matrix): tiles of up to 64 rows and 64 or 128 columns, the sum cut into stages for the block's four waves and `parts` blocks.
// us with 64 | 128 columns: 40 x 6144 x 4096 15.4 | 13.3, 48 x 25600 x 7168 66 | 47, 64 x 25600 x 7168 73 | 57, but 64 x 6144 x 5120 21.8 | 23.6,
// 64 x 1024 x 1024 8.7 | 10.6, 10 x 3584 x 3584 8.0 | 10.4.  Against the tiles of 128 rows: 1 x 6144 x 4096 8.6 for 19.4, 65 x 6144 x 4096 16.2 for
// 22.8, 128 x 2048 x 2048 10.4 for 16.2, 64 x 25600 x 7168 57 for 59, but 128 x 5120 x 5120 28.7 for 25.1.
constexpr int GF_ROWS = 64, GF_WAVES = 4;
inline int gf_cols(int rows, int NOUT, int K) { return (rows > 48 ? (int64_t)NOUT * K >= 1 << 26 : K >= 4096) ? 128 : 64; }
inline bool few_rows(int64_t rows, int NOUT, int K) { return rows <= GF_ROWS || (rows <= 2 * GF_ROWS && rows * NOUT * K <= (int64_t)1 << 31); }
// (rows: of a tile; row_tiles: of them.  Two blocks to a CU, also where three fit: 768 | 512 blocks at most, 10 x 3584 x 3584 9.8 | 8.0 us, 5 x 20480 x
// 1024 11.1 | 10.0, 30 x 2048 x 1024 8.0 | 7.9; 512 | 384, 40 x 6144 x 4096 13.3 | 14.7)
inline int gf_parts(int rows, int row_tiles, int NOUT, int K) {
    const int room = G_SLOTS / (K / gf_cols(rows, NOUT, K) * row_tiles), most = NOUT / GK / GF_WAVES, parts = room < most ? room : most;
    return parts < 1 ? 1 : parts;
}

// The norm's rows of a block: several, for the sake of their scales, as long as 32 waves are left for a CU and no block is so long that the last ones run
// alone (32768 x 7168: 16 rows 352 us, 8 340, 4 332; 16384 x 2048: 8 rows 45.5, 4 47.7)
constexpr int NORM_ROWS = 16;
inline int norm_rows_per_block(int64_t rows, int cols, int threads, bool codes) {
    if (!codes) return 1;
    int64_t n = rows * (threads / 64) / 8192;
    if (n > 32768 / cols) n = 32768 / cols;
    return n < 1 ? 1 : n > NORM_ROWS ? NORM_ROWS : (int)n;
}
// blocks of the next launch over `rows` rows (a grid has fewer than 2^32 threads)
inline int64_t norm_blocks(int64_t rows, int threads, int per_block) {
    const int64_t blocks = (rows + per_block - 1) / per_block, most = ((int64_t)1 << 31) / threads;
    return blocks < most ? blocks : most;
}

// blocks of a launch that reach every one of up to `units` units
inline int64_t blocks_of(int64_t units, bool turns) { return turns ? (units + 8 * G_RUN - 1) / (8 * G_RUN) * (8 * G_RUN) : (units + 7) / 8 * 8 + 8; }

}  // namespace moe355
