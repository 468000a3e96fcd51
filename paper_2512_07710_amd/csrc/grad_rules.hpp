// How the products of linear_grad.hip are cut into units and dealt to blocks.  Host and device.
#pragma once
#include <cstdint>

namespace moe355 {

constexpr int GM = 128, GN = 256;              // tile of the result: rows (along dy) and columns (along the codes)
constexpr int GK = 64;                         // steps of the sum that are staged at a time
constexpr int G_MIN_PART = 4;                  // stages of a part of a sum at least

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

// The unit of block b, or -1.  Units 0 .. whole-1 are whole tiles, the others the cut ones' parts.  turns: runs of 64 units, taken in turns
// (where sums differ in length); otherwise one run for each XCD.
__host__ __device__ inline int unit_of_block(const split_plan& p, bool turns, int b) {
    const int units = p.whole + p.cut * p.parts, x = b & 7, at = b >> 3;
    if (turns) {
        const int n = (at / 64 * 8 + x) * 64 + at % 64;
        return n < units ? n : -1;
    }
    // whole tiles in eight runs, then the parts
    const int from = (int)((int64_t)p.whole * x / 8), count = (int)((int64_t)p.whole * (x + 1) / 8) - from;
    const int parts = units - p.whole, pfrom = (int)((int64_t)parts * x / 8), pcount = (int)((int64_t)parts * (x + 1) / 8) - pfrom;
    if (at >= count + pcount) return -1;
    return at < count ? from + at : p.whole + pfrom + (at - count);
}
// blocks of a launch that reach every one of up to `units` units
inline int64_t blocks_of(int64_t units, bool turns) { return turns ? (units + 511) / 512 * 512 : (units + 7) / 8 * 8 + 8; }

}  // namespace moe355
