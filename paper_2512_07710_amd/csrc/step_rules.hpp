// How rows of logits are dealt to blocks by token_logp.hip, and rows of an embedding's table by embed.hip.  Host and device.
#pragma once
#include <cstdint>

namespace moe355 {

// A part of a row of logits: its vectors begin .. end-1, and `rest` elements behind them (the row's last part has them)
struct row_part {
    int begin, end, place, rest;               // place: of the first element behind the vectors
    // The element that a thread has behind the vectors, or -1: it is a sum only where there is one, since V goes up to 2^31 - 1
    __host__ __device__ int behind(int thread) const { return thread < rest ? place + thread : -1; }
};
// V logits in vectors of N; part_vecs vectors to a part
__host__ __device__ inline row_part part_of_row(int V, int N, int part, int parts, int part_vecs) {
    const int vecs = V / N, first = part * part_vecs, begin = first < vecs ? first : vecs, end = part_vecs < vecs - begin ? begin + part_vecs : vecs;
    return row_part{begin, end, end * N, part == parts - 1 ? V % N : 0};
}

// Rows of a table of V that blocks of embed.hip clear where their token does not occur: few to a block, so that none ends late, but twice the bytes of the ids that
// it looks through (4096 x 4096 f32 of 131072: 64 rows 437 us, 16 386; 32768 x 7168 bf16 496 and 502)
constexpr int CLEAR_MOST = 4096;               // rows of a block at most
struct clear_plan {
    int rows, blocks;                          // (blocks: 2^19 at most)
};
inline clear_plan clearing(int V, int64_t T, int64_t row_bytes) {
    int64_t rows = ((int64_t)V + 8191) / 8192;
    const int64_t least = (8 * T + row_bytes - 1) / row_bytes;
    if (rows < least) rows = least;
    if (rows > CLEAR_MOST) rows = CLEAR_MOST;
    return clear_plan{(int)rows, (int)((V + rows - 1) / rows)};
}

}  // namespace moe355
