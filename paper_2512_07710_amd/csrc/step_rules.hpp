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

// Sorted tokens in runs, one to a block (a part of the columns each), by embed.hip: eight tokens, more where there are enough blocks all the same, and where the
// workspace or the tickets would not hold the runs' sums.  room: runs that the workspace holds
constexpr int EMBED_BLOCKS = 512;              // that add up sorted tokens, about, of 2048 columns
inline int64_t run_of_tokens(int64_t T, int parts, int columns, int64_t room, int64_t tickets) {
    int64_t run = 8;
    while ((T + run - 1) / run > room || T / (2 * run) * parts * columns >= EMBED_BLOCKS * 8 || (T + run - 1) / run * parts > tickets) run *= 2;
    return run;
}
// Rows of a run that are added up before their sum joins the run's: 64, the rows that a block looks at together, or about the root of a long run.  One after another
// 2048 equal rows lose up to 500 half units of the last place, with no sign that evens it out, and so would every run
__host__ __device__ inline int rows_of_fold(int64_t run) {
    int fold = 64;
    while ((int64_t)fold * fold < run) fold *= 2;
    return fold;
}
// Runs of a token's sums that are joined first, of `all`: about the root
constexpr int JOIN_AT_ONCE = 8;                // sums that a thread has on their way
__host__ __device__ inline int runs_of_group(int64_t all) {
    int group = 1;
    while ((int64_t)group * group < all) group += JOIN_AT_ONCE;
    return group;
}

}  // namespace moe355
