// How rows of logits are dealt to blocks by token_logp.hip.  Host and device.
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

}  // namespace moe355
