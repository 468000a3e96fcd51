// Rows of an embedding table for token ids, and the table's gradient by sorted tokens.
#include "grad_common.hpp"
#include "lanes.hpp"
#include "step_rules.hpp"
#include "ticket.hpp"

namespace moe355 {
namespace {

constexpr int EMBED_THREADS = 256;
constexpr int64_t EMBED_MAX_GRID = 1 << 22;
constexpr int FEW_TOKENS = 1024, FEW_NARROW = 2048;    // tokens that need no sorting, and of at most FEW_ELEMENTS together
constexpr int64_t FEW_ELEMENTS = (int64_t)5 << 20;
constexpr int FEW_RUN = 16;                            // rows of one token that one block adds up
constexpr int RANK_THREADS = 1024, RANK_CHUNK = 4096, RANK_ALONE = 8192, MERGE_WAYS = 32, MERGE_AT_ONCE = 8;
constexpr int SUM_AT_ONCE = 8;                         // sorted rows that a thread has on their way
constexpr int JOIN_TWICE = 32;                         // sums of a token's runs from which on they are joined in groups first
constexpr uint32_t NO_ID = 0xFFFFFFFFu;                // of tokens outside the table: behind the others

// A thread's W columns of a row of d.  TAIL: d need not be a multiple of W; the last thread then reads the last W columns, and `skip` of them are its neighbour's,
// which it leaves alone.  A thread behind the row reads what the last one does and writes nothing.  So no load has a condition: one in a branch of its own waits
// for the one before it.
template <int W, bool TAIL>
struct piece {
    int nominal, at, skip;
    bool in_row;
    __device__ piece(int thread, int d) {
        const int last = (d - 1) / W;
        in_row = thread <= last;
        nominal = (in_row ? thread : last) * W;
        at = TAIL && nominal + W > d ? (d > W ? d - W : 0) : nominal;
        skip = nominal - at;
    }
};
// They lie in memory at any element.  PAST: past the caches
typedef u32x2 __attribute__((aligned(2))) u32x2_odd;
template <bool BF16, int W, bool TAIL>
struct columns {
    static constexpr int WORDS = W * (BF16 ? 2 : 4) / 4;
    uint32_t w[WORDS];
    template <bool PAST = false>
    __device__ void load(const void* row, int i, int d) {
        const char* const at = static_cast<const char*>(row) + (int64_t)i * (BF16 ? 2 : 4);
        if (!TAIL || d >= W) {
            if (WORDS == 4) {
                const u32x4_any* const p = reinterpret_cast<const u32x4_any*>(at);
                const u32x4 v = PAST ? __builtin_nontemporal_load(p) : *p;
#pragma unroll
                for (int j = 0; j < WORDS; ++j) w[j] = v[j & 3];
            } else {
                const u32x2_odd* const p = reinterpret_cast<const u32x2_odd*>(at);
                const u32x2 v = PAST ? __builtin_nontemporal_load(p) : *p;
#pragma unroll
                for (int j = 0; j < WORDS; ++j) w[j] = v[j & 1];
            }
        } else {                               // (rows shorter than W)
#pragma unroll
            for (int j = 0; j < WORDS; ++j) w[j] = 0;
            for (int j = 0; j < d; ++j) {
                const uint32_t b = BF16 ? (uint32_t) static_cast<const uint16_t*>(row)[i + j] << (j & 1) * 16 : static_cast<const uint32_t*>(row)[i + j];
#pragma unroll
                for (int k = 0; k < WORDS; ++k) w[k] |= k == (BF16 ? j / 2 : j) ? b : 0;
            }
        }
    }
    __device__ void here() {                   // (a load is not put off into the branch that uses it)
#pragma unroll
        for (int j = 0; j < WORDS; ++j) asm volatile("" : "+v"(w[j]));
    }
    __device__ float at(int j) const { return BF16 ? (j & 1 ? bf16hi(w[j >> 1]) : bf16lo(w[j >> 1])) : __uint_as_float(w[j % WORDS]); }
};
template <class V>
__device__ inline void store_any(const V& v, void* at) {
    typedef V __attribute__((aligned(2))) any;
    __builtin_nontemporal_store(v, static_cast<any*>(at));
}
template <bool BF16, int W, bool TAIL>
__device__ inline void store_columns(void* row, const piece<W, TAIL>& p, int d, const float (&v)[W]) {
    if (!p.in_row) return;
    char* const at = static_cast<char*>(row) + (int64_t)p.at * (BF16 ? 2 : 4);
    if (!TAIL || (p.skip == 0 && d >= W)) {
        if constexpr (BF16 && W == 8) store_any(u32x4{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7])}, at);
        else if constexpr (BF16) store_any(u32x2{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])}, at);
        else
#pragma unroll
            for (int h = 0; h < W; h += 4)
                store_any(u32x4{__float_as_uint(v[h]), __float_as_uint(v[h + 1]), __float_as_uint(v[h + 2]), __float_as_uint(v[h + 3])}, at + h * 4);
    } else {
#pragma unroll
        for (int j = 0; j < W; ++j)
            if (j >= p.skip && j < d) store1<BF16>(row, p.at + j, v[j]);
    }
}
// Columns of a thread: 16 bytes of the wider of the two rows
constexpr int width_of(bool a_bf16, bool b_bf16) { return a_bf16 && b_bf16 ? 8 : 4; }

struct embed_args {
    const int32_t* ids;
    const void* table;
    void* y;
    int64_t T, ld, ld_y, first;
    int V, d, parts;
    float scale;
};
// y[t] = scale table[ids[t]]: a copy.  A block has a part of the columns of AT_ONCE tokens, all on their way at a time; rows of the table are kept in the caches,
// tokens come again, y is written past them.  Bound by memory, mostly y: 32768 x 7168 bf16 of 12 thousand different tokens 132 us, 4.8 TB/s
// with each row read once (a token after another 235); 1 x 4096 2.1 us, two loads one behind the other and a store.
template <bool BF16, bool OUT_BF16, bool TAIL>
__global__ __launch_bounds__(EMBED_THREADS) void embed_kernel(const embed_args a) {
    constexpr int W = width_of(BF16, OUT_BF16), AT_ONCE = 4;
    const int64_t b = a.first + blockIdx.x, t0 = b / a.parts * AT_ONCE;
    const piece<W, TAIL> p((int)(b % a.parts) * blockDim.x + threadIdx.x, a.d);
    columns<BF16, W, TAIL> v[AT_ONCE];
    bool there[AT_ONCE];
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
        const int id = a.ids[t0 + u < a.T ? t0 + u : a.T - 1];
        there[u] = (uint32_t)id < (uint32_t)a.V;
        v[u].load(row_of<BF16>(a.table, (there[u] ? id : 0) * a.ld), p.at, a.d);
    }
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
        if (t0 + u >= a.T) return;
        float y[W];
#pragma unroll
        for (int j = 0; j < W; ++j) y[j] = there[u] ? v[u].at(j) * a.scale : 0.f;
        store_columns<OUT_BF16>(row_of<OUT_BF16>(a.y, (t0 + u) * a.ld_y), p, a.d, y);
    }
}

struct embed_back_args {
    const void* dy;
    const int32_t* ids;
    void* dtable;
    int64_t ld, ld_grad, T, first;
    int V, d, parts, threads;                  // (threads of the blocks that add up, each W columns)
    float scale;
    int zero_rows, zero_blocks;                // rows that a block clears; 0: dtable is added to
    // few tokens: the blocks that add up; rows of many occurrences in parts
    int64_t sum_blocks;
    float* partial;                            // [slots][width]
    int width;
    int32_t* tickets;
    // sorted tokens in runs of `run`
    const uint64_t* keys;
    int run, fold;
};
__device__ inline uint32_t id_of(uint64_t key) { return (uint32_t)(key >> 32); }

// Rows of tokens that do not occur: each block looks through the batch for those of its rows that do, and clears the others past the caches (into them 8 % slower).
// Bound by the writes: 1.72 GB beside 32768 ids' ranks 320 us, 5.4 TB/s.
template <bool OUT_BF16, bool TAIL>
__device__ inline void clear_absent(const embed_back_args& a, int64_t v0, int rows, const uint32_t* seen) {
    constexpr int W = OUT_BF16 ? 8 : 4;
    const int pieces = (a.d + W - 1) / W, row_step = blockDim.x / pieces, at_step = blockDim.x % pieces;
    int row = threadIdx.x / pieces, at = threadIdx.x % pieces;
    const float none[W] = {};
    while (row < rows) {
        if (!(seen[row / 32] >> row % 32 & 1)) store_columns<OUT_BF16, W, TAIL>(row_of<OUT_BF16>(a.dtable, (v0 + row) * a.ld_grad), piece<W, TAIL>(at, a.d), a.d, none);
        row += row_step;
        at += at_step;
        if (at >= pieces) at -= pieces, ++row;
    }
}
template <bool OUT_BF16>
__device__ inline void clear_rows(const embed_back_args& a, int block, uint32_t* seen) {
    const int v0 = block * a.zero_rows, rows = min(a.zero_rows, a.V - v0);
    for (int i = threadIdx.x; i < (rows + 31) / 32; i += blockDim.x) seen[i] = 0;
    __syncthreads();
    constexpr int AT_ONCE = 8;
    for (int64_t t = threadIdx.x; t < a.T; t += AT_ONCE * blockDim.x) {
        int id[AT_ONCE];
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) id[u] = a.ids[t + u * blockDim.x < a.T ? t + u * blockDim.x : t];
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
            const uint32_t at = (uint32_t)id[u] - (uint32_t)v0;                // (ids in front of v0 wrap to large numbers)
            if (at < (uint32_t)rows && id[u] >= 0 && !(seen[at / 32] >> at % 32 & 1)) atomicOr(&seen[at / 32], 1u << at % 32);     // (once for a frequent token)
        }
    }
    __syncthreads();
    if (a.d % 8) clear_absent<OUT_BF16, true>(a, v0, rows, seen);
    else clear_absent<OUT_BF16, false>(a, v0, rows, seen);
}

// A token's finished sum into its row
template <bool OUT_BF16, bool ADD, int W, bool TAIL>
__device__ inline void finish(const embed_back_args& a, uint32_t id, const piece<W, TAIL>& p, const columns<OUT_BF16, W, TAIL>& was, const float (&sum)[W]) {
    float g[W];
#pragma unroll
    for (int j = 0; j < W; ++j) g[j] = ADD ? fmaf(sum[j], a.scale, was.at(j)) : sum[j] * a.scale;
    store_columns<OUT_BF16>(row_of<OUT_BF16>(a.dtable, id * a.ld_grad), p, a.d, g);
}
// A thread's sums in the workspace, past the L2 caches of an XCD: another block will read them
template <int W>
__device__ inline void store_partial(float* at, const float (&sum)[W]) {
#pragma unroll
    for (int j = 0; j < W; j += 2)
        __hip_atomic_store(reinterpret_cast<uint64_t*>(at) + j / 2, (uint64_t)__float_as_uint(sum[j + 1]) << 32 | __float_as_uint(sum[j]), __ATOMIC_RELAXED,
                           __HIP_MEMORY_SCOPE_AGENT);
}
// The sum of n of them, at(q)
template <int W, class At>
__device__ inline void join_partials(int64_t n, At at, float (&total)[W]) {
    constexpr int AT_ONCE = JOIN_AT_ONCE;
#pragma unroll
    for (int j = 0; j < W; ++j) total[j] = 0.f;
    for (int64_t q = 0; q < n; q += AT_ONCE) {
        uint64_t v[AT_ONCE][W / 2];
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
            const uint64_t* const theirs = reinterpret_cast<const uint64_t*>(at(q + u < n ? q + u : n - 1));
#pragma unroll
            for (int j = 0; j < W / 2; ++j) v[u][j] = __hip_atomic_load(theirs + j, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u)
#pragma unroll
            for (int j = 0; j < W; ++j) total[j] += q + u < n ? __uint_as_float((uint32_t)(v[u][j / 2] >> j % 2 * 32)) : 0.f;
    }
}

// Few tokens in one launch, without sorting: a block looks through the ids for the others of its token, and has work if FEW_RUN divides the number of those in
// front of it; the runs of a frequent token are joined by the last of their blocks.  Bound by a chain of its token's id, all ids, the counts, the rows and the
// result, five trips to memory: 777 x 2177 f32 added to 10.5 us for 14 MB, sorted 15.2.  A block looks through T ids, so only for few and narrow rows: 1000 x 7168
// 19.0 us, sorted 20.5; 1500 x 1024 bf16 10.7 and 13.8, 1100 x 4096 14.9 and 16.0, 1100 x 7168 20.8 and 21.0, 2000 x 4096 bf16 19.6 and 17.2.  A form for 2048 tokens
// of its own: with that one the 1000 x 7168 take 21.2.
template <bool BF16, bool OUT_BF16, bool ADD, bool TAIL, int TOKENS>
__global__ __launch_bounds__(EMBED_THREADS) void embed_few_kernel(const embed_back_args a) {
    constexpr int W = width_of(BF16, OUT_BF16), MASKS = TOKENS / 64, AT_ONCE = 8;
    __shared__ uint64_t s_same[MASKS];
    __shared__ uint16_t s_list[TOKENS];
    __shared__ uint32_t s_seen[CLEAR_MOST / 32];
    __shared__ int32_t s_last;
    if (blockIdx.x >= a.sum_blocks) {
        if (!ADD) clear_rows<OUT_BF16>(a, (int)(blockIdx.x - a.sum_blocks), s_seen);
        return;
    }
    const int t = (int)(blockIdx.x / a.parts), part = (int)(blockIdx.x % a.parts), T = (int)a.T;
    const piece<W, TAIL> p(part * a.threads + threadIdx.x, a.d);
    const int id = a.ids[t];
    if ((uint32_t)id >= (uint32_t)a.V) return;
    for (int k0 = threadIdx.x; k0 < TOKENS; k0 += 4 * blockDim.x) {    // (a wave has 64 consecutive ones)
        int other[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) other[u] = a.ids[min(k0 + u * (int)blockDim.x, T - 1)];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int k = k0 + u * blockDim.x;
            const uint64_t same = __ballot(k < T && other[u] == id);
            if ((threadIdx.x & 63) == 0 && k < TOKENS) s_same[k / 64] = same;
        }
    }
    __syncthreads();
    // a lane has 64 tokens: how many occurrences there are up to them
    const int lane = threadIdx.x & 63;
    const uint64_t mine = lane < MASKS ? s_same[lane] : 0;
    const int upto = wave_scan(__popcll(mine)), total = __builtin_amdgcn_readlane(upto, 63);
    const int ahead = __builtin_amdgcn_readlane(upto - __popcll(mine >> t % 64), t / 64);
    if (ahead % FEW_RUN) return;
    const int group = __builtin_ctzll(__ballot(mine != 0)), first = group * 64 + __builtin_ctzll(s_same[group]);
    // the occurrences in their order
    for (int k = threadIdx.x; k < TOKENS; k += blockDim.x) {
        const uint64_t same = s_same[k / 64];
        if (same >> lane & 1)
            s_list[__builtin_amdgcn_readlane(upto, k / 64) - __popcll(same >> lane)] = (uint16_t)k;
    }
    __syncthreads();
    const bool whole = total <= FEW_RUN;
    const int left = min(FEW_RUN, total - ahead);
    columns<OUT_BF16, W, TAIL> was;
    if (ADD && whole) was.load(row_of<OUT_BF16>(a.dtable, id * a.ld_grad), p.at, a.d);
    float sum[W] = {};
    for (int q = 0; q < left; q += AT_ONCE) {
        columns<BF16, W, TAIL> v[AT_ONCE];
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u)
            v[u].load(row_of<BF16>(a.dy, __builtin_amdgcn_readfirstlane(s_list[ahead + min(q + u, left - 1)]) * a.ld), p.at, a.d);
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u)
#pragma unroll
            for (int j = 0; j < W; ++j) sum[j] += q + u < left ? v[u].at(j) : 0.f;
    }
    if (whole) {
        finish<OUT_BF16, ADD>(a, id, p, was, sum);
        return;
    }
    const int runs = (total + FEW_RUN - 1) / FEW_RUN;
    if (p.in_row) store_partial(a.partial + (int64_t)t * a.width + p.nominal, sum);
    if (!last_block(a.tickets + first * a.parts + part, runs, s_last)) return;
    if (ADD) was.load(row_of<OUT_BF16>(a.dtable, id * a.ld_grad), p.at, a.d);
    join_partials(runs, [&](int64_t q) { return a.partial + (int64_t)s_list[q * FEW_RUN] * a.width + p.nominal; }, sum);
    finish<OUT_BF16, ADD>(a, id, p, was, sum);
}

// Keys (id, token) in ascending order: tokens of one id stand together in the order of the batch.  A token's place in its chunk is the number of tokens there that
// come before it: TOKENS of them to a block, the chunk's ids dealt to the 16 waves and to 64 / TOKENS groups of lanes.  Two instructions for 64 comparisons on all
// CUs take less than a sorting network on few: 4096 tokens 5.3 us, the network 17.  The other blocks of the launch clear rows.
template <bool OUT_BF16, int TOKENS>
__global__ __launch_bounds__(RANK_THREADS, 8) void rank_tokens_kernel(const embed_back_args a, const int32_t* __restrict__ ids, int blocks, int chunk,
                                                                      uint64_t* __restrict__ out) {
    constexpr int WAVES = RANK_THREADS / 64, SLICES = 64 / TOKENS, PAD = 4, LOADS = RANK_ALONE / RANK_THREADS;
    constexpr uint32_t LAST = 0x7FFFFFFFu;     // in place of ids outside the table; one more is a number still
    static_assert(RANK_ALONE >= RANK_CHUNK && RANK_ALONE % (RANK_THREADS * SLICES) == 0 && RANK_ALONE >= CLEAR_MOST / 32, "whole groups of ids for each lane");
    __shared__ u32x4 s_ids[(RANK_ALONE + WAVES * SLICES * PAD) / 4];
    __shared__ uint32_t s_rank[WAVES][TOKENS];
    if ((int)blockIdx.x >= blocks) {
        clear_rows<OUT_BF16>(a, blockIdx.x - blocks, reinterpret_cast<uint32_t*>(s_ids));
        return;
    }
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int T = (int)a.T, t0 = blockIdx.x * TOKENS, t = t0 + lane % TOKENS, begin = t0 / chunk * chunk, end = min(begin + chunk, T);
    const uint32_t V = (uint32_t)a.V;
    auto known = [&](int j) {
        const uint32_t id = j < end ? (uint32_t)ids[j] : LAST;
        return id < V ? id : LAST;
    };
    const int each = ((end - begin + WAVES * SLICES - 1) / (WAVES * SLICES) + TOKENS - 1) / TOKENS * TOKENS, from = begin + wave * SLICES * each;
    uint32_t theirs[LOADS];                    // (all on their way at a time)
#pragma unroll
    for (int g = 0; g < LOADS; ++g) theirs[g] = known(g * 64 + lane < SLICES * each ? from + g * 64 + lane : end);
    const uint32_t id = known(t);
    uint32_t* const mine = reinterpret_cast<uint32_t*>(s_ids) + wave * SLICES * (each + PAD);
#pragma unroll
    for (int g = 0; g < LOADS; ++g) {
        const int j = g * 64 + lane;
        if (j < SLICES * each) mine[j + j / each * PAD] = theirs[g];
    }
    uint32_t rank = 0;
    const int slice = lane / TOKENS;
    for (int g = 0; g < each; g += TOKENS) {   // (a wave reads what it has written)
        const u32x4* const of = reinterpret_cast<const u32x4*>(mine + slice * (each + PAD) + g);
        const int j0 = from + slice * each + g;
        const uint32_t bound = j0 < t0 ? id + 1 : j0 > t0 ? id : 0;            // in front of this block's tokens an equal id comes before
#pragma unroll 4
        for (int q = 0; q < TOKENS / 4; ++q)
#pragma unroll
            for (int k = 0; k < 4; ++k) rank += of[q][k] < bound;
    }
    if (wave == 0 && lane < TOKENS) {          // this block's own
        for (int k = 0; k < TOKENS; ++k) {
            const uint32_t o = (uint32_t)__builtin_amdgcn_readlane((int)id, k);
            rank += (int)(o < id) | ((int)(o == id) & (int)(k < lane));
        }
    }
#pragma unroll
    for (int o = TOKENS; o < 64; o *= 2) rank += (uint32_t)__shfl_xor((int)rank, o);
    if (lane < TOKENS) s_rank[wave][lane] = rank;
    __syncthreads();
    if (wave || lane >= TOKENS || t >= T) return;
#pragma unroll
    for (int w = 1; w < WAVES; ++w) rank += s_rank[w][lane];
    out[begin + rank] = (uint64_t)(id == LAST ? NO_ID : id) << 32 | (uint32_t)t;
}

// Sorted runs of `run` keys, MERGE_WAYS of them to one: a key's place is the number of keys in the runs that are smaller (no two are equal).  The searches of
// eight runs go side by side, each step waits for the memory once: 12 steps of 0.5 us, 32768 tokens 7.9 us.
__global__ __launch_bounds__(EMBED_THREADS) void merge_tokens_kernel(const uint64_t* __restrict__ keys, int T, int run, uint64_t* __restrict__ out) {
    const int i = blockIdx.x * EMBED_THREADS + threadIdx.x;
    if (i >= T) return;
    const uint64_t mine = keys[i];
    const int first = i / (run * MERGE_WAYS) * (run * MERGE_WAYS);
    int place = first;
    for (int at = first; at < T && at < first + run * MERGE_WAYS; at += run * MERGE_AT_ONCE) {
        int below[MERGE_AT_ONCE] = {};         // of each run
        for (int step = run; step > 0; step /= 2) {            // (run: a power of two)
            uint64_t there[MERGE_AT_ONCE];
#pragma unroll
            for (int u = 0; u < MERGE_AT_ONCE; ++u) there[u] = keys[min(at + u * run + below[u] + step, T) - 1];
#pragma unroll
            for (int u = 0; u < MERGE_AT_ONCE; ++u) {          // (no branches: the reads go out together)
                const int to = below[u] + step;
                below[u] = (int)(to <= run) & (int)(at + u * run + to <= T) & (int)(there[u] < mine) ? to : below[u];
            }
        }
#pragma unroll
        for (int u = 0; u < MERGE_AT_ONCE; ++u) place += below[u];
    }
    out[place] = mine;
}

// A run of sorted tokens and a part of the columns to a block, whatever the tokens' frequencies.  A token whose rows all lie in the run is finished here; of one
// that goes on from the run before, or into the next, there are sums in several runs, places 2 run and 2 run + 1, which the last of their blocks joins; of many
// runs the last of each group first (4096 x 5120 bf16 of one token added to f32 34 us, half of them 37; joined by one block 55 and 41).
// Bound by rows of dy that lie anywhere, SUM_AT_ONCE of a thread on their way: 32768 x 7168 bf16 of 12 thousand different tokens 143 us, 4.5 TB/s; by its chain (keys, rows,
// partial sums, ticket, join) where a block has eight rows: 4096 x 5120 bf16 added to f32 30 us.
template <bool BF16, bool OUT_BF16, bool ADD, bool TAIL>
__global__ __launch_bounds__(EMBED_THREADS) void embed_sum_kernel(const embed_back_args a) {
    constexpr int W = width_of(BF16, OUT_BF16), AT_ONCE = SUM_AT_ONCE;
    __shared__ int32_t s_last;
    const int64_t r = blockIdx.x / a.parts, begin = r * a.run, end = begin + a.run < a.T ? begin + a.run : a.T;
    const int part = (int)(blockIdx.x % a.parts), lane = threadIdx.x & 63;
    const piece<W, TAIL> p(part * a.threads + threadIdx.x, a.d);
    float sum[W] = {}, older[W] = {}, head[W] = {};            // (of the present token: rows since the last fold, those before it)
    const uint32_t first_id = id_of(a.keys[begin]), last_id = id_of(a.keys[end - 1]);
    const bool from_before = begin > 0 && first_id != NO_ID && id_of(a.keys[begin - 1]) == first_id;
    const bool goes_on = end < a.T && last_id != NO_ID && id_of(a.keys[end]) == last_id;
    bool open = from_before;                   // the present token began in an earlier run
    for (int64_t k0 = begin; k0 < end; k0 += 64) {
        const int rows = (int)(end - k0 < 64 ? end - k0 : 64);
        const uint64_t key = lane < rows ? a.keys[k0 + lane] : ~(uint64_t)0;
        const uint32_t id = id_of(key), token = (uint32_t)key, next = lane < rows && k0 + lane + 1 < a.T ? id_of(a.keys[k0 + lane + 1]) : NO_ID;
        const int known = __popcll(__ballot(id != NO_ID));     // (the others are the last ones)
        const uint64_t ends = __ballot(id != NO_ID && id != next);
        for (int q = 0; q < known; q += AT_ONCE) {
            columns<BF16, W, TAIL> v[AT_ONCE];
            columns<OUT_BF16, W, TAIL> was[AT_ONCE];
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                const int k = min(q + u, known - 1);
                v[u].template load<true>(row_of<BF16>(a.dy, (int64_t)(uint32_t)__builtin_amdgcn_readlane(token, k) * a.ld), p.at, a.d);
                if (ADD) {                     // (of other rows than a token's last one, something near by)
                    const bool wanted = ends >> k & 1;
                    const void* const row = row_of<OUT_BF16>(a.dtable, (int64_t)(uint32_t)__builtin_amdgcn_readlane(id, k) * a.ld_grad);
                    was[u].load(wanted ? row : a.keys, wanted ? p.at : lane * W, a.d);
                }
            }
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
#pragma unroll
                for (int j = 0; j < W; ++j) sum[j] += q + u < known ? v[u].at(j) : 0.f;
                if (ADD) was[u].here();
                if (!(ends >> (q + u) & 1)) continue;          // (no bits from `known` on)
#pragma unroll
                for (int j = 0; j < W; ++j) sum[j] += older[j];
                if (open) {
#pragma unroll
                    for (int j = 0; j < W; ++j) head[j] = sum[j];
                } else {
                    finish<OUT_BF16, ADD>(a, (uint32_t)__builtin_amdgcn_readlane(id, q + u), p, was[u], sum);
                }
                open = false;
#pragma unroll
                for (int j = 0; j < W; ++j) sum[j] = older[j] = 0.f;
            }
        }
        if (((k0 - begin + 64) & (a.fold - 1)) == 0) {
#pragma unroll
            for (int j = 0; j < W; ++j) {
                older[j] += sum[j];
                sum[j] = 0.f;
            }
        }
    }
#pragma unroll
    for (int j = 0; j < W; ++j) sum[j] += older[j];
    auto place = [&](int64_t n) { return a.partial + n * a.width + p.nominal; };
    if (from_before && !open && p.in_row) store_partial(place(2 * r), head);
    if (goes_on && p.in_row) store_partial(place(open ? 2 * r : 2 * r + 1), sum);

    // runs that this token goes through: from the one in which it begins to the one in which it ends, 64 looked at together
    auto join = [&](uint32_t id, bool before, bool behind) {
        int64_t from = r, to = r;
        while (before) {
            const int64_t q = from - 1 - lane; // whose last token is this one
            const uint64_t same = __ballot(q >= 0 && id_of(a.keys[q >= 0 ? (q + 1) * a.run - 1 : 0]) == id);
            from -= __popcll(same);
            before = !~same;
        }
        const int64_t runs = (a.T + a.run - 1) / a.run;
        while (behind) {
            const int64_t q = to + 1 + lane;   // whose first token is this one
            const uint64_t same = __ballot(q < runs && id_of(a.keys[q < runs ? q * a.run : 0]) == id);
            to += __popcll(same);
            behind = !~same;
        }
        auto sum_of = [&](int64_t q) { return place(q == from ? 2 * q + 1 : 2 * q); };         // of run q
        int64_t all = to - from + 1;
        int group = 1;
        float total[W];
        if (all >= JOIN_TWICE) {
            group = runs_of_group(all);
            const int64_t groups = all / group, mine = (r - from) / group < groups ? (r - from) / group : groups - 1, first = from + mine * group;
            const int64_t n = mine == groups - 1 ? to - first + 1 : group;
            // (the ticket of a run in which no other token begins)
            if (!last_block(a.tickets + (first + 1) * a.parts + part, (int)n, s_last)) return;
            join_partials(n, [&](int64_t q) { return sum_of(first + q); }, total);
            if (p.in_row) store_partial(sum_of(first), total);
            all = groups;
        }
        if (!last_block(a.tickets + from * a.parts + part, (int)all, s_last)) return;
        columns<OUT_BF16, W, TAIL> was;
        if (ADD) was.load(row_of<OUT_BF16>(a.dtable, id * a.ld_grad), p.at, a.d);
        join_partials(all, [&](int64_t q) { return sum_of(from + q * group); }, total);
        finish<OUT_BF16, ADD>(a, id, p, was, total);
    };
    const bool through = from_before && goes_on && first_id == last_id;
    if (from_before) join(first_id, true, through);
    if (goes_on && !through) join(last_id, false, true);
}

// blocks 0 .. n-1 in launches that a grid holds
template <class Kernel, class Args>
hipError_t launch_blocks(hipStream_t s, Kernel kernel, Args a, int64_t n, int threads) {
    for (a.first = 0; a.first < n; a.first += EMBED_MAX_GRID)
        hipLaunchKernelGGL(kernel, dim3((unsigned)(n - a.first < EMBED_MAX_GRID ? n - a.first : EMBED_MAX_GRID)), dim3(threads), 0, s, a);
    return hipGetLastError();
}
// Parts of a row of `pieces` threads and their blocks' threads
void cut_row(int pieces, int& parts, int& threads) {
    parts = (pieces + EMBED_THREADS - 1) / EMBED_THREADS;
    threads = ((pieces + parts - 1) / parts + 63) / 64 * 64;
}

template <bool BF16, bool OUT_BF16, bool ADD>
hipError_t launch_embed_sums(moe_ctx* c, embed_back_args a) {
    const int pieces = (a.d + width_of(BF16, OUT_BF16) - 1) / width_of(BF16, OUT_BF16);
    cut_row(pieces, a.parts, a.threads);
    a.width = (a.d + 7) / 8 * 8;
    if (!ADD) {
        const clear_plan clear = clearing(a.V, a.T, (int64_t)a.d * (OUT_BF16 ? 2 : 4));
        a.zero_rows = clear.rows;
        a.zero_blocks = clear.blocks;
    }
    const bool few = a.T <= FEW_TOKENS;
    if ((few || (a.T <= FEW_NARROW && a.T * a.d <= FEW_ELEMENTS)) && a.T * a.parts <= GRAD_TICKETS && a.T * a.width * sizeof(float) <= GRAD_WS_BYTES) {
        a.sum_blocks = a.T * a.parts;
        a.partial = static_cast<float*>(c->grad_ws);
        a.tickets = c->grad_tickets;
        const unsigned grid = (unsigned)(a.sum_blocks + a.zero_blocks);
        if (!grid) return hipSuccess;
        auto launch = [&](auto kernel) { kernel<<<grid, a.threads, 0, c->stream>>>(a); };
        if (a.d % width_of(BF16, OUT_BF16)) launch(few ? embed_few_kernel<BF16, OUT_BF16, ADD, true, FEW_TOKENS> : embed_few_kernel<BF16, OUT_BF16, ADD, true, FEW_NARROW>);
        else launch(few ? embed_few_kernel<BF16, OUT_BF16, ADD, false, FEW_TOKENS> : embed_few_kernel<BF16, OUT_BF16, ADD, false, FEW_NARROW>);
        return hipGetLastError();
    }
    uint64_t *keys = static_cast<uint64_t*>(c->grad_ws), *other = keys + a.T;
    const bool alone = a.T <= RANK_ALONE;
    const int chunk = alone ? RANK_ALONE : RANK_CHUNK, tokens = alone ? 16 : 64, blocks = (int)((a.T + tokens - 1) / tokens);
    if (alone) rank_tokens_kernel<OUT_BF16, 16><<<blocks + a.zero_blocks, RANK_THREADS, 0, c->stream>>>(a, a.ids, blocks, chunk, keys);
    else rank_tokens_kernel<OUT_BF16, 64><<<blocks + a.zero_blocks, RANK_THREADS, 0, c->stream>>>(a, a.ids, blocks, chunk, keys);
    for (int64_t run = chunk; run < a.T; run *= MERGE_WAYS) {
        merge_tokens_kernel<<<(unsigned)((a.T + EMBED_THREADS - 1) / EMBED_THREADS), EMBED_THREADS, 0, c->stream>>>(keys, (int)a.T, (int)run, other);
        uint64_t* const sorted = other;
        other = keys;
        keys = sorted;
    }
    a.keys = keys;
    a.partial = reinterpret_cast<float*>(static_cast<uint64_t*>(c->grad_ws) + (2 * a.T + 1) / 2 * 2);
    const int64_t room = (GRAD_WS_BYTES - 16 * (a.T + 1)) / (2 * sizeof(float) * a.width);
    a.run = (int)run_of_tokens(a.T, a.parts, width_of(BF16, OUT_BF16), room, GRAD_TICKETS);
    a.fold = rows_of_fold(a.run);
    a.tickets = c->grad_tickets;
    const unsigned grid = (unsigned)((a.T + a.run - 1) / a.run * a.parts);
    if (a.d % width_of(BF16, OUT_BF16)) embed_sum_kernel<BF16, OUT_BF16, ADD, true><<<grid, a.threads, 0, c->stream>>>(a);
    else embed_sum_kernel<BF16, OUT_BF16, ADD, false><<<grid, a.threads, 0, c->stream>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_embed(hipStream_t s, const int32_t* ids, int64_t T, const void* table, int32_t V, int32_t d, int64_t ld, int32_t dtype, float scale,
                        void* y, int64_t ld_y, int32_t out_dtype) {
    const bool bf16 = dtype == MOE_BF16, out_bf16 = out_dtype == MOE_BF16;
    const int W = width_of(bf16, out_bf16);
    int parts, threads;
    cut_row((d + W - 1) / W, parts, threads);
    const embed_args a{ids, table, y, T, ld, ld_y, 0, V, d, parts, scale};
    const int64_t n = (T + 3) / 4 * parts;
    auto launch = [&](auto kernel, auto tail_kernel) { return d % W ? launch_blocks(s, tail_kernel, a, n, threads) : launch_blocks(s, kernel, a, n, threads); };
    if (bf16) return out_bf16 ? launch(embed_kernel<true, true, false>, embed_kernel<true, true, true>) : launch(embed_kernel<true, false, false>, embed_kernel<true, false, true>);
    return out_bf16 ? launch(embed_kernel<false, true, false>, embed_kernel<false, true, true>) : launch(embed_kernel<false, false, false>, embed_kernel<false, false, true>);
}

hipError_t launch_embed_backward(moe_ctx* c, const void* dy, const int32_t* ids, int64_t T, int32_t V, int32_t d, int64_t ld, int32_t dtype, float scale,
                                 int32_t accumulate, void* dtable, int64_t ld_grad, int32_t grad_dtype) {
    embed_back_args a{};
    a.dy = dy;
    a.ids = ids;
    a.dtable = dtable;
    a.ld = ld;
    a.ld_grad = ld_grad;
    a.T = T;
    a.V = V;
    a.d = d;
    a.scale = scale;
    if (dtype == MOE_BF16) {
        if (grad_dtype == MOE_BF16) return accumulate ? launch_embed_sums<true, true, true>(c, a) : launch_embed_sums<true, true, false>(c, a);
        return accumulate ? launch_embed_sums<true, false, true>(c, a) : launch_embed_sums<true, false, false>(c, a);
    }
    if (grad_dtype == MOE_BF16) return accumulate ? launch_embed_sums<false, true, true>(c, a) : launch_embed_sums<false, true, false>(c, a);
    return accumulate ? launch_embed_sums<false, false, true>(c, a) : launch_embed_sums<false, false, false>(c, a);
}

}  // namespace moe355
