// Log-probabilities of given tokens, entropy and the most likely tokens of rows of logits; and the logits' gradient from those of the first two.
#include "softmax_rows.hpp"
#include "step_rules.hpp"
#include "ticket.hpp"

namespace moe355 {
namespace {

constexpr int LOGP_THREADS = 256;
constexpr int64_t LOGP_MAX_GRID = 1 << 22;
constexpr int FEW_THREADS = 512, PART_THREADS = 1024, FEW_ROWS_IN_PARTS = 32, MAX_PARTS = 64; // rows in parts: a block's threads, parts of a row at most
constexpr int MAX_SPLIT_ROWS = 128;            // (two parts or more in 256 blocks)
constexpr int AT_ONCE = 4;                     // vectors that a thread works on together
constexpr int RANKED = 64;                     // held logits that are ranked together
// groups of a block's threads, whose largest logits make the bound for n alternatives.  Ranking 128 takes 1.2 us more of a short call, but a third as many
// logits reach the bound of 64 of them (100 x 131072 bf16, n = 64 21.5 us, with 64 groups 48; 4096 rows n = 64 231 and 301, n = 20 206 and 202)
constexpr int FEW_TOP = 32, GROUPS_OF_FEW = 64, GROUPS_OF_MANY = 128;
__device__ inline bool many_groups(int threads, int n) { return threads > 256 && n > FEW_TOP; }
// logits that a block holds: several times what reaches the bound of a row of 131072 at random, and all parts' lists; 38 KB of LDS for each 512 threads of a CU's 2048
constexpr int top_held(int threads) { return threads > 256 ? 4160 : threads > 64 ? 1088 : 320; }
const float ABOVE_LOWEST = __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, LOWEST) - 1);

struct logp_args {
    const void* logits;
    int64_t ld, rows, first;                   // (first: of a launch)
    int V, m, n;
    const int32_t* ids;
    float inv_temp;
    float *logp, *entropy, *top_logp, *stats;
    int32_t* top_idx;
    // rows in parts (few rows): their number, a power of two, and length in vectors, the parts' sums and largest logits, the rows' tickets
    int parts, part_vecs;
    float* part_sums;                          // [rows][parts][3]
    uint64_t* part_tops;                       // [rows][parts][n]
    int32_t* tickets;
};

// (v - m) / temperature - log s to fp32's resolution: in fp64, the logits as they are
__device__ inline float logp_of(float v, const softmax_stats& st, double log_s, float inv_temp) {
    if (v <= LOWEST && st.s == st.s) return -INFINITY;
    return (float)(((double)v - (double)st.m) * (double)inv_temp - log_s);
}

// the next fp32 number (of +inf and NaN: NaN, which nothing reaches)
__device__ inline float next_above(float v) { return v != v ? v : __int_as_float(v == 0.f ? 1 : __float_as_int(v) + (v > 0.f ? 1 : -1)); }

// A logit and its place as one number: of two, the one that comes first among the alternatives is larger.  0 is below all
__device__ inline uint32_t ordered(float v) {
    const uint32_t b = __float_as_uint(v + 0.f);               // (-0 is equal to 0)
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ inline uint64_t key_of(float v, int i) { return (uint64_t)ordered(v) << 32 | (uint32_t)~i; }
__device__ inline float value_of(uint64_t key) {
    const uint32_t o = (uint32_t)(key >> 32);
    return __uint_as_float(o ^ (o >> 31 ? 0x80000000u : 0xFFFFFFFFu));
}
__device__ inline int index_of(uint64_t key) { return ~(int)(uint32_t)key; }

template <int THREADS>
struct top_scratch {
    static constexpr int HELD = top_held(THREADS);
    float groups[GROUPS_OF_MANY];
    float bound;
    int count;
    uint64_t least, tops[THREADS], held[HELD], best[LOGP_MAX_TOP], kept[LOGP_MAX_TOP];
};
// over the lanes of a group of SIZE consecutive ones, in each of them
template <int SIZE, class F>
__device__ inline int over_group(int v, F f) {
    static_assert(SIZE == 1 || SIZE == 2 || SIZE == 4 || SIZE == 8 || SIZE == 16, "lanes that one instruction reaches");
    if (SIZE > 1) v = f(v, __builtin_amdgcn_update_dpp(0, v, 0xB1, 0xf, 0xf, true));       // quad_perm 1 0 3 2
    if (SIZE > 2) v = f(v, __builtin_amdgcn_update_dpp(0, v, 0x4E, 0xf, 0xf, true));       // quad_perm 2 3 0 1
    if (SIZE > 4) v = f(v, __builtin_amdgcn_update_dpp(0, v, 0x141, 0xf, 0xf, true));      // row_half_mirror
    if (SIZE > 8) v = f(v, __builtin_amdgcn_update_dpp(0, v, 0x140, 0xf, 0xf, true));      // row_mirror
    return v;
}
// The n-th largest of the first GROUPS of s.groups: n different logits are not below it.  Called by the whole block, which has written groups.
template <int GROUPS, int THREADS>
__device__ inline float nth_of(int n, top_scratch<THREADS>& s) {
    constexpr int SIZE = THREADS / GROUPS;
    __syncthreads();
    const int i = threadIdx.x / SIZE, j0 = threadIdx.x % SIZE;
    const float mine = s.groups[i];
    int rank = 0;
#pragma unroll
    for (int j = 0; j < GROUPS; j += SIZE) {                   // (no branches: the reads go out together)
        const float v = s.groups[j + j0];
        rank += (int)(v > mine) | ((int)(v == mine) & (int)(j + j0 < i));
    }
    rank = over_group<SIZE>(rank, [](int x, int y) { return x + y; });
    if (rank == n - 1 && j0 == 0) s.bound = mine;
    __syncthreads();
    return s.bound;
}
// The same of the largest that groups of threads have
template <int GROUPS, int THREADS>
__device__ inline float nth_of_largest(float v, int n, top_scratch<THREADS>& s) {
    constexpr int SIZE = THREADS / GROUPS;
    const int g = over_group<SIZE>(__float_as_int(v), [](int x, int y) { return __float_as_int(fmaxf(__int_as_float(x), __int_as_float(y))); });
    if (threadIdx.x % SIZE == 0) s.groups[threadIdx.x / SIZE] = __int_as_float(g);
    return nth_of<GROUPS>(n, s);
}
template <int THREADS>
__device__ inline float bound_of(float v, int n, top_scratch<THREADS>& s) {
    if constexpr (THREADS > 256)
        if (__builtin_expect(many_groups(THREADS, n), 0)) return nth_of_largest<GROUPS_OF_MANY>(v, n, s);
    return nth_of_largest<GROUPS_OF_FEW>(v, n, s);
}
// what keys of logits from a bound on are not below; masked ones never are
__device__ inline uint64_t bound_key(float bound) { return (uint64_t)ordered(fmaxf(bound, ABOVE_LOWEST)) << 32; }
// (in any order: what is held in the end is the same)
template <int THREADS>
__device__ inline void hold(uint64_t key, top_scratch<THREADS>& s) {
    const int slot = atomicAdd(&s.count, 1);
    if (slot < s.HELD) s.held[slot] = key;
}
// The n first of the held ones in s.best, in order: SIZE threads count who is before one.  Called by the whole block, with a barrier before and behind it
template <int THREADS>
__device__ __forceinline__ void rank_held(int count, int n, top_scratch<THREADS>& s) {
    constexpr int SIZE = THREADS / RANKED;
    const int i = threadIdx.x / SIZE, j0 = threadIdx.x % SIZE;
    if (threadIdx.x < RANKED && (count & -RANKED) + (int)threadIdx.x >= count && count % RANKED)
        s.held[(count & -RANKED) + threadIdx.x] = 0;
    __syncthreads();
    for (int i0 = 0; i0 < count; i0 += RANKED) {
        const uint64_t mine = s.held[i0 + i];
        int rank = 0;
        for (int k0 = 0; k0 < count; k0 += RANKED)
#pragma unroll 8
            for (int k = 0; k < RANKED; k += SIZE) rank += s.held[k0 + k + j0] > mine;
        rank = over_group<SIZE>(rank, [](int x, int y) { return x + y; });
        if (j0 == 0 && rank < n && i0 + i < count) s.best[rank] = mine;
    }
}
// What of the held ones is not below `least`.  Returns how many.
template <int THREADS>
__device__ __forceinline__ int keep_held(int count, uint64_t least, top_scratch<THREADS>& s) {
    if (threadIdx.x == 0) s.count = 0;
    for (int k0 = 0; k0 < count; k0 += THREADS) {              // (into places that have been read)
        const uint64_t key = k0 + (int)threadIdx.x < count ? s.held[k0 + threadIdx.x] : 0;
        __syncthreads();
        if (key >= least) hold(key, s);
    }
    __syncthreads();
    return s.count;
}
// The n first of `count` held ones in s.best.  Returns their number.  Ranking takes count^2 / THREADS steps of a thread, so many are thinned first: by the bound
// of the groups' largest, which leaves little more than n as a rule, and by the n-th of the threads' largest, which leaves n threads' at most.
template <int THREADS>
__device__ __forceinline__ int first_held(int count, int n, top_scratch<THREADS>& s) {
    if (__builtin_expect(count > 2 * RANKED, 0)) {             // (a program that goes straight on is fetched sooner)
        uint64_t top = 0;
        for (int k = threadIdx.x; k < count; k += THREADS) top = s.held[k] > top ? s.held[k] : top;
        s.tops[threadIdx.x] = top;
        count = keep_held<THREADS>(count, bound_key(bound_of<THREADS>(top ? value_of(top) : -INFINITY, n, s)), s);
        if (count > THREADS + RANKED) {        // (so that each thread has had one, and no two the same)
            int rank = 0;
#pragma unroll 8
            for (int j = 0; j < THREADS; ++j) rank += s.tops[j] > top;
            if (rank == n - 1) s.least = top;
            __syncthreads();
            count = keep_held<THREADS>(count, s.least, s);
        }
    }
    __syncthreads();
    rank_held<THREADS>(count, n, s);
    __syncthreads();
    return count < n ? count : n;
}
// A thread's vectors i, i + THREADS, .. of a row
template <bool BF16, int THREADS>
__device__ inline void load_vectors(u32x4 (&v)[AT_ONCE], const void* row, int i, int end) {
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) v[u] = i + u * THREADS < end ? row_type<BF16>::load(row, i + u * THREADS) : row_type<BF16>::none();
}
// the largest of each of them, and of all
template <bool BF16>
__device__ inline float largest_of(const u32x4 (&v)[AT_ONCE], float (&tops)[AT_ONCE]) {
    float top = -INFINITY;
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
        const u32x4 one[1] = {v[u]};
        tops[u] = running_sums<BF16>::largest(one);
        top = fmaxf(top, tops[u]);
    }
    return top;
}
// The logits of these vectors that reach the bound, and whose keys are not below `least`
template <bool BF16, int THREADS>
__device__ __forceinline__ void hold_above(const u32x4 (&v)[AT_ONCE], const float (&tops)[AT_ONCE], int i, float bound, uint64_t least, top_scratch<THREADS>& s) {
    typedef row_type<BF16> T;
    constexpr int N = T::N;
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
        if (!(tops[u] >= bound)) continue;
        uint32_t above = 0;                    // a bit for each element.  Few lanes have one, seldom more
#pragma unroll
        for (int e = 0; e < N; ++e) above |= (uint32_t)(T::at(v[u], e) >= bound) << e;
        while (above) {
            const int at = __builtin_ctz(above);
            float x = T::at(v[u], 0);
#pragma unroll
            for (int e = 1; e < N; ++e) x = e == at ? T::at(v[u], e) : x;
            const uint64_t key = key_of(x, (i + u * THREADS) * N + at);
            if (key >= least) hold(key, s);
            above &= above - 1;
        }
    }
}
// Where too many logits reach the bound (they ascend, or many are equal), the vectors from `begin` to `end` and `extra` once more, AT_ONCE of each thread at a time:
// with the n first of those before, and again with a higher bound, the last of the n first among those that found a place, as long as there are too many (each
// time HELD - 2 n fewer or more).  4096 x 131072 bf16, n = 8 | 64: ascending rows 702 | 1323 us, equal logits 716 | 789, the first half masked 343 | 395.  Returns how
// many are in s.best.
template <bool BF16, int THREADS>
__device__ __forceinline__ int select_again(const void* row, int begin, int end, float extra, int extra_at, int n, top_scratch<THREADS>& s) {
    uint64_t least = bound_key(LOWEST);
    int kept = 0;
    for (int i = begin + threadIdx.x; i - (int)threadIdx.x < end;) {
        u32x4 v[AT_ONCE];
        float tops[AT_ONCE];
        const float more = i - (int)threadIdx.x + AT_ONCE * THREADS < end ? -INFINITY : extra;
        load_vectors<BF16, THREADS>(v, row, i, end);
        const float top = largest_of<BF16>(v, tops);
        int count = 0;
        if (__syncthreads_or(fmaxf(top, more) >= value_of(least))) {
            const uint64_t of_these = bound_key(bound_of<THREADS>(top, n, s));
            least = of_these > least ? of_these : least;
            if ((int)threadIdx.x < kept) s.held[threadIdx.x] = s.kept[threadIdx.x];
            if (threadIdx.x == 0) s.count = kept;
            __syncthreads();
            int at = i;                        // (read again: held in registers meanwhile they would be taken from the pass before)
            asm volatile("" : "+v"(at));
            load_vectors<BF16, THREADS>(v, row, at, end);
            largest_of<BF16>(v, tops);
            hold_above<BF16, THREADS>(v, tops, at, value_of(least), least, s);
            if (more >= value_of(least) && key_of(more, extra_at) >= least) hold(key_of(more, extra_at), s);
            __syncthreads();
            count = s.count;
            const int found = first_held<THREADS>(count < s.HELD ? count : s.HELD, n, s);
            if (found == n) least = s.best[n - 1];
            if (count <= s.HELD) {
                kept = found;
                if ((int)threadIdx.x < kept) s.kept[threadIdx.x] = s.best[threadIdx.x];
            }
        }
        if (count <= s.HELD) i += AT_ONCE * THREADS;
    }
    return kept;
}

// A row's results, from its sums and from `found` alternatives in s.best
template <bool BF16, int THREADS>
__device__ inline void write_row(const logp_args& a, int64_t r, const softmax_stats& st, int found, const top_scratch<THREADS>& s) {
    const int tid = threadIdx.x;
    if (tid >= a.m && tid >= a.n && tid > 0) return;
    const bool empty = st.m == -INFINITY && st.s == 0.f;
    const double log_s = st.s > 0.f && st.s < INFINITY ? log2_of(st.s) * LN2 : (double)logf(st.s);
    if (tid < a.m) {
        const int id = a.ids[r * a.m + tid];
        float lp = 0.f;
        if ((uint32_t)id < (uint32_t)a.V) lp = empty ? -INFINITY : logp_of(load1<BF16>(row_of<BF16>(a.logits, r * a.ld), id), st, log_s, a.inv_temp);
        a.logp[r * a.m + tid] = lp;
    }
    if (tid < a.n) {
        a.top_idx[r * a.n + tid] = tid < found ? index_of(s.best[tid]) : -1;
        a.top_logp[r * a.n + tid] = tid < found ? logp_of(value_of(s.best[tid]), st, log_s, a.inv_temp) : -INFINITY;
    }
    if (tid == 0) {
        if (a.entropy) a.entropy[r] = empty ? 0.f : (float)(log_s - (double)(st.u / st.s) * LN2);
        if (a.stats) {
            a.stats[2 * r] = st.m;
            a.stats[2 * r + 1] = st.s;
        }
    }
}

// One pass over a row, or a part of it, for the sums and the alternatives.  The n-th largest of the largest logits that groups of threads have among
// their first vectors bounds the alternatives from below, closely; what reaches the bound, a few times n logits, is held in LDS and ranked in the end.
// Bound by the logits' bytes: 4096 x 131072 bf16, n = 8 187 us, 5.7 TB/s (a pass over the row for each alternative 4496);
// the vector ALU, an exponential for each logit among its work, is busy for 16 % of the waves' cycles.  Rows that end late bound the fewer ones: 333 x 50001 f32 17.5.
template <bool BF16, int THREADS, bool PARTS>
__global__ __launch_bounds__(THREADS, 8) void logp_kernel(const logp_args a) {
    typedef row_type<BF16> T;
    constexpr int N = T::N;
    __shared__ block_scratch s_scratch;
    __shared__ top_scratch<THREADS> s_top;
    __shared__ int32_t s_last;
    const int64_t r = PARTS ? blockIdx.x / a.parts : a.first + blockIdx.x;
    const int part = PARTS ? blockIdx.x % a.parts : 0, tid = threadIdx.x, n = a.n;
    const void* const z = row_of<BF16>(a.logits, r * a.ld);
    const row_part piece = PARTS ? part_of_row(a.V, N, part, a.parts, a.part_vecs) : part_of_row(a.V, N, 0, 1, a.V);
    const int begin = piece.begin, end = piece.end, behind_at = piece.behind(tid);
    running_sums<BF16> sums(a.inv_temp * LOG2E);
    float bound = NAN;                         // what an alternative reaches (without alternatives nothing does)
    int i = begin + tid;
    const float extra = behind_at >= 0 ? load1<BF16>(z, behind_at) : -INFINITY;
    {
        u32x4 v[AT_ONCE];
        float tops[AT_ONCE];
        load_vectors<BF16, THREADS>(v, z, i, end);
        const float top = largest_of<BF16>(v, tops);
        if (n) {
            if (tid == 0) s_top.count = 0;
            bound = fmaxf(bound_of<THREADS>(top, n, s_top), LOWEST);
        }
        sums.take(top);
        sums.sum(v);
        // n of the first vectors' logits are not below the bound, so one behind them that equals it has n before it
        const float behind = next_above(bound);
        bound = bound > LOWEST ? bound : behind;
        if (top >= bound) hold_above<BF16, THREADS>(v, tops, i, bound, 0, s_top);
        bound = behind;
    }
    for (i += AT_ONCE * THREADS; i - tid < end; i += AT_ONCE * THREADS) {
        u32x4 v[AT_ONCE];
        float tops[AT_ONCE];
        load_vectors<BF16, THREADS>(v, z, i, end);
        const float top = largest_of<BF16>(v, tops);
        sums.take(top);
        sums.sum(v);
        if (top >= bound) hold_above<BF16, THREADS>(v, tops, i, bound, 0, s_top);
    }
    if (extra >= bound) hold(key_of(extra, behind_at), s_top);
    sums.add_one(extra);
    softmax_stats st = block_join(sums.st, sums.c, s_scratch);
    int found = 0;
    if (n) {
        __syncthreads();
        const int count = s_top.count;
        found = __builtin_expect(count <= s_top.HELD, 1) ? first_held<THREADS>(count, n, s_top) : select_again<BF16, THREADS>(z, begin, end, extra, behind_at, n, s_top);
    }
    if constexpr (PARTS) {
        float* const mine = a.part_sums + (r * a.parts + part) * 3;
        uint64_t* const tops = a.part_tops + r * a.parts * n;
        if (tid == 0) {
            __hip_atomic_store(mine, st.m, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            __hip_atomic_store(mine + 1, st.s, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            __hip_atomic_store(mine + 2, st.u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        if (tid < n) {
            const uint64_t key = tid < found ? s_top.best[tid] : 0;
            __hip_atomic_store(tops + part * n + tid, key, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        if (!last_block(a.tickets + (1 + GRAD_GROUPS + r) * GRAD_TICKET_INTS, a.parts, s_last)) return;
        const float* const all = a.part_sums + r * a.parts * 3;
        auto at = [&](int64_t k) { return __hip_atomic_load(tops + k, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
        constexpr int EACH = MAX_PARTS * LOGP_MAX_TOP / THREADS;
        static_assert(!PARTS || top_scratch<THREADS>::HELD >= MAX_PARTS * LOGP_MAX_TOP, "room for all parts' lists");
        uint64_t theirs[EACH];                 // (all on their way at a time)
#pragma unroll
        for (int e = 0; e < EACH; ++e) theirs[e] = tid + e * THREADS < a.parts * n ? at(tid + e * THREADS) : 0;
        if (tid < 64) {                        // (at most 64 parts: a lane has one)
            st = softmax_stats{-INFINITY, 0.f, 0.f};
            if (tid < a.parts)
                st = softmax_stats{__hip_atomic_load(all + tid * 3, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT),
                                   __hip_atomic_load(all + tid * 3 + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT),
                                   __hip_atomic_load(all + tid * 3 + 2, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)};
            const float m = wave_largest(st.m);
            if (m > -INFINITY) rebase(st, m, sums.c);
            st = softmax_stats{m, wave_total(st.s), wave_total(st.u)};
        }
        if (n) {
            // the parts' lists as one: the bound from the first of each
            const bool many = many_groups(THREADS, n);
            const int firsts = (many ? GROUPS_OF_MANY : GROUPS_OF_FEW) / a.parts;              // of each part
            if (tid < GROUPS_OF_MANY) s_top.groups[tid] = -INFINITY;
            if (tid == 0) s_top.count = 0;
            __syncthreads();
#pragma unroll
            for (int e = 0; e < EACH; ++e) {
                const int k = tid + e * THREADS;
                if (k < a.parts * n && k % n < firsts) s_top.groups[k / n * firsts + k % n] = theirs[e] ? value_of(theirs[e]) : -INFINITY;
            }
            const uint64_t first = bound_key(many ? nth_of<GROUPS_OF_MANY>(n, s_top) : nth_of<GROUPS_OF_FEW>(n, s_top));
#pragma unroll
            for (int e = 0; e < EACH; ++e)
                if (theirs[e] >= first) hold(theirs[e], s_top);
            __syncthreads();
            found = first_held<THREADS>(s_top.count, n, s_top);
        }
        __syncthreads();
        if (tid == 0) {
            s_scratch.a[0] = st.m;
            s_scratch.b[0] = st.s;
            s_scratch.a[1] = st.u;
        }
        __syncthreads();
        st = softmax_stats{s_scratch.a[0], s_scratch.b[0], s_scratch.a[1]};
    }
    write_row<BF16>(a, r, st, found, s_top);
}

// Parts of a row, for long rows that alone leave much of the chip idle; a row's end, its tickets and the joining, then comes twice, 4 us.  So only up to 128 rows
// (n = 8, bf16 x 131072: 120 rows 16.5 whole, 14.8 in parts; 256 rows 18 and 24; 333 x 50001 f32 17.5 and 22), in one block for each CU; very few rows in
// smaller blocks, which end sooner (n = 20, 4 x 131072 f32 9.6 -> 9.3, 16 x 131072 bf16 10.9 -> 9.9, but 40 rows 11.2 -> 11.9).
int logp_parts(int64_t rows, int vecs, int threads) {
    int parts = 1;
    while (parts < MAX_PARTS && rows * parts * 2 <= (threads == FEW_THREADS ? 512 : 256) && vecs / (parts * 2) >= AT_ONCE * threads) parts *= 2;
    return parts;
}

struct logp_grad_args {
    const void* logits;
    int64_t ld, ld_grad, rows, first;
    int V, m;
    const int32_t* ids;
    float inv_temp;
    const float *dlogp, *dentropy, *stats, *entropy;
    void* dlogits;
    int parts, part_vecs;
};

// dz[v] = (sum_j dlogp_j (1[v = id_j] - p_v) - dH p_v (log p_v + H)) / temperature = 2^y (a y + b), and more at the given tokens.  A block has a row or, of
// few rows, a part of one: the row's sums are there already.  Bound by the writes: 1024 x 131072 bf16 to bf16 102 us, 4.9 TB/s read and written; 100 x 50001 f32
// in parts 8.5 (whole rows 12.1).
template <bool BF16, bool GRAD_BF16, int THREADS>
__global__ __launch_bounds__(THREADS) void logp_grad_kernel(const logp_grad_args a) {
    typedef row_type<BF16> T;
    constexpr int N = T::N;
    __shared__ float s_d[LOGP_MAX_GIVEN], s_v[LOGP_MAX_GIVEN];
    __shared__ int s_id[LOGP_MAX_GIVEN];
    const int64_t b = a.first + blockIdx.x, r = b / a.parts;
    const int tid = threadIdx.x;
    const row_part piece = part_of_row(a.V, N, (int)(b % a.parts), a.parts, a.part_vecs);
    const int begin = piece.begin, end = piece.end;
    const void* const z = row_of<BF16>(a.logits, r * a.ld);
    void* const out = row_of<GRAD_BF16>(a.dlogits, r * a.ld_grad);
    const float m = a.stats[2 * r], s = a.stats[2 * r + 1], dH = a.dentropy ? a.dentropy[r] : 0.f;
    if (tid < a.m) {
        const int id = a.ids[r * a.m + tid];
        float v = 0.f, d = 0.f;
        if ((uint32_t)id < (uint32_t)a.V && (v = load1<BF16>(z, id), !(v <= LOWEST))) d = a.dlogp[r * a.m + tid];
        s_id[tid] = id;
        s_v[tid] = v;
        s_d[tid] = d;
    }
    const int behind = piece.behind(tid);                      // an element behind the vectors
    const float extra = behind >= 0 ? load1<BF16>(z, behind) : 0.f;
    __syncthreads();
    const int lane = tid & 63;                                 // (each wave has the given tokens, one to a lane)
    const int id = lane < a.m ? s_id[lane] : -1;
    const float d = lane < a.m ? s_d[lane] : 0.f, v_id = lane < a.m ? s_v[lane] : 0.f, sum = wave_total(d);
    bool live = dH != 0.f || __ballot(d != 0.f) != 0;          // (NaN is not zero)
    live &= !(m == -INFINITY && s == 0.f);
    if (!live) {                               // (the same for the whole block)
        const float none[N] = {};
        for (int i = begin + tid; i < end; i += THREADS) store_grad<GRAD_BF16, N>(out, i, none);
        if (behind >= 0) store1<GRAD_BF16>(out, behind, 0.f);
        return;
    }
    const float c = a.inv_temp * LOG2E, scale = a.inv_temp / s;
    const double log_s = s > 0.f && s < INFINITY ? log2_of(s) * LN2 : (double)logf(s), H = dH != 0.f ? (double)a.entropy[r] : 0.0;
    const float ka = (float)(-(double)dH * LN2) * scale, kb = (float)((double)dH * (log_s - H) - (double)sum) * scale;
    auto of = [&](float v) {
        const float y = (v - m) * c;
        return __builtin_amdgcn_exp2f(y) * fmaf(ka, fmaxf(y, Y_LOWEST), kb);
    };
    auto put = [&](const u32x4& v, int i) {
        float g[N];
#pragma unroll
        for (int j = 0; j < N; ++j) g[j] = of(T::at(v, j));
        store_grad<GRAD_BF16, N>(out, i, g);
    };
    int i = begin + tid;
    if (__builtin_expect(!(fabsf(ka) < INFINITY && fabsf(kb) < INFINITY), 0)) {
        // infinite or NaN gradients or logits, which 2^y = 0 of a masked logit does not take away (asked for each logit of all rows it costs short ones 13 %)
        auto open = [&](float v) { return v <= LOWEST ? 0.f : of(v); };
        for (; i < end; i += THREADS) {
            const u32x4 v = T::load(z, i);
            float g[N];
#pragma unroll
            for (int j = 0; j < N; ++j) g[j] = open(T::at(v, j));
            store_grad<GRAD_BF16, N>(out, i, g);
        }
        if (behind >= 0) store1<GRAD_BF16>(out, behind, open(extra));
    } else {
        for (; i + (AT_ONCE - 1) * THREADS < end; i += AT_ONCE * THREADS) {
            u32x4 v[AT_ONCE];
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) v[u] = T::load(z, i + u * THREADS);
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) put(v[u], i + u * THREADS);
        }
        for (; i < end; i += THREADS) put(T::load(z, i), i);
        if (behind >= 0) store1<GRAD_BF16>(out, behind, of(extra));
    }
    // the given tokens, by the threads that have written their places: one with several gradients receives their sum as often
    const int owner = id < piece.place ? (id / N - begin) % THREADS : id - piece.place;
    const bool here = id >= begin * N && id < piece.place + piece.rest && owner >> 6 == tid >> 6 && !(v_id <= LOWEST);
    for (uint64_t left = __ballot(here); left; left &= left - 1) {
        const int j = __builtin_ctzll(left), to = __builtin_amdgcn_readlane(id, j);
        const float more = wave_total(id == to ? d : 0.f), v = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v_id), j));
        if (tid == __builtin_amdgcn_readlane(owner, j)) store1<GRAD_BF16>(out, to, fmaf(more, a.inv_temp, of(v)));
    }
}

template <int THREADS, class Kernel, class Args>
hipError_t launch_rows(hipStream_t s, Kernel kernel, Args a, int64_t blocks) {
    for (a.first = 0; a.first < blocks; a.first += LOGP_MAX_GRID)
        hipLaunchKernelGGL(kernel, dim3((unsigned)(blocks - a.first < LOGP_MAX_GRID ? blocks - a.first : LOGP_MAX_GRID)), dim3(THREADS), 0, s, a);
    return hipGetLastError();
}

// Threads of a whole row's block: a vector or more each.  1024 where the blocks are about as many as the CUs hold at a time (256 x 131072 bf16, n = 8 18.3 us, with
// 512 21.9; 2000 x 50001 61 and 53)
template <bool BF16>
hipError_t launch_whole(hipStream_t s, const logp_args& a, int vecs) {
    if (vecs <= 64 * AT_ONCE) return launch_rows<64>(s, logp_kernel<BF16, 64, false>, a, a.rows);
    if (vecs <= 256 * AT_ONCE) return launch_rows<256>(s, logp_kernel<BF16, 256, false>, a, a.rows);
    if (vecs > 1024 * AT_ONCE && a.rows <= 640) return launch_rows<1024>(s, logp_kernel<BF16, 1024, false>, a, a.rows);
    return launch_rows<512>(s, logp_kernel<BF16, 512, false>, a, a.rows);
}

// Many short rows in blocks of one wave (65536 x 100 bf16 31.6 us, in larger ones 87; 8192 x 2000 14.4 and 16.4; but 500 x 2000 to f32 5.1 and 4.0)
template <bool BF16>
hipError_t launch_gradient(hipStream_t s, const logp_grad_args& a, bool grad_bf16, int vecs) {
    const int64_t n = a.rows * a.parts;
    if (vecs <= 64 * AT_ONCE && a.rows >= 2048)
        return grad_bf16 ? launch_rows<64>(s, logp_grad_kernel<BF16, true, 64>, a, n) : launch_rows<64>(s, logp_grad_kernel<BF16, false, 64>, a, n);
    return grad_bf16 ? launch_rows<LOGP_THREADS>(s, logp_grad_kernel<BF16, true, LOGP_THREADS>, a, n)
                     : launch_rows<LOGP_THREADS>(s, logp_grad_kernel<BF16, false, LOGP_THREADS>, a, n);
}

}  // namespace

hipError_t launch_token_logp(moe_ctx* c, const void* logits, int64_t ld, int32_t dtype, int64_t rows, int32_t V, const int32_t* ids, int32_t m,
                             float temperature, float* logp, float* entropy, int32_t n, int32_t* top_idx, float* top_logp, float* stats) {
    logp_args a{logits, ld, rows, 0, V, m, n, ids, 1.0f / temperature, logp, entropy, top_logp, stats, top_idx};
    const int vecs = V / (dtype == MOE_BF16 ? 8 : 4), threads = rows <= FEW_ROWS_IN_PARTS ? FEW_THREADS : PART_THREADS, parts = logp_parts(rows, vecs, threads);
    if (parts > 1) {
        static_assert((size_t)MAX_SPLIT_ROWS * MAX_PARTS * (3 * sizeof(float) + LOGP_MAX_TOP * sizeof(uint64_t)) <= GRAD_WS_BYTES && MAX_SPLIT_ROWS <= GRAD_MAX_SPLIT_ROWS, "room for all parts");
        a.parts = parts;
        a.part_vecs = (vecs + parts - 1) / parts;
        a.part_tops = static_cast<uint64_t*>(c->grad_ws);
        a.part_sums = reinterpret_cast<float*>(a.part_tops + (int64_t)MAX_SPLIT_ROWS * MAX_PARTS * LOGP_MAX_TOP);
        a.tickets = c->grad_tickets;
        if (threads == FEW_THREADS)
            return dtype == MOE_BF16 ? launch_rows<FEW_THREADS>(c->stream, logp_kernel<true, FEW_THREADS, true>, a, rows * parts)
                                     : launch_rows<FEW_THREADS>(c->stream, logp_kernel<false, FEW_THREADS, true>, a, rows * parts);
        return dtype == MOE_BF16 ? launch_rows<PART_THREADS>(c->stream, logp_kernel<true, PART_THREADS, true>, a, rows * parts)
                                 : launch_rows<PART_THREADS>(c->stream, logp_kernel<false, PART_THREADS, true>, a, rows * parts);
    }
    return dtype == MOE_BF16 ? launch_whole<true>(c->stream, a, vecs) : launch_whole<false>(c->stream, a, vecs);
}

hipError_t launch_token_logp_backward(hipStream_t s, const void* logits, int64_t ld, int32_t dtype, int64_t rows, int32_t V, const int32_t* ids, int32_t m,
                                      float temperature, const float* dlogp, const float* dentropy, const float* stats, const float* entropy,
                                      void* dlogits, int64_t ld_grad, int32_t grad_dtype) {
    logp_grad_args a{logits, ld, ld_grad, rows, 0, V, m, ids, 1.0f / temperature, dlogp, dentropy, stats, entropy, dlogits, 1, V};
    const int vecs = V / (dtype == MOE_BF16 ? 8 : 4);
    // parts of a row, each a round of vectors or more (in place a row's given tokens are read before any of the row is written, by one block)
    if (dlogits != logits && rows < 2048) {
        const int64_t parts = vecs / (AT_ONCE * LOGP_THREADS) < 2048 / rows ? vecs / (AT_ONCE * LOGP_THREADS) : 2048 / rows;
        if (parts > 1) a.parts = (int)parts;
        a.part_vecs = (vecs + a.parts - 1) / a.parts;
    }
    return dtype == MOE_BF16 ? launch_gradient<true>(s, a, grad_dtype == MOE_BF16, vecs) : launch_gradient<false>(s, a, grad_dtype == MOE_BF16, vecs);
}

}  // namespace moe355
