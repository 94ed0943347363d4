// Embedding lookup with scaling, and the table's gradient.
//
// Forward:   out[m] = alpha table[token m], the table in a float type or as int8 rows with a scale each.
// Gradient:  dtable[v] = alpha sum over the m with token v of dy[m]  (+ dtable[v]).
//
// The gradient goes by sorted tokens, so that every sum has a fixed order and no atomics:
//  (1) a launch that puts the tokens in order.  Up to 8192 are placed by comparing all with all (4111: 9 us, where sorting and placing
//      took 16); of more, workgroups sort 2048 each in their LDS (radix sort, stable; 16384 each in batches of more than 32768), and a
//      second launch places a chunk's tokens by binary searches in the other chunks.  Meanwhile the first launch's other workgroups
//      write the table's zeros, which bound it where they are many (32000 x 4096 bf16, 262 MB: 44 us, 6.0 TB/s).
//  (2) Eight or sixteen consecutive sorted rows at a time are read and added up (8192 x 4096 bf16: 18.5 us, 3.6 TB/s).  A token whose
//      rows lie inside such a stretch gets its row at once; one that crosses its ends leaves partial sums in the workspace, and
//  (3) those are joined in order (6.8 us, latency).
// However often a token occurs, (1) and (2) are split evenly.  (3) is not: one token's partial sums, one a stretch, are
// one workgroup's for 1024 columns, sixteen loads at a time (65536 x 1024 bf16 added: tokens spread 102 us, a tenth of them one token 126, all of
// them 355).  Batches of few thousand are bound by three launches one after the other, of which (1) has one workgroup for 64 tokens.
#include "linear.h"

#include <type_traits>

namespace niti {

namespace {

// Tokens are compared all with all up to kRankMax (the gradient of M x 256, added: 4096 18.1 us, by sorting 25.5; 8192 26.4 and 29.7;
// 12000 31.6 and 33.9, 16384 38.8 and 35.7).
constexpr int kRankMax = 8192;
constexpr int kSortFew = 2048;    // tokens that a workgroup sorts, in batches of up to kMergeMax, all of whose keys the next launch has in LDS
constexpr int kMergeMax = 32768;
constexpr int kSortMax = 16384;   // and in larger ones
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64, kRounds = kSortMax / kSortThreads;
constexpr int kBins = 256;
constexpr int kRunMin = 8;        // sorted rows of a stretch: 8 or 16
constexpr int64_t kMaxTokens = (int64_t)1 << 22;

// ---------------------------------------------------------------- forward
struct EmbArgs {
    const void* table;
    const float* scale;      // of int8 rows
    const int32_t* tokens;
    void* out;
    int64_t ldt, ldo, M, V, D;
    uint32_t ppr;            // pieces of a row
    float alpha;
};

// Eight codes of column c on, moved down where the row ends (D >= 8).
__device__ __forceinline__ void load_codes(const int8_t* row, int c, int D, float (&v)[CH]) {
    const int from = min(c, D - CH);
    uint64_t w;
    __builtin_memcpy(&w, row + from, 8);
    const int down = c - from;
    w >>= 8 * min(down, 7);
#pragma unroll
    for (int e = 0; e < CH; e++) v[e] = (float)(int8_t)(w >> (8 * e));
}

// TT: the table's type, int8_t for rows of codes.
template <typename TT, typename T>
__global__ __launch_bounds__(256) void embedding_kernel(EmbArgs a) {
    const uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t m = (int64_t)(i / a.ppr);
    if (m >= a.M) return;
    const int c = (int)(i % a.ppr) * CH, D = (int)a.D;
    const int tok = a.tokens[m];
    const bool in = (uint32_t)tok < (uint64_t)a.V;   // (negative ones are above every V)
    const TT* row = (const TT*)a.table + (in ? tok : 0) * a.ldt;
    float v[CH], f = a.alpha;
    if constexpr (__is_same(TT, int8_t)) {
        f *= a.scale[in ? tok : 0];
        if (D >= CH) {
            load_codes(row, c, D, v);
        } else {
#pragma unroll
            for (int e = 0; e < CH; e++) v[e] = (float)row[min(c + e, D - 1)];
        }
    } else if (D >= CH) {
        piece_values<TT, false>(load_piece<TT, false>(row, c, D), c, D, v);
    } else {
        load_some(row + c, D - c, v);
    }
#pragma unroll
    for (int e = 0; e < CH; e++) v[e] = in ? v[e] * f : 0.f;
    store_first((T*)a.out + m * a.ldo + c, D - c, v);
}

// ---------------------------------------------------------------- gradient
struct EmbBwdArgs {
    const void* dy;
    const int32_t* tokens;
    void* dtable;
    int64_t lddy, ldt, M, V, D;
    float alpha;
    int32_t accumulate, passes;   // passes of the sort
    int32_t run;                  // sorted rows of a stretch
    int32_t sorters;              // workgroups that sort, ahead of those that write zeros
    int32_t *order, *key;         // [M]: rows by token, and their tokens (V for those outside the table)
    int32_t *order1, *key1;       // the same of each chunk that is sorted
    int32_t chunk;                // tokens of one
    float* part;                  // [stretches][2][D]
};

// A token's place in the order: tokens outside the table after all others.
__device__ __forceinline__ int32_t sort_key(const EmbBwdArgs& a, int64_t i) {
    const int tok = a.tokens[i];
    return (uint32_t)tok < (uint64_t)a.V ? tok : (int32_t)a.V;
}

// The workgroups past those that sort write the zeros: of a whole table in one go, of spaced rows row by row.
template <typename TG>
__device__ __forceinline__ void write_zeros(const EmbBwdArgs& a) {
    const int t = threadIdx.x;
    const int64_t first = (int64_t)blockIdx.x - a.sorters, step = (int64_t)gridDim.x - a.sorters;
    const float zero[CH] = {};
    if (a.ldt == a.D) {
        constexpr int64_t BLOCK = (int64_t)kSortThreads * CH;
        const int64_t n = a.V * a.D;
        for (int64_t i = first * BLOCK + t * CH; i < n; i += step * BLOCK) {
            if (i + CH <= n) store_whole<true>((TG*)a.dtable + i, zero);
            else store_first((TG*)a.dtable + i, (int)(n - i), zero);
        }
    } else {
        for (int64_t r = first; r < a.V; r += step) {
            TG* row = (TG*)a.dtable + r * a.ldt;
            for (int c = t * CH; c < a.D; c += kSortThreads * CH) store_first(row + c, (int)(a.D - c), zero);
        }
    }
}

// (1) Few tokens: a token's place is the number of those before it, smaller ones and equal ones with a smaller index, counted by
// comparing all with all (two instructions a pair; bound by them and by each workgroup's reading of all tokens).  A
// workgroup places 64, its sixteen waves count in a sixteenth of the batch each: 65 workgroups, on as many of the 256 CUs, for 4111 tokens, 128 at most.
template <typename TG>
__global__ __launch_bounds__(kSortThreads) void token_rank_kernel(EmbBwdArgs a) {
    extern __shared__ __attribute__((aligned(16))) int32_t keys[];   // [M to a multiple of 64], and [16][64] counts
    if ((int)blockIdx.x >= a.sorters) {
        write_zeros<TG>(a);
        return;
    }
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int M = (int)a.M, room = (M + 63) / 64 * 64, i0 = (int)blockIdx.x * 64, i = i0 + lane;
    for (int j = t; j < room; j += kSortThreads) keys[j] = j < M ? sort_key(a, j) : 0x7FFFFFFF;   // (before none)
    __syncthreads();
    const int32_t k = keys[i];
    const int per = room / 64 * 4, from = wave * per, to = from + per;   // (multiples of 4, as i0 is)
    int n = 0;
    auto count = [&](int lo, int hi, auto before) {
#pragma unroll 4
        for (int j = max(from, lo); j < min(to, hi); j += 4) {
            const v4i x = *(const v4i*)(keys + j);
#pragma unroll
            for (int e = 0; e < 4; e++) n += before(x[e], j + e) ? 1 : 0;
        }
    };
    count(0, i0, [&](int32_t x, int) { return x <= k; });
    count(i0, i0 + 64, [&](int32_t x, int j) { return x < k || (x == k && j < i); });
    count(i0 + 64, room, [&](int32_t x, int) { return x < k; });
    int* counts = keys + room;
    counts[wave * 64 + lane] = n;
    __syncthreads();
    if (wave != 0 || i >= M) return;
    n = 0;
#pragma unroll
    for (int w = 0; w < kSortWaves; w++) n += counts[w * 64 + lane];
    a.order[n] = i;
    a.key[n] = k;
}

// LDS: the chunk's tokens, two lists of places, a counter for each digit and wave.
template <typename TG>
__global__ __launch_bounds__(kSortThreads) void token_sort_kernel(EmbBwdArgs a) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int t = threadIdx.x;
    if ((int)blockIdx.x >= a.sorters) {
        write_zeros<TG>(a);
        return;
    }
    const int64_t base = (int64_t)blockIdx.x * a.chunk;
    const int n = (int)min((int64_t)a.chunk, a.M - base);
    const int rounds = (n + kSortThreads - 1) / kSortThreads, room = rounds * kSortThreads;
    uint32_t* key = (uint32_t*)lds;
    uint16_t* src = (uint16_t*)(key + room);
    uint16_t* dst = src + room;
    uint16_t* bins = dst + room;                                  // [digit][wave]
    uint32_t* totals = (uint32_t*)(bins + kSortWaves * kBins);    // of the four waves that scan
    for (int i = t; i < n; i += kSortThreads) {
        key[i] = (uint32_t)sort_key(a, base + i);
        src[i] = (uint16_t)i;
    }
    const int wave = __builtin_amdgcn_readfirstlane(t >> 6), lane = t & 63;
    const uint64_t below = ((uint64_t)1 << lane) - 1;
    for (int pass = 0; pass < a.passes; pass++) {
        const int shift = 8 * pass;
        if (t < 2 * kBins) ((uint4*)bins)[t] = make_uint4(0, 0, 0, 0);
        __syncthreads();
        // A wave's places are consecutive.  All of a thread's are read before the first is counted.
        uint16_t place[kRounds], rank[kRounds];
        uint8_t digit[kRounds];
#pragma unroll
        for (int r = 0; r < kRounds; r++) {
            if (r < rounds) place[r] = src[min((wave * rounds + r) * 64 + lane, n - 1)];
        }
#pragma unroll
        for (int r = 0; r < kRounds; r++) {
            if (r < rounds) digit[r] = (uint8_t)(key[place[r]] >> shift);
        }
        // Each counts those of its digit before it, in this wave.
#pragma unroll
        for (int r = 0; r < kRounds; r++) {
            if (r >= rounds) continue;
            const bool in = (wave * rounds + r) * 64 + lane < n;
            const uint32_t d = digit[r];
            uint32_t lo = 0, hi = 0;   // lanes that differ in a bit
#pragma unroll
            for (int b = 0; b < 8; b++) {
                const uint64_t ones = __ballot(d >> b & 1);
                const uint32_t mine = (uint32_t)((int32_t)(d << (31 - b)) >> 31);
                lo |= (uint32_t)ones ^ mine;
                hi |= (uint32_t)(ones >> 32) ^ mine;
            }
            const uint64_t peers = __ballot(in) & ~((uint64_t)hi << 32 | lo);
            volatile uint16_t* bin = bins + d * kSortWaves + wave;
            const uint32_t old = *bin, before = (uint32_t)__popcll(peers & below);
            rank[r] = (uint16_t)(old + before);
            __builtin_amdgcn_wave_barrier();
            if (in && before == 0) *bin = (uint16_t)(old + (uint32_t)__popcll(peers));
            __builtin_amdgcn_wave_barrier();
        }
        __syncthreads();
        // bins[d][wave] = places of smaller digits, and of this one in the waves before: below 2^14
        uint32_t count[kSortWaves], sum = 0, incl = 0;
        if (t < kBins) {
            uint16_t c[kSortWaves];
            __builtin_memcpy(c, __builtin_assume_aligned(bins + t * kSortWaves, 16), sizeof(c));
#pragma unroll
            for (int w = 0; w < kSortWaves; w++) {
                count[w] = sum;
                sum += c[w];
            }
            incl = sum;
#pragma unroll
            for (int o = 1; o < 64; o *= 2) {
                const uint32_t u = (uint32_t)__shfl_up((int)incl, o, kWave);
                incl += lane >= o ? u : 0u;
            }
            if (lane == 63) totals[wave] = incl;
        }
        __syncthreads();
        if (t < kBins) {
            uint32_t before = incl - sum;
#pragma unroll
            for (int w = 0; w < 3; w++) before += w < wave ? totals[w] : 0u;
            uint16_t c[kSortWaves];
#pragma unroll
            for (int w = 0; w < kSortWaves; w++) c[w] = (uint16_t)(count[w] + before);
            __builtin_memcpy(__builtin_assume_aligned(bins + t * kSortWaves, 16), c, sizeof(c));
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kRounds; r++) {
            if (r < rounds && (wave * rounds + r) * 64 + lane < n) dst[bins[(int)digit[r] * kSortWaves + wave] + rank[r]] = place[r];
        }
        __syncthreads();
        uint16_t* x = src;
        src = dst, dst = x;
    }
    for (int i = t; i < n; i += kSortThreads) {
        const int p = src[i];
        a.order1[base + i] = (int32_t)(base + p);
        a.key1[base + i] = (int32_t)key[p];
    }
}

// Number of keys below k (or up to k) of n in order.
__device__ __forceinline__ int64_t count_below(const int32_t* key, int64_t n, int32_t k, bool equal) {
    int64_t lo = 0, hi = n;
    while (lo < hi) {
        const int64_t mid = (lo + hi) >> 1;
        const int32_t v = key[mid];
        if (v < k || (equal && v == k)) lo = mid + 1;
        else hi = mid;
    }
    return lo;
}

// Several chunks: an element's place is its own in its chunk and, in every other, the
// number of smaller tokens, equal ones among them in the chunks before.
__global__ __launch_bounds__(256) void token_merge_kernel(EmbBwdArgs a) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= a.M) return;
    const int32_t k = a.key1[i];
    const int64_t mine = i / kSortMax;
    int64_t at = i - mine * kSortMax;
    for (int64_t c = 0; c * kSortMax < a.M; c++)
        if (c != mine) at += count_below(a.key1 + c * kSortMax, min((int64_t)kSortMax, a.M - c * kSortMax), k, c < mine);
    a.order[at] = a.order1[i];
    a.key[at] = k;
}

// The same for chunks of 2048 that all fit in LDS: four searches of twelve steps at a time.
__global__ __launch_bounds__(1024) void token_merge_few_kernel(EmbBwdArgs a) {
    extern __shared__ __attribute__((aligned(16))) int32_t keys[];
    const int M = (int)a.M, chunks = (M + kSortFew - 1) / kSortFew;
    const int i = (int)blockIdx.x * 1024 + (int)threadIdx.x, mine = (int)blockIdx.x * 1024 / kSortFew;
    const int32_t place = a.order1[min(i, M - 1)];
#pragma unroll 4
    for (int j = (int)threadIdx.x * 4; j < M; j += 4096) {   // (whole fours: the workspace holds more than the last)
        const v4i x = *(const v4i*)(a.key1 + j);
        *(v4i*)(keys + j) = x;
    }
    __syncthreads();
    if (i >= M) return;
    const int32_t k = keys[i];
    int at = i - mine * kSortFew;
    for (int c0 = 0; c0 < chunks; c0 += 4) {
        int pos[4] = {0, 0, 0, 0};
#pragma unroll
        for (int step = kSortFew; step >= 1; step /= 2)
#pragma unroll
            for (int j = 0; j < 4; j++) {
                const int c = c0 + j, n = min(kSortFew, M - c * kSortFew);   // (of a chunk past the last: none)
                const int32_t v = keys[min(c * kSortFew + pos[j] + step, M) - 1];
                const bool before = v < k || (v == k && c < mine);
                pos[j] += pos[j] + step <= n && before ? step : 0;
            }
#pragma unroll
        for (int j = 0; j < 4; j++) at += c0 + j == mine ? 0 : pos[j];
    }
    a.order[at] = place;
    a.key[at] = k;
}

constexpr int kSumThreads = 256, kSumCols = kSumThreads * CH;

// A sum on top of old, where there is something to add to.
template <int N>
__device__ __forceinline__ void sum_on(const EmbBwdArgs& a, const float (&sum)[N], float (&old)[N]) {
#pragma unroll
    for (int e = 0; e < N; e++) old[e] = a.accumulate ? __builtin_fmaf(a.alpha, sum[e], old[e]) : a.alpha * sum[e];
}

// (2) A stretch of sorted rows, 2048 columns.  KIND: the number of columns is a multiple of 8 (2), is at least 8 (1), or neither (0).
// ADD: with each row goes what its token's row in the table holds (read for every row: tokens' last rows are known later than the
// loads are to go out, and the others hit a cache).
template <typename T, typename TG, int KIND, bool ADD, int RUN>
__global__ __launch_bounds__(kSumThreads) void token_sum_kernel(EmbBwdArgs a, int slices) {
    constexpr int AHEAD = sizeof(T) == 4 && RUN > 8 ? 8 : RUN;   // rows in flight
    const int64_t s = blockIdx.x / (uint32_t)slices;
    const int D = (int)a.D, c = (int)(blockIdx.x % (uint32_t)slices) * kSumCols + (int)threadIdx.x * CH;
    const int64_t i0 = s * RUN;
    const int n = (int)min((int64_t)RUN, a.M - i0);
    // tokens and rows of the stretch, and its neighbours' tokens (-1: none): one load each, lane by lane
    const int lane = threadIdx.x & 63;
    const int64_t at = i0 + lane - 1;
    int32_t keys = a.key[min(max(at, (int64_t)0), a.M - 1)];
    const int32_t rows = a.order[min(i0 + min(lane, RUN - 1), a.M - 1)];
    keys = at >= 0 && at < a.M ? keys : -1;
    auto key_of = [&](int i) { return __builtin_amdgcn_readlane(keys, i + 1); };   // -1 .. RUN
    float sum[CH] = {};
    bool first = true;    // no row of this stretch has ended a token yet
    int32_t k = key_of(0);
    const int32_t before = key_of(-1);
#pragma unroll
    for (int j0 = 0; j0 < RUN; j0 += AHEAD) {
        if (j0 >= n) break;
        Piece<T> p[AHEAD];
        Piece<TG> o[ADD ? AHEAD : 1];
        if constexpr (KIND > 0) {
#pragma unroll
            for (int j = 0; j < AHEAD; j++)
                p[j] = load_piece<T, KIND == 2>((const T*)a.dy + (int64_t)__builtin_amdgcn_readlane(rows, j0 + j) * a.lddy, c, D);
            if constexpr (ADD) {
#pragma unroll
                for (int j = 0; j < AHEAD; j++) {
                    const int32_t t = key_of(j0 + j);   // (past the end -1)
                    o[j] = load_piece<TG, KIND == 2>((const TG*)a.dtable + ((uint32_t)t < (uint64_t)a.V ? t : 0) * a.ldt, c, D);
                }
            }
        }
#pragma unroll
        for (int j = 0; j < AHEAD; j++) {
            const int i = j0 + j;
            if (i >= n) break;
            float v[CH];
            if constexpr (KIND > 0) piece_values<T, KIND == 2>(p[j], c, D, v);
            else load_some((const T*)a.dy + (int64_t)__builtin_amdgcn_readlane(rows, i) * a.lddy + c, D - c, v);
#pragma unroll
            for (int e = 0; e < CH; e++) sum[e] += v[e];
            const int32_t next = key_of(i + 1);
            if (next == k && i + 1 < n) continue;
            // the last row of token k here
            const bool from = first && before == k, on = i + 1 == n && next == k;
            if (c < D && k < a.V) {
                if (from || on) {
                    store_first(a.part + (2 * s + (from ? 0 : 1)) * a.D + c, D - c, sum);
                } else {
                    float old[CH] = {};
                    if constexpr (ADD && KIND > 0) piece_values<TG, KIND == 2>(o[j], c, D, old);
                    else if (ADD) load_some((const TG*)a.dtable + k * a.ldt + c, D - c, old);
                    sum_on(a, sum, old);
                    store_first((TG*)a.dtable + k * a.ldt + c, D - c, old);
                }
            }
#pragma unroll
            for (int e = 0; e < CH; e++) sum[e] = 0.f;
            first = false;
            k = next;
        }
    }
}

// (3) The token that crosses the end of a stretch that it begins in: its partial sums in order.  Threads that rows of fewer than 1024
// columns leave over take every `groups`-th partial sum, and the groups' sums are added in order.  No load is in a branch that part of a
// wave takes, where it would be waited for: the four columns at a row's end are read, and added up, from four before it on, and only
// those of this thread are stored (NARROW: of fewer than four, one by one).  The first two partial sums, all that most tokens have,
// are on their way with the tokens (8192 x 4096: 8.3 -> 6.8 us; the three launches for 4111 x 1111 added 25.7 -> 23.5).
constexpr int kJoinCols = 1024;
template <typename TG, bool GROUPS, bool NARROW>
__global__ __launch_bounds__(256) void token_join_kernel(EmbBwdArgs a, int slices, int of_groups) {
    __shared__ float sums[GROUPS ? 256 : 1][4];
    const int groups = GROUPS ? of_groups : 1;
    const int64_t s = blockIdx.x / (uint32_t)slices;
    const int per = 256 / groups, group = GROUPS ? (int)threadIdx.x / per : 0;
    const int c = (int)(blockIdx.x % (uint32_t)slices) * kJoinCols + (int)threadIdx.x % per * 4;
    const int64_t i0 = s * a.run, end = i0 + a.run;   // (the last stretch crosses nothing)
    if (end >= a.M) return;
    const int D = (int)a.D, from = NARROW ? c : min(c, D - 4);
    auto load = [&](const auto* row, float (&v)[4]) {
        if constexpr (NARROW) {
#pragma unroll
            for (int e = 0; e < 4; e++) v[e] = to_f(row[min(c + e, D - 1)]);
        } else {
            load_n(row + from, v);
        }
    };
    const int64_t stretches = (a.M + a.run - 1) / a.run;
    float sum[4], next[4];
    load(a.part + (2 * s + 1) * a.D, sum);
    load(a.part + 2 * min(s + 1 + group, stretches - 1) * a.D, next);
    const int lane = threadIdx.x & 63;
    // stretches after this one that the token fills to their ends, 64 at a time: the next stretch's first token, and the one before it
    auto ends = [&](int64_t at, int i) { return a.key[min((at + lane + 1) * a.run - 1 + i, a.M - 1)]; };
    int32_t x = ends(s + 1, 0), y = ends(s + 1, 1);
    const int32_t k = a.key[end], own = a.key[end - 1], left_of = a.key[max(i0 - 1, (int64_t)0)];
    if (own != k || k >= a.V || (i0 > 0 && left_of == k)) return;   // (the same for all threads)
    float old[4] = {};
    if (a.accumulate) load((const TG*)a.dtable + k * a.ldt, old);
    int64_t last = s + 1;
    for (;;) {
        const uint64_t on = __ballot((last + lane + 1) * a.run < a.M && x == k && y == k);
        const int n = __ffsll((long long)~on);   // (0: all 64)
        last += n ? n - 1 : 64;
        if (n) break;
        x = ends(last, 0), y = ends(last, 1);
    }
    const bool mine = s + 1 + group <= last;
#pragma unroll
    for (int e = 0; e < 4; e++) sum[e] = (group == 0 ? sum[e] : 0.f) + (mine ? next[e] : 0.f);
    for (int64_t p0 = s + 1 + groups; p0 <= last; p0 += 16 * groups) {   // (the same for all threads)
        const int64_t p = p0 + group;
        float v[16][4];
#pragma unroll
        for (int i = 0; i < 16; i++) load(a.part + 2 * min(p + i * groups, last) * a.D, v[i]);
#pragma unroll
        for (int i = 0; i < 16; i++)
#pragma unroll
            for (int e = 0; e < 4; e++) sum[e] += p + i * groups <= last ? v[i][e] : 0.f;
    }
    if constexpr (GROUPS) {
#pragma unroll
        for (int e = 0; e < 4; e++) sums[threadIdx.x][e] = sum[e];
        __syncthreads();
        for (int g = 1; g < groups && group == 0; g++)
#pragma unroll
            for (int e = 0; e < 4; e++) sum[e] += sums[g * per + threadIdx.x][e];
    }
    if (c >= D || group != 0) return;
    sum_on(a, sum, old);
    TG* row = (TG*)a.dtable + k * a.ldt + from;
    if (!NARROW && from == c) {
        store_whole(row, old);
    } else {
#pragma unroll
        for (int e = 0; e < 4; e++)
            if (from + e >= c && from + e < D) row[e] = from_f<TG>(old[e]);
    }
}

// ---------------------------------------------------------------- launches
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

struct EmbSpace {
    int64_t order, key, order1, key1, part, total;
};
EmbSpace emb_space(int64_t M, int64_t D) {
    EmbSpace s{};
    const bool chunks = M > kRankMax;
    s.order = 0;
    s.key = s.order + up256(M * 4);
    s.order1 = s.key + up256(M * 4);
    s.key1 = s.order1 + (chunks ? up256(M * 4) : 0);
    s.part = s.key1 + (chunks ? up256(M * 4) : 0);
    s.total = s.part + up256(ceil_div(M, kRunMin) * 2 * D * 4);
    return s;
}

// Short stretches where long ones leave CUs without work (1000 x 1024 13.4 us, with stretches of 16 16.6; 16384 x 4096 91, of 8 102).
int run_of(int64_t M, int64_t D) { return ceil_div(M, 16) * ceil_div(D, kSumCols) < 1024 ? 8 : 16; }

int sort_passes(int64_t V) {   // bytes of the largest key, V
    int p = 1;
    while (p < 4 && (V >> (8 * p)) > 0) p++;
    return p;
}

constexpr int kSortLds = kSortMax * 8 + kSortWaves * kBins * 2 + 64;

template <typename TG>
hipError_t run_sort(EmbBwdArgs& a, hipStream_t stream) {
    // zeros: many workgroups with a store each (262 MB 43 us; by 1024 that go on 52)
    const int64_t stores = a.ldt == a.D ? ceil_div(a.V * a.D, (int64_t)kSortThreads * CH) : a.V;
    const int64_t zeros = a.accumulate ? 0 : (stores < (1 << 20) ? stores : 1 << 20);
    if (a.M <= kRankMax) {
        a.sorters = (int32_t)ceil_div(a.M, 64);
        if (a.sorters + zeros == 0) return hipSuccess;
        hipLaunchKernelGGL((token_rank_kernel<TG>), dim3((unsigned)(a.sorters + zeros)), dim3(kSortThreads),
                           (unsigned)(a.sorters * 256 + kSortWaves * 256), stream, a);
        return hipGetLastError();
    }
    const hipError_t e = allow_lds<token_sort_kernel<TG>, kSortLds>();
    if (e != hipSuccess) return e;
    a.sorters = (int32_t)ceil_div(a.M, a.chunk);
    const unsigned lds = (unsigned)(ceil_div(a.chunk, kSortThreads) * kSortThreads * 8 + kSortWaves * kBins * 2 + 64);
    hipLaunchKernelGGL((token_sort_kernel<TG>), dim3((unsigned)(a.sorters + zeros)), dim3(kSortThreads), lds, stream, a);
    return hipGetLastError();
}

hipError_t run_merge(const EmbBwdArgs& a, hipStream_t stream) {
    if (a.M <= kMergeMax) {
        const hipError_t e = allow_lds<token_merge_few_kernel, kMergeMax * 4>();
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL(token_merge_few_kernel, dim3((unsigned)ceil_div(a.M, 1024)), dim3(1024), (unsigned)(ceil_div(a.M, 4) * 16), stream, a);
    } else {
        hipLaunchKernelGGL(token_merge_kernel, dim3((unsigned)ceil_div(a.M, 256)), dim3(256), 0, stream, a);
    }
    return hipGetLastError();
}

template <typename T, typename TG>
hipError_t run_sums(const EmbBwdArgs& a, hipStream_t stream) {
    const int64_t runs = ceil_div(a.M, a.run);
    const int slices = (int)ceil_div(a.D, kSumCols);
    const dim3 grid((unsigned)(runs * slices)), block(a.D <= 64 * CH ? 64 : kSumThreads);
    auto launch = [&](auto kind) {
        constexpr int KIND = decltype(kind)::value;
        auto by_run = [&](auto run) {
            constexpr int RUN = decltype(run)::value;
            if (a.accumulate) hipLaunchKernelGGL((token_sum_kernel<T, TG, KIND, true, RUN>), grid, block, 0, stream, a, slices);
            else hipLaunchKernelGGL((token_sum_kernel<T, TG, KIND, false, RUN>), grid, block, 0, stream, a, slices);
        };
        if (a.run == 8) by_run(std::integral_constant<int, 8>());
        else by_run(std::integral_constant<int, 16>());
    };
    if (a.D % CH == 0) launch(std::integral_constant<int, 2>());
    else if (a.D > CH) launch(std::integral_constant<int, 1>());
    else launch(std::integral_constant<int, 0>());
    return hipGetLastError();
}

template <typename TG>
hipError_t run_join(const EmbBwdArgs& a, hipStream_t stream) {
    const int64_t runs = ceil_div(a.M, a.run);
    if (runs < 2) return hipSuccess;
    const int slices = (int)ceil_div(a.D, kJoinCols);
    int groups = 1;
    while (groups < 16 && a.D * 2 * groups <= kJoinCols) groups *= 2;
    auto launch = [&](auto in_groups, auto narrow) {
        hipLaunchKernelGGL((token_join_kernel<TG, decltype(in_groups)::value, decltype(narrow)::value>), dim3((unsigned)(runs * slices)),
                           dim3(256), 0, stream, a, slices, groups);
    };
    if (a.D < 4) launch(std::true_type(), std::true_type());
    else if (groups > 1) launch(std::true_type(), std::false_type());
    else launch(std::false_type(), std::false_type());
    return hipGetLastError();
}

template <typename TT, typename T>
hipError_t run_embedding(EmbArgs a, hipStream_t stream) {
    // a launch holds fewer than 2^32 threads: very many rows go in slabs
    const int64_t M = a.M, slab = ((int64_t)1 << 31) / a.ppr;
    for (int64_t m0 = 0; m0 < M; m0 += slab) {
        a.M = M - m0 < slab ? M - m0 : slab;
        hipLaunchKernelGGL((embedding_kernel<TT, T>), dim3((unsigned)ceil_div(a.M * a.ppr, 256)), dim3(256), 0, stream, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        a.tokens += slab;
        a.out = (T*)a.out + slab * a.ldo;
    }
    return hipSuccess;
}

}  // namespace

size_t embedding_bwd_workspace(int64_t M, int64_t V, int64_t D) {
    return M > 0 && V > 0 && D > 0 && M <= kMaxTokens && V < kMaxDim && D < kMaxLd ? (size_t)emb_space(M, D).total : 0;
}

}  // namespace niti

using namespace niti;

extern "C" {

niti_status niti_embedding_fwd(const void* table, int64_t ldt, int table_type, const float* table_scale, const int32_t* tokens,
                               void* out, int64_t ldout, int64_t M, int64_t V, int64_t D, float alpha, int type, void* stream) {
    if (M < 0 || V < 1 || D < 1) return NITI_ERR_SHAPE;
    if (!valid_type(type) || (table_type != NITI_I8 && !valid_type(table_type)) || !(alpha - alpha == 0.f)) return NITI_ERR_ARG;
    if (M >= kMaxDim || V >= kMaxDim || D >= kMaxLd) return NITI_ERR_UNSUPPORTED;
    if (M == 0) return NITI_OK;
    if (!table || !tokens || !out || (table_type == NITI_I8) != (table_scale != nullptr)) return NITI_ERR_NULL;
    if (bad_ld(V > 1 ? ldt : D, D, false) || bad_ld(M > 1 ? ldout : D, D, true)) return NITI_ERR_SHAPE;
    const EmbArgs a{table, table_scale, tokens, out, V > 1 ? ldt : D, M > 1 ? ldout : D, M, V, D, (uint32_t)((D + CH - 1) / CH), alpha};
    hipStream_t s = (hipStream_t)stream;
    const hipError_t e = by_type(type, [&](auto t) {
        using T = decltype(t);
        if (table_type == NITI_I8) return run_embedding<int8_t, T>(a, s);
        return by_type(table_type, [&](auto tt) { return run_embedding<decltype(tt), T>(a, s); });
    });
    return e == hipSuccess ? NITI_OK : NITI_ERR_HIP;
}

niti_status niti_embedding_bwd(const void* dy, int64_t lddy, int type, const int32_t* tokens, void* dtable, int64_t ldt, int dtable_type,
                               int64_t M, int64_t V, int64_t D, float alpha, int accumulate, void* ws, size_t ws_bytes, void* stream) {
    if (M < 0 || V < 1 || D < 1) return NITI_ERR_SHAPE;
    if (!valid_type(type) || !valid_type(dtable_type) || !(alpha - alpha == 0.f)) return NITI_ERR_ARG;
    if (M > kMaxTokens || V >= kMaxDim || D >= kMaxLd) return NITI_ERR_UNSUPPORTED;
    if (M == 0 && accumulate) return NITI_OK;
    if (!dtable || (M > 0 && (!dy || !tokens))) return NITI_ERR_NULL;
    if ((M > 0 && bad_ld(M > 1 ? lddy : D, D, false)) || bad_ld(V > 1 ? ldt : D, D, true)) return NITI_ERR_SHAPE;
    const EmbSpace w = emb_space(M, D);
    if (M > 0 && (!ws || ws_bytes < (size_t)w.total)) return NITI_ERR_WORKSPACE;
    if (M > 0 && ((uintptr_t)ws & 15)) return NITI_ERR_ARG;
    char* base = (char*)ws;
    const bool chunks = M > kRankMax;
    hipStream_t s = (hipStream_t)stream;
    EmbBwdArgs a{dy, tokens, dtable, M > 1 ? lddy : D, V > 1 ? ldt : D, M, V, D, alpha, accumulate != 0, sort_passes(V), run_of(M, D), 0,
                 (int32_t*)(base + w.order), (int32_t*)(base + w.key), chunks ? (int32_t*)(base + w.order1) : nullptr,
                 chunks ? (int32_t*)(base + w.key1) : nullptr, M <= kMergeMax ? kSortFew : kSortMax, (float*)(base + w.part)};
    hipError_t e = by_type(dtable_type, [&](auto g) { return run_sort<decltype(g)>(a, s); });
    if (e == hipSuccess && chunks) {
        e = run_merge(a, s);
    }
    if (e == hipSuccess && M > 0)
        e = by_type(dtable_type, [&](auto g) {
            return by_type(type, [&](auto t) { return run_sums<decltype(t), decltype(g)>(a, s); });
        });
    if (e == hipSuccess && M > 0) e = by_type(dtable_type, [&](auto g) { return run_join<decltype(g)>(a, s); });
    return e == hipSuccess ? NITI_OK : NITI_ERR_HIP;
}

}  // extern "C"
