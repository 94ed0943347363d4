// What the logits of a language model are read for: log probabilities of given
// tokens with the entropy and the top alternatives, and the divergence from a
// teacher's top logits with its gradient.
//
// With u_v = x_v - max x:  S = sum exp(scale u_v), W = sum u_v exp(scale u_v),
//   lse = scale max + ln S,  log p_v = scale u_v - ln S,  entropy = ln S - scale W / S,
//   dx_v = dloss scale (exp(scale u_v) / S - sum of the p_j of v).
// A row is read once: it stays in the registers of one workgroup (up to 64K columns, in distillation 128K of 16 bits; the plans below) as it
// was loaded, the maximum is found first and the sums next, so that every element costs one exponential; longer rows, and few of
// them, are split over workgroups whose parts a second launch joins.  The fused gradient writes from the same registers; that of split rows reads
// them again, and takes the joined maximum and sum.  Powers below 2^-126 are 0, as the hardware gives them.
// What bounds them: distillation and its gradient memory (4096 x 32000 bf16 with the gradient, 524 MB, 99 us: 5.3 TB/s); log
// probabilities of 16 bits the vector units (4096 x 32000, 262 MB, 62 us, 4.2 TB/s: fourteen instructions an element, of which the
// exponential takes four issue slots) between the barriers of two workgroups a CU, which is what narrower rows from 16385 columns on have too
// (4000 x 20000 54 us for 30 of memory; 4096 x 10000, eight waves, 27 for 15.5); of 32 bits memory, in parts (77 x 128001 14.5 us and
// 5 for the join); one row latency (1 x 32000 7.5 us).  Workgroups that go on to another row, its loads out while the last one's results
// are joined, spilled registers and took 101 us for 69.
//
// The k largest of a row: 64 groups of threads have a maximum each, and the k-th
// largest of those is a bound that at least k logits reach.  Logits that reach it
// (some 25 where k is 20) are collected in any order and placed by counting,
// for each, those before it: larger, or equal with a lower column.  Where more than kCand reach the bound
// (masked rows whose bound is minus infinity, many equal ones) the k-th value is found by bisection on its bits, and
// its equals are taken in the order of their columns.
#include "linear.h"

#include <math.h>

#include <algorithm>
#include <initializer_list>
#include <type_traits>

namespace niti {

namespace {

constexpr int kTopMax = 64;     // alternatives of a row
constexpr int kListMax = 256;   // teacher's logits of a row
constexpr int kCand = 512;      // collected logits of a row
constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f;
constexpr uint32_t kNegInf = 0xFF800000u;

__device__ __forceinline__ float neg_inf() { return __uint_as_float(kNegInf); }
__device__ __forceinline__ float quiet_nan() { return __uint_as_float(0x7FC00000u); }

// Integers of the order of floats (no NaN among them; both zeros alike), and the float of one.
__device__ __forceinline__ uint32_t order_key(float v) {
    const uint32_t b = __float_as_uint(v + 0.f);
    return b ^ (b >> 31 ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k) { return __uint_as_float(k ^ (k >> 31 ? 0x80000000u : 0xFFFFFFFFu)); }
// Of two logits the one with the larger rank stands first: by value, then by column.
__device__ __forceinline__ uint64_t rank_of(float v, int col) { return (uint64_t)order_key(v) << 32 | (uint32_t)~col; }
__device__ __forceinline__ int rank_col(uint64_t r) { return (int)~(uint32_t)r; }

// ---------------------------------------------------------------- reductions
// Row-local steps of a wave: after the first two, four neighbouring lanes have the same, after three, eight, after four, sixteen.
template <int CTRL>
__device__ __forceinline__ float lane_step(float v) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xF, 0xF, false));
}
__device__ __forceinline__ float lane_of(float v, int lane) { return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), lane)); }
__device__ __forceinline__ float max_of_4(float v) {
    v = fmaxf(v, lane_step<0xB1>(v));
    return fmaxf(v, lane_step<0x4E>(v));
}
__device__ __forceinline__ float max_of_8(float v) {
    v = max_of_4(v);
    return fmaxf(v, lane_step<0x141>(v));
}
__device__ __forceinline__ float max_of_16(float v) {
    v = max_of_8(v);
    return fmaxf(v, lane_step<0x140>(v));
}
__device__ __forceinline__ float max_of_rows(float v) {   // sixteen lanes have the same
    return fmaxf(fmaxf(lane_of(v, 0), lane_of(v, 16)), fmaxf(lane_of(v, 32), lane_of(v, 48)));
}
__device__ __forceinline__ float wave_max(float v) { return max_of_rows(max_of_16(v)); }
__device__ __forceinline__ float wave_sum(float v) {
    v += lane_step<0xB1>(v);
    v += lane_step<0x4E>(v);
    v += lane_step<0x141>(v);
    v += lane_step<0x140>(v);
    return (lane_of(v, 0) + lane_of(v, 16)) + (lane_of(v, 32) + lane_of(v, 48));
}
// Of the NW values that the waves left in LDS, each lane reading one of them; uniform.  (As all lane steps: by whole waves.)
template <int NW>
__device__ __forceinline__ float join_max(const float* red) {
    const float v = red[threadIdx.x & (NW - 1)];
    if constexpr (NW == 1) return lane_of(v, 0);
    if constexpr (NW == 4) return lane_of(max_of_4(v), 0);
    if constexpr (NW == 8) return lane_of(max_of_8(v), 0);
    return lane_of(max_of_16(v), 0);
}
template <int NW>
__device__ __forceinline__ float join_sum(const float* red) {
    float v = red[threadIdx.x & (NW - 1)];
    if constexpr (NW > 1) {
        v += lane_step<0xB1>(v);
        v += lane_step<0x4E>(v);
    }
    if constexpr (NW > 4) v += lane_step<0x141>(v);
    if constexpr (NW > 8) v += lane_step<0x140>(v);
    return lane_of(v, 0);
}

// ---------------------------------------------------------------- a row in registers
// Eight logits of column c on, as they are loaded.  No load is in a branch, where it would be waited for: the
// row's last piece is loaded from eight columns before its end, and its first `down` elements, which belong to the piece before it
// (past the row: all eight), count for nothing.  TINY: rows of fewer than eight.
template <bool TINY>
struct Place {
    int from, down, end;   // elements down .. end - 1 are the piece's own, of columns from + e
    __device__ __forceinline__ Place(int c, int V) {
        from = TINY ? c : min(c, V - CH);
        down = TINY ? 0 : c - from;
        end = TINY ? V - c : CH;
    }
    __device__ __forceinline__ bool own(int e) const { return e >= down && (!TINY || e < end); }
    __device__ __forceinline__ bool whole() const { return !TINY && down == 0; }
};

template <typename T, bool TINY>
__device__ __forceinline__ Piece<T> load_logits(const T* row, int c, int V) {
    Piece<T> p;
    if constexpr (TINY) {
        T t[CH];
#pragma unroll
        for (int e = 0; e < CH; e++) t[e] = row[min(c + e, V - 1)];
        __builtin_memcpy(p.w, t, sizeof(t));
    } else {
        __builtin_memcpy(p.w, row + min(c, V - CH), sizeof(p.w));
    }
    return p;
}
template <typename T>
__device__ __forceinline__ void logit_values(const Piece<T>& p, float (&v)[CH]) {
#pragma unroll
    for (int e = 0; e < CH; e++) {   // (halves by shifts: taken from a copy as an array, fp16 stayed apart in two registers a word)
        if constexpr (sizeof(T) == 2) v[e] = to_f(__builtin_bit_cast(T, (uint16_t)(p.w[e / 2] >> (e % 2 * 16))));
        else v[e] = __uint_as_float(p.w[e]);
    }
}
// A wave's pieces that are whole, and those that have any columns of the row: the others cost no arithmetic (10000 columns in a
// workgroup's 16384: log probabilities of 4096 rows of bf16 42.3 -> 27.3 us).  left: columns from the workgroup's first to the row's end.
template <int NW, int VPT>
struct Live {
    int whole, all;
    __device__ __forceinline__ Live(int left, int wave) {
        constexpr int STEP = 64 * NW * CH;
        const int mine = left - wave * 64 * CH;
        whole = min(max(mine - 64 * CH + STEP, 0) / STEP, VPT);
        all = min(max(mine + STEP - 1, 0) / STEP, VPT);
    }
};

// Minus infinity in the place of the elements that are not the piece's own.
template <typename T, bool TINY>
__device__ __forceinline__ void mask_logits(Piece<T>& p, int c, int V) {
    const Place<TINY> at(c, V);
    if (at.whole()) return;
    constexpr int BITS = 8 * sizeof(T), IN = 32 / BITS;   // elements in a word
    const uint32_t mask = sizeof(T) == 4 ? kNegInf : (std::is_same_v<T, f16> ? 0xFC00u : 0xFF80u);
#pragma unroll
    for (int e = 0; e < CH; e++) {
        const uint32_t mine = (uint32_t)(((uint64_t)1 << BITS) - 1) << (e % IN * BITS);
        p.w[e / IN] = at.own(e) ? p.w[e / IN] : (p.w[e / IN] & ~mine) | mask << (e % IN * BITS);
    }
}
template <typename T, bool TINY>
__device__ __forceinline__ void store_logits(T* row, int c, int V, const float (&v)[CH], bool stream) {
    const Place<TINY> at(c, V);
    if (at.whole() && stream) {
        store_whole<true>(row + c, v);
    } else if (at.whole()) {
        store_whole(row + c, v);
    } else {
#pragma unroll
        for (int e = 0; e < CH; e++)
            if (at.own(e)) row[at.from + e] = from_f<T>(v[e]);
    }
}
// p[want], want uniform, by selects over constant indices: the pieces stay in registers.
template <typename T, int VPT>
__device__ __forceinline__ Piece<T> pick(const Piece<T> (&p)[VPT], int want) {
    Piece<T> x = p[0];
#pragma unroll
    for (int i = 1; i < VPT; i++)
#pragma unroll
        for (int w = 0; w < (int)(sizeof(x.w) / 4); w++) x.w[w] = want == i ? p[i].w[w] : x.w[w];
    return x;
}

// What exponents of a row are taken from.  With c2 = scale log2 e an element's power is 2^(x c2 - mc), one multiply-add,
// with mc = m c2 rounded; all of a row's are 2^r times too large, r = m c2 - mc, which the sums are freed of once.  Where
// |m c2| is above 2^30 (a row of a type's lowest value, say) that r could be large; but whatever is not equal to m is then 2^6 or more
// below it (a step of 32 bits is 2^-24 of a value), its power nothing beside that of m.  A power of two in c2's place, with
// which m c2 is exact and any other value 2^100 below it, keeps the equals and drops the others.
struct Base {
    float c2, mc, r;
    __device__ __forceinline__ Base(float top, float c) {   // (a row without a maximum: 0 in its place)
        const float m = top == neg_inf() ? 0.f : top;
        const uint32_t expo = __float_as_uint(m) >> 23 & 255u;
        const bool far = fabsf(m * c) > 0x1p30f && expo < 255u;
        c2 = far ? __uint_as_float((min(380u - expo, 254u)) << 23) : c;   // 2^126 over m's power of two
        mc = m * c2;
        r = __builtin_fmaf(m, c2, -mc);
    }
    __device__ __forceinline__ float arg(float x) const { return __builtin_fmaf(x, c2, -mc); }
    __device__ __forceinline__ float power(float x) const { return __builtin_amdgcn_exp2f(arg(x)); }
};

// A row's (or a part's) statistics: the maximum, S = sum 2^u and W = sum u 2^u of u = (x - m) c2.  A row
// of minus infinities has -inf, 0 and 0; a NaN or an infinity in the row leaves a NaN in S.
struct Stat {
    float m, s, w;
    __device__ __forceinline__ bool empty() const { return m == neg_inf() && s == 0.f; }
    __device__ __forceinline__ float log() const { return logf(s); }
    __device__ __forceinline__ float base() const { return m == neg_inf() ? 0.f : m; }
    __device__ __forceinline__ float lse(float scale, float logs) const { return empty() ? neg_inf() : scale * base() + logs; }
    __device__ __forceinline__ float logp(float scale, float logs, float x) const { return empty() ? neg_inf() : scale * (x - base()) - logs; }
    __device__ __forceinline__ float entropy(float logs) const { return empty() ? 0.f : logs - kLn2 * (w / s); }
};

// The pieces are converted anew in each pass over them: converted values that stay would take twice the registers.
template <typename T, int VPT>
__device__ __forceinline__ void forget_values(Piece<T> (&p)[VPT]) {
#pragma unroll
    for (int i = 0; i < VPT; i++)
#pragma unroll
        for (int w = 0; w < (int)(sizeof(p[i].w) / 4); w++) asm volatile("" : "+v"(p[i].w[w]));
}
// S and W over a thread's pieces, both as their powers are; KEEP: the powers stay in e.  GUARD: there may be minus
// infinities, whose terms of W are 0; without it they leave W a NaN.
template <typename T, int NW, int VPT, bool WANT_W, bool KEEP, bool GUARD>
__device__ __forceinline__ void row_sums(Piece<T> (&p)[VPT], const Live<NW, VPT>& live, const Base& b, float& s, float& w,
                                         float (&e)[KEEP ? VPT : 1][CH]) {
    if (sizeof(T) == 2) forget_values(p);
    s = w = 0.f;
#pragma unroll
    for (int i = 0; i < VPT; i++) {
        auto add = [&](auto guard) {
            float v[CH];
            logit_values(p[i], v);
#pragma unroll
            for (int k = 0; k < CH; k++) {
                const float u = b.arg(v[k]), x = __builtin_amdgcn_exp2f(u);
                s += x;
                if (WANT_W) w = __builtin_fmaf(x, decltype(guard)::value ? fmaxf(u, -0x1p100f) : u, w);
                if (KEEP) e[i][k] = x;
            }
        };
        constexpr bool BOTH = WANT_W && !GUARD;   // (past the row's end there are minus infinities)
        if (i < (BOTH ? live.whole : live.all)) add(std::integral_constant<bool, GUARD>());
        else if (BOTH && i < live.all) add(std::true_type());
    }
    if (sizeof(T) == 2 && !KEEP) forget_values(p);
}

// The larger of three.  (fmaxf would first quiet signalling NaNs, one instruction for each; what one
// does to a maximum does not matter: its row is NaN by its power.  The compiler does not know the
// instruction's result for one that a lane step has to wait for: it goes through an operation of its own first.)
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}
// A thread's largest, and that of each piece.
template <typename T, int NW, int VPT>
__device__ __forceinline__ float max_of(const Piece<T> (&p)[VPT], const Live<NW, VPT>& live, float (&top)[VPT]) {
    float mx = neg_inf();
#pragma unroll
    for (int i = 0; i < VPT; i++) {
        top[i] = neg_inf();
        if (i >= live.all) continue;
        float v[CH];
        logit_values(p[i], v);
        top[i] = max3(max3(max3(v[0], v[1], v[2]), v[3], v[4]), v[5], v[6]);
        top[i] = fmaxf(top[i], v[7]);
        mx = fmaxf(mx, top[i]);
    }
    return mx;
}

// ---------------------------------------------------------------- log probabilities
struct LogArgs {
    const void* x;
    const int32_t* tokens;
    float *logp, *lse, *entropy, *top_logp;
    int32_t* top_idx;
    int64_t ldx, M, V;
    int32_t top, parts;
    float scale, c2;
    // Parts of split rows: [M][parts] statistics, [M][parts][top] ranks in order (0: fewer logits than that).
    Stat* stat;
    uint64_t* ranks;
};

// A row's scalars, by one thread.
__device__ __forceinline__ void put_scalars(const LogArgs& a, int64_t m, const Stat& st, float logs, int tok, float x) {
    if (a.logp) a.logp[m] = (uint32_t)tok < (uint64_t)a.V ? st.logp(a.scale, logs, x) : 0.f;
    if (a.lse) a.lse[m] = st.lse(a.scale, logs);
    if (a.entropy) a.entropy[m] = st.entropy(logs);
}
// Alternative r of a row; rank 0: none.
__device__ __forceinline__ void put_top(const LogArgs& a, int64_t m, int r, const Stat& st, float logs, uint64_t rank) {
    const bool bad = !(st.s == st.s) || rank == 0;
    if (a.top_logp) a.top_logp[m * a.top + r] = bad ? quiet_nan() : st.logp(a.scale, logs, key_value((uint32_t)(rank >> 32)));
    if (a.top_idx) a.top_idx[m * a.top + r] = bad ? -1 : rank_col(rank);
}

// The largest of 64 values (in LDS, 16-byte aligned; each lane's own in g) that at least k of them reach.  By one wave.
__device__ __forceinline__ float bound_of(const float* values, float g, int k) {
    int reach = 0;
#pragma unroll
    for (int j = 0; j < 16; j++) {
        const v4f x = *(const v4f*)(values + 4 * j);
#pragma unroll
        for (int i = 0; i < 4; i++) reach += x[i] >= g ? 1 : 0;
    }
    return wave_max(reach >= k ? g : neg_inf());
}

// Adds n to a counter in LDS for each lane by itself (the compiler would first join the lanes, one after the other).
__device__ __forceinline__ int lds_add(int* p, int n) {
    int old;
    asm volatile("ds_add_rtn_u32 %0, %1, %2\n\ts_waitcnt lgkmcnt(0)" : "=v"(old) : "v"(lds_address(p)), "v"(n) : "memory");
    return old;
}

// The top logits of a workgroup's columns: kCand places for the logits that reach a bound, placed by counting.
template <typename T, int NW, int VPT, bool TINY>
struct Select {
    static constexpr int NT = 64 * NW;
    uint64_t* cand;      // [kCand]
    int* n;              // zeroed by the caller, who has a barrier after it
    int (*red)[NW];      // [2][NW]
    int c0, V;

    // hits(v, e, at): f gets a piece's hits as a mask, its values and its place
    template <typename Hit, typename F>
    __device__ __forceinline__ void piece(const Piece<T>& x, int i, Hit hit, F f) {
        const Place<TINY> at(c0 + (i * NT + (int)threadIdx.x) * CH, V);
        float v[CH];
        logit_values(x, v);
        uint32_t mask = 0;
#pragma unroll
        for (int e = 0; e < CH; e++) mask |= (hit(v[e]) && at.own(e) ? 1u : 0u) << e;
        f(mask, v, at.from);
    }
    // All above tau (or: equal to it as well), in any order; what is past kCand is only counted.
    __device__ __forceinline__ void collect(const Piece<T> (&p)[VPT], const float (&tops)[VPT], float tau, bool equal) {
#pragma unroll
        for (int i = 0; i < VPT; i++)
            if (tops[i] > tau || (equal && tops[i] == tau))
                piece(p[i], i, [&](float v) { return v > tau || (equal && v == tau); },
                      [&](uint32_t mask, const float (&v)[CH], int from) {
                          int at = lds_add(n, __popc(mask));
#pragma unroll
                          for (int e = 0; e < CH; e++)
                              if (mask >> e & 1) {
                                  if (at < kCand) cand[at] = rank_of(v[e], from + e);
                                  at++;
                              }
                      });
    }
    // The `need` equals of tau with the lowest columns, behind the first n0.
    __device__ __forceinline__ int equals(const Piece<T> (&p)[VPT], float tau, int n0, int need) {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        int got = 0;
#pragma unroll 1
        for (int i = 0; i < VPT && got < need; i++)   // (the same for all threads)
            piece(pick(p, i), i, [&](float v) { return v == tau; }, [&](uint32_t mask, const float (&v)[CH], int from) {
                int incl = __popc(mask);
#pragma unroll
                for (int o = 1; o < 64; o *= 2) {
                    const int u = __shfl_up(incl, o, kWave);
                    incl += lane >= o ? u : 0;
                }
                int (&r)[NW] = red[i & 1];   // a wave that is a piece ahead writes the other half
                if (lane == 63) r[wave] = incl;
                __syncthreads();
                int at = got + incl - __popc(mask), all = 0;
#pragma unroll 1
                for (int w = 0; w < NW; w++) {
                    at += w < wave ? r[w] : 0;
                    all += r[w];
                }
#pragma unroll
                for (int e = 0; e < CH; e++)
                    if (mask >> e & 1) {
                        if (at < need) cand[n0 + at] = rank_of(v[e], from + e);
                        at++;
                    }
                got += all;
            });
        return min(got, need);
    }
    // The key of the k-th largest, by bisection on its bits.
    __device__ __forceinline__ uint32_t kth(const Piece<T> (&p)[VPT], int k) {
        uint32_t key = 0;
#pragma unroll 1
        for (int b = 31; b >= 0; b--) {
            const uint32_t want = key | 1u << b;
            int c = 0;
#pragma unroll 1
            for (int i = 0; i < VPT; i++)
                piece(pick(p, i), i, [&](float v) { return v == v && order_key(v) >= want; },
                      [&](uint32_t mask, const float (&)[CH], int) { c += __popc(mask); });
#pragma unroll
            for (int o = 32; o >= 1; o >>= 1) c += __shfl_xor(c, o, kWave);
            int (&r)[NW] = red[b & 1];
            if ((threadIdx.x & 63) == 0) r[threadIdx.x >> 6] = c;
            __syncthreads();
            c = 0;
#pragma unroll 1
            for (int w = 0; w < NW; w++) c += r[w];
            if (c >= k) key = want;
        }
        return key;
    }
    // Number of candidates, among them the top ones; tops: the pieces' largest.
    __device__ __forceinline__ int run(Piece<T> (&p)[VPT], const float (&tops)[VPT], float tau, int top) {
        int count, pass = 0;
#pragma unroll 1
        for (;; pass++) {   // all that reach the bound; if too many, those above it; if too many, those above the top-th
            forget_values(p);                // (and nothing that every pass needs is formed, and kept, before the first)
            asm volatile("" : "+s"(V));
            collect(p, tops, tau, pass == 0);
            __syncthreads();
            count = *n;
            if (count <= kCand) break;
            if (pass == 1) tau = key_value(kth(p, top));
            __syncthreads();
            if (threadIdx.x == 0) *n = 0;
            __syncthreads();
        }
        // (the first pass has the bound's equals already: fewer than top are all the numbers that there are)
        if (pass > 0 && count < top) {
            count += equals(p, tau, count, top - count);
            __syncthreads();
        }
        return count;
    }
};

// Waves that a SIMD is to hold: two workgroups of sixteen a CU, one loading while the other computes, where 64 registers do.
template <typename T>
constexpr int two_a_cu(int nw, int vpt) { return nw == 16 && vpt <= 4 && vpt * (int)sizeof(T) <= 8 ? 8 : 1; }

template <typename T, int NW, int VPT, bool TINY>
__global__ __launch_bounds__(64 * NW, two_a_cu<T>(NW, VPT)) void logprobs_kernel(LogArgs a) {
    constexpr int NT = 64 * NW, LEN = NT * VPT * CH;
    __shared__ float red_m[NW], red_s[NW], red_w[NW], tau_s;
    __shared__ __attribute__((aligned(16))) float group[64];
    __shared__ int red_c[2][NW], n_s;
    __shared__ uint64_t cand[kCand];
    const int t = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int64_t m = blockIdx.x / (uint32_t)a.parts;
    const int part = blockIdx.x % (uint32_t)a.parts, V = (int)a.V, c0 = part * LEN;
    const T* row = (const T*)a.x + m * a.ldx;
    const int tok = a.parts == 1 && a.tokens ? a.tokens[m] : -1;
    const Live<NW, VPT> live(V - c0, wave);
    Piece<T> p[VPT];
#pragma unroll
    for (int i = 0; i < VPT; i++) p[i] = load_logits<T, TINY>(row, c0 + (i * NT + t) * CH, V);
    const T x_tok = row[(uint32_t)tok < (uint32_t)V ? tok : 0];
    if (t == 0) n_s = 0;
#pragma unroll
    for (int i = 0; i < VPT; i++)
        if (i >= live.whole && i < live.all) mask_logits<T, TINY>(p[i], c0 + (i * NT + t) * CH, V);
    float top[VPT];
    const float mx = max_of(p, live, top);
    const float x_of_tok = lane_of(to_f(x_tok), 0);   // (the same in all lanes, as some below: in a scalar register)
    // 64 groups of NW neighbouring threads
    const float m16 = max_of_16(mx), of_group = NW == 1 ? mx : (NW == 4 ? max_of_4(mx) : (NW == 8 ? max_of_8(mx) : m16));
    if (t % NW == 0) group[t / NW] = of_group;   // (lane steps take all lanes: none of them in a branch)
    const float wm = max_of_rows(m16);
    if ((t & 63) == 0) red_m[wave] = wm;
    __syncthreads();
    Stat st;
    st.m = join_max<NW>(red_m);
    if (a.top && wave == 0) {
        const float tau = bound_of(group, group[t], a.top);
        if (t == 0) tau_s = tau;
    }
    const Base base(st.m, a.c2);
    float none[1][CH];
    row_sums<T, NW, VPT, true, false, false>(p, live, base, st.s, st.w, none);
    if (__any(st.w != st.w)) row_sums<T, NW, VPT, true, false, true>(p, live, base, st.s, st.w, none);   // masks here
    st.s = wave_sum(st.s);
    st.w = wave_sum(st.w);
    if ((t & 63) == 0) red_s[wave] = st.s, red_w[wave] = st.w;
    __syncthreads();
    const float back = __builtin_amdgcn_exp2f(-base.r);
    st.s = lane_of(join_sum<NW>(red_s) * back, 0);
    st.w = lane_of(join_sum<NW>(red_w) * back - base.r * st.s, 0);
    const float logs = lane_of(st.log(), 0);
    if (t == 0) {
        if (a.parts == 1) put_scalars(a, m, st, logs, tok, x_of_tok);
        else a.stat[m * a.parts + part] = st;
    }
    if (!a.top) return;
    Select<T, NW, VPT, TINY> sel{cand, &n_s, red_c, c0, V};
    const int n = sel.run(p, top, tau_s, a.top);
    auto put = [&](int r, uint64_t rank) {
        if (a.parts == 1) put_top(a, m, r, st, logs, rank);
        else a.ranks[(m * a.parts + part) * a.top + r] = rank;
    };
    for (int j = t; j < n; j += NT) {
        const uint64_t mine = cand[j];
        int r = 0;
        for (int i = 0; i < n; i++) r += cand[i] > mine ? 1 : 0;
        if (r < a.top) put(r, mine);
    }
    for (int r = n + t; r < a.top; r += NT) put(r, 0);   // fewer logits than that in this part, or NaNs among them
}

// Statistics of a row from those of its parts, by all 64 lanes of a wave, in an order fixed by the number of parts.
__device__ __forceinline__ Stat join_stats(const Stat* parts, int n, float c2) {
    const int lane = threadIdx.x & 63;
    Stat p = lane < n ? parts[lane] : Stat{neg_inf(), 0.f, 0.f};
    Stat st;
    st.m = wave_max(p.m);
    // W = sum f (W_i + d S_i) with f = 2^d; a part of minus infinities (base 0, whatever the row's is) adds nothing
    const float d = p.s == 0.f ? 0.f : (p.base() - st.base()) * c2, f = __builtin_amdgcn_exp2f(d);
    st.s = wave_sum(f * p.s);
    st.w = wave_sum(f * (p.w + fmaxf(d, -0x1p100f) * p.s));
    return st;
}

constexpr int kPartsMax = 64;   // parts of a row

// Joins a row's parts: 256 threads.  Every part's k candidates are in order, so the (r + 1)-st of
// each of j parts with j (r + 1) >= k bounds the k-th of the row.
template <typename T>
__global__ __launch_bounds__(256) void logprobs_join_kernel(LogArgs a) {
    __shared__ uint64_t cand[kPartsMax * kTopMax];
    __shared__ __attribute__((aligned(16))) float group[64];
    __shared__ float tau_s;
    __shared__ int n_s;
    const int t = threadIdx.x;
    const int64_t m = blockIdx.x;
    const int top = a.top, parts = a.parts;
    const int tok = a.tokens ? a.tokens[m] : -1;
    const T x_tok = ((const T*)a.x + m * a.ldx)[(uint32_t)tok < (uint32_t)a.V ? tok : 0];
    const uint64_t* ranks = a.ranks + m * parts * top;
    const Stat st = join_stats(a.stat + m * parts, parts, a.c2);
    if (t == 0) n_s = 0;
    if (top && t < 64) {
        const int r = (top + parts - 1) / parts - 1, j = (top + r) / (r + 1);
        const float g = t < parts && ranks[t * top + r] != 0 ? key_value((uint32_t)(ranks[t * top + r] >> 32)) : neg_inf();
        group[t] = g;
        __builtin_amdgcn_wave_barrier();
        const float tau = bound_of(group, g, j);
        if (t == 0) tau_s = tau;
    }
    const float logs = st.log();
    if (t == 0) put_scalars(a, m, st, logs, tok, to_f(x_tok));
    if (!top) return;
    __syncthreads();
    const float tau = tau_s;
    for (int i = t; i < parts * top; i += 256) {
        const uint64_t rank = ranks[i];
        if (rank != 0 && key_value((uint32_t)(rank >> 32)) >= tau) cand[lds_add(&n_s, 1)] = rank;
    }
    __syncthreads();
    const int n = n_s;
    for (int j = t; j < n; j += 256) {
        const uint64_t mine = cand[j];
        int r = 0;
        for (int i = 0; i < n; i++) r += cand[i] > mine ? 1 : 0;
        if (r < top) put_top(a, m, r, st, logs, mine);
    }
    for (int r = n + t; r < top; r += 256) put_top(a, m, r, st, logs, 0);
}

// ---------------------------------------------------------------- distillation
struct DistArgs {
    const void* x;
    const void* t_val;
    const int32_t* t_idx;
    float *loss, *lse;
    const float* lse_in;   // of the backward pass
    const float* dloss;
    void* dx;
    int64_t ldx, ldt, ldi, lddx, M, V;
    int32_t top, t_type, parts, g_step, stream;
    float scale, c2;
    Stat* stat;            // [M][stats] of split rows' parts; the first then the whole row's
    int64_t stats;
};

// The teacher's distribution over its list: KPT entries a thread.
template <int NW, int KPT>
struct Teacher {
    int col[KPT];     // -1: no entry, or a column outside the row
    float t[KPT], p[KPT], logp[KPT];
    bool any;         // whether the list has a probability
    float unit;       // 1; NaN for a list with a NaN or an infinity
    uint32_t wide[KPT];
    uint16_t narrow[KPT];
    // Of two places to load from, by the type, the other is a stand-in: no load is in a branch.
    __device__ __forceinline__ void load(const DistArgs& a, int64_t m) {
        const bool f32 = a.t_type == NITI_F32;
#pragma unroll
        for (int i = 0; i < KPT; i++) {
            const int j = min(i * 64 * NW + (int)threadIdx.x, a.top - 1);
            col[i] = a.t_idx[m * a.ldi + j];
            wide[i] = (f32 ? (const uint32_t*)a.t_val : (const uint32_t*)a.t_idx)[f32 ? m * a.ldt + j : m * a.ldi + j];
            narrow[i] = (f32 ? (const uint16_t*)a.t_idx : (const uint16_t*)a.t_val)[f32 ? m * a.ldi + j : m * a.ldt + j];
        }
    }
    // The row's logits at the listed columns from c0 to c1 (any other: that of c0).
    template <typename T>
    __device__ __forceinline__ void gather(const DistArgs& a, const T* row, int c0, int c1, T (&z)[KPT]) {
#pragma unroll
        for (int i = 0; i < KPT; i++) {
            const bool in = i * 64 * NW + (int)threadIdx.x < a.top && (uint32_t)col[i] < (uint64_t)a.V;
            col[i] = in ? col[i] : -1;
            z[i] = row[col[i] >= c0 && col[i] < c1 ? col[i] : c0];
        }
    }
    __device__ __forceinline__ float top(const DistArgs& a) {   // this thread's largest
        float mx = neg_inf();
#pragma unroll
        for (int i = 0; i < KPT; i++) {
            const uint16_t h = narrow[i];
            const float half = a.t_type == NITI_F16 ? to_f(__builtin_bit_cast(f16, h)) : to_f(bf16{h});
            t[i] = col[i] < 0 ? neg_inf() : (a.t_type == NITI_F32 ? __uint_as_float(wide[i]) : half);
            mx = fmaxf(mx, t[i]);
        }
        return mx;
    }
    __device__ __forceinline__ float powers(const DistArgs& a, float mx) {   // this thread's sum
        const float base = mx == neg_inf() ? 0.f : mx;
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < KPT; i++) {
            t[i] -= base;
            p[i] = __builtin_amdgcn_exp2f(t[i] * a.c2);
            s += p[i];
        }
        return s;
    }
    __device__ __forceinline__ void form(const DistArgs& a, float s) {
        any = __builtin_amdgcn_readfirstlane(s != 0.f);
        unit = s / s;
        const float logs = logf(s);
#pragma unroll
        for (int i = 0; i < KPT; i++) {
            p[i] = any ? p[i] / s : 0.f;
            logp[i] = a.scale * t[i] - logs;
        }
    }
    // This thread's terms of the loss.
    template <typename T>
    __device__ __forceinline__ float loss(const DistArgs& a, const T (&z)[KPT], const Stat& st, float logs) const {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < KPT; i++) {
            const float term = p[i] * (logp[i] - st.logp(a.scale, logs, to_f(z[i])));
            s += p[i] == 0.f ? 0.f : term;
        }
        return s;
    }
    __device__ __forceinline__ void put(const DistArgs& a, int* cols, float* probs) const {   // for all threads; kListMax of each
#pragma unroll
        for (int i = 0; i < KPT; i++) {
            const int j = i * 64 * NW + (int)threadIdx.x;
            if (j < kListMax) cols[j] = j < a.top ? col[i] : -1, probs[j] = p[i];
        }
    }
    // The listed columns' own gradients, from c0 to c1, after the whole row's: a column that is listed twice has both probabilities.
    template <typename T>
    __device__ __forceinline__ void store(const DistArgs& a, T* dx, const int* cols, const float* probs, const float (&q)[KPT], float g,
                                          int c0, int c1) const {
#pragma unroll
        for (int i = 0; i < KPT; i++) {
            const int mine = col[i];
            if (mine < 0 || mine < c0 || mine >= c1) continue;
            float s = 0.f;
            for (int j = 0; j < a.top; j += 4) {   // (entries past the list: column -1)
                const v4i c = *(const v4i*)(cols + j);
                const v4f x = *(const v4f*)(probs + j);
#pragma unroll
                for (int e = 0; e < 4; e++) s += c[e] == mine ? x[e] : 0.f;
            }
            dx[mine] = from_f<T>(g * (q[i] - s));
        }
    }
};

constexpr int list_per_thread(int nw) { return nw >= 4 ? 1 : 4; }

// Loss of a row (GRAD: and its gradient) by one workgroup, or a part's statistics.
template <typename T, int NW, int VPT, bool TINY, bool GRAD>
__global__ __launch_bounds__(64 * NW, two_a_cu<T>(NW, VPT)) void distill_kernel(DistArgs a) {
    constexpr int NT = 64 * NW, LEN = NT * VPT * CH, KPT = list_per_thread(NW);
    constexpr bool KEEP = GRAD && VPT <= 8;   // the powers of the sum serve the gradient: with more, they find no registers
    __shared__ float red_m[NW], red_s[NW], red_t[NW], red_u[NW], red_l[NW];
    __shared__ __attribute__((aligned(16))) int cols[kListMax];
    __shared__ __attribute__((aligned(16))) float probs[kListMax];
    const int t = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int64_t m = blockIdx.x / (uint32_t)a.parts;
    const int part = blockIdx.x % (uint32_t)a.parts, V = (int)a.V, c0 = part * LEN;
    const T* row = (const T*)a.x + m * a.ldx;
    Teacher<NW, KPT> teach;
    teach.load(a, m);
    const float g1 = GRAD && a.dloss ? a.dloss[a.g_step ? m : 0] : 1.f;
    const Live<NW, VPT> live(V - c0, wave);
    Piece<T> p[VPT];
#pragma unroll
    for (int i = 0; i < VPT; i++) p[i] = load_logits<T, TINY>(row, c0 + (i * NT + t) * CH, V);
    T z[KPT];
    teach.gather(a, row, 0, V, z);
#pragma unroll
    for (int i = 0; i < VPT; i++)
        if (i >= live.whole && i < live.all) mask_logits<T, TINY>(p[i], c0 + (i * NT + t) * CH, V);
    float tops[VPT];
    const float wm = wave_max(max_of(p, live, tops)), wt = wave_max(teach.top(a));
    if ((t & 63) == 0) red_m[wave] = wm, red_t[wave] = wt;
    __syncthreads();
    Stat st;
    st.m = join_max<NW>(red_m);
    const Base base(st.m, a.c2);
    float e[KEEP ? VPT : 1][CH];
    row_sums<T, NW, VPT, false, KEEP, false>(p, live, base, st.s, st.w, e);
    const float ws = wave_sum(st.s), wu = wave_sum(teach.powers(a, join_max<NW>(red_t)));
    if ((t & 63) == 0) red_s[wave] = ws, red_u[wave] = wu;
    __syncthreads();
    const float sum = join_sum<NW>(red_s);   // as the powers are
    st.s = sum * __builtin_amdgcn_exp2f(-base.r);
    st.w = 0.f;
    if (a.parts > 1) {
        if (t == 0) a.stat[m * a.stats + part] = st;
        return;
    }
    const float logs = st.log();
    teach.form(a, join_sum<NW>(red_u));
    const float wl = wave_sum(teach.loss(a, z, st, logs));
    if ((t & 63) == 0) red_l[wave] = wl;
    if (GRAD) teach.put(a, cols, probs);
    if constexpr (GRAD) {
        // Every load of the row has returned, here and, past the barriers above, in the other waves: dx may be x.
        const float inv = sum == 0.f ? 0.f : 1.f / sum, g = g1 * a.scale * teach.unit, f = g * inv;
        T* dx = (T*)a.dx + m * a.lddx;
#pragma unroll
        for (int i = 0; i < VPT; i++) {
            if (i >= live.all) continue;
            float v[CH];
            if constexpr (!KEEP) logit_values(p[i], v);
            if (teach.any) {   // (uniform)
#pragma unroll
                for (int k = 0; k < CH; k++) v[k] = (KEEP ? e[KEEP ? i : 0][k] : base.power(v[k])) * f;
            } else {
#pragma unroll
                for (int k = 0; k < CH; k++) v[k] = 0.f;
            }
            const int c = (i * NT + t) * CH;
            if (c < V) store_logits<T, TINY>(dx, c, V, v, a.stream);
        }
        __syncthreads();   // the row's stores before the listed columns'
        if (teach.any) {
            float q[KPT];
#pragma unroll
            for (int i = 0; i < KPT; i++) q[i] = base.power(to_f(z[i])) * inv;
            teach.store(a, dx, cols, probs, q, g, 0, V);
        }
    } else {
        __syncthreads();
    }
    const float loss = join_sum<NW>(red_l);
    if (t == 0) {
        a.loss[m] = loss;
        if (a.lse) a.lse[m] = st.lse(a.scale, logs);
    }
}

// Joins a row's parts: 256 threads.
template <typename T>
__global__ __launch_bounds__(256) void distill_join_kernel(DistArgs a) {
    __shared__ float red_t[4], red_u[4], red_l[4];
    const int t = threadIdx.x, wave = t >> 6;
    const int64_t m = blockIdx.x;
    const T* row = (const T*)a.x + m * a.ldx;
    Teacher<4, 1> teach;
    T z[1];
    teach.load(a, m);
    teach.gather(a, row, 0, (int)a.V, z);
    const Stat st = join_stats(a.stat + m * a.stats, a.parts, a.c2);
    const float logs = st.log();
    const float wt = wave_max(teach.top(a));
    if ((t & 63) == 0) red_t[wave] = wt;
    __syncthreads();
    const float wu = wave_sum(teach.powers(a, join_max<4>(red_t)));
    if ((t & 63) == 0) red_u[wave] = wu;
    __syncthreads();
    teach.form(a, join_sum<4>(red_u));
    const float wl = wave_sum(teach.loss(a, z, st, logs));
    if ((t & 63) == 0) red_l[wave] = wl;
    __syncthreads();
    const float loss = join_sum<4>(red_l);
    if (t == 0) {
        a.stat[m * a.stats] = st;   // (all waves have joined the parts' before the barriers)
        a.loss[m] = loss;
        if (a.lse) a.lse[m] = st.lse(a.scale, logs);
    }
}

// The gradient from lse, or from the maxima and sums that the loss has left (JOINED): an lse is off by |lse| 2^-24, and so
// are shares of the row formed from it, relative, which those from the sum are not.  A part of a row each.  The whole part is loaded before any of it is stored, and so are its
// listed columns: dx may be x.  (What a row's last piece reads of the part before counts for nothing.)
template <typename T, int NW, int VPT, bool TINY, bool JOINED>
__global__ __launch_bounds__(64 * NW) void distill_bwd_kernel(DistArgs a) {
    constexpr int NT = 64 * NW, LEN = NT * VPT * CH, KPT = list_per_thread(NW);
    __shared__ float red_t[NW], red_u[NW];
    __shared__ __attribute__((aligned(16))) int cols[kListMax];
    __shared__ __attribute__((aligned(16))) float probs[kListMax];
    const int t = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int64_t m = blockIdx.x / (uint32_t)a.parts;
    const int part = blockIdx.x % (uint32_t)a.parts, V = (int)a.V, c0 = part * LEN, c1 = min(c0 + LEN, V);
    const T* row = (const T*)a.x + m * a.ldx;
    Teacher<NW, KPT> teach;
    teach.load(a, m);
    const Stat st = JOINED ? a.stat[m * a.stats] : Stat{0.f, 1.f, 0.f};
    const float lse = JOINED ? 0.f : a.lse_in[m], g1 = a.dloss ? a.dloss[a.g_step ? m : 0] : 1.f;
    const Live<NW, VPT> live(V - c0, wave);
    Piece<T> p[VPT];
#pragma unroll
    for (int i = 0; i < VPT; i++) p[i] = load_logits<T, TINY>(row, c0 + (i * NT + t) * CH, V);
    T z[KPT];
    teach.gather(a, row, c0, c1, z);
    const float wt = wave_max(teach.top(a));
    if ((t & 63) == 0) red_t[wave] = wt;
    __syncthreads();
    const float wu = wave_sum(teach.powers(a, join_max<NW>(red_t)));
    if ((t & 63) == 0) red_u[wave] = wu;
    __syncthreads();
    teach.form(a, join_sum<NW>(red_u));
    teach.put(a, cols, probs);
    const float g = g1 * a.scale * teach.unit;
    const bool none = lse == neg_inf();   // a row of minus infinities: q = 0
    const Base base(st.m, a.c2);
    const float inv = st.s == 0.f ? 0.f : __builtin_amdgcn_exp2f(-base.r) / st.s;
    auto share = [&](float x) {
        if constexpr (JOINED) return base.power(x) * inv;
        // A share above 1 is lse's rounding: by little it goes as it is; where lse has no digits of that size (a row of the type's
        // lowest value) the difference may be any number, and counts for 0.  (A NaN stays one.)
        const float d = __builtin_fmaf(x, a.scale, -lse);
        return none ? 0.f : __builtin_amdgcn_exp2f((d > 0x1p-7f ? 0.f : d) * kLog2e);
    };
    T* dx = (T*)a.dx + m * a.lddx;
    // (every wave's loads of the row come before the barriers above: dx may be x)
#pragma unroll
    for (int i = 0; i < VPT; i++) {
        if (i >= live.all) continue;
        float v[CH];
        logit_values(p[i], v);
#pragma unroll
        for (int e = 0; e < CH; e++) v[e] = teach.any ? g * share(v[e]) : 0.f;
        const int c = c0 + (i * NT + t) * CH;
        if (c < V) store_logits<T, TINY>(dx, c, V, v, a.stream);
    }
    __syncthreads();
    if (!teach.any) return;
    float q[KPT];
#pragma unroll
    for (int i = 0; i < KPT; i++) q[i] = share(to_f(z[i]));
    teach.store(a, dx, cols, probs, q, g, c0, c1);
}

// ---------------------------------------------------------------- choice
// Kernels by the waves of a workgroup and the pieces of a thread, in the order of the columns that they hold.
struct Shape {
    int nw, vpt;
    constexpr int cols() const { return 64 * nw * vpt * CH; }
};
enum { k512, k2048, k4096, k8192, k16384, k32768, k32768w, k65536, k131072 };   // (w: of twice the waves)
constexpr Shape kShapes[] = {{1, 1}, {1, 4}, {4, 2}, {4, 4}, {8, 4}, {8, 8}, {16, 4}, {16, 8}, {16, 16}};

// Calls f with the shape's sizes as constants.
template <typename F>
hipError_t by_shape(int shape, F f) {
    switch (shape) {
        case k512: return f(std::integral_constant<int, 1>(), std::integral_constant<int, 1>());
        case k2048: return f(std::integral_constant<int, 1>(), std::integral_constant<int, 4>());
        case k4096: return f(std::integral_constant<int, 4>(), std::integral_constant<int, 2>());
        case k8192: return f(std::integral_constant<int, 4>(), std::integral_constant<int, 4>());
        case k16384: return f(std::integral_constant<int, 8>(), std::integral_constant<int, 4>());
        case k32768: return f(std::integral_constant<int, 8>(), std::integral_constant<int, 8>());
        case k32768w: return f(std::integral_constant<int, 16>(), std::integral_constant<int, 4>());
        case k65536: return f(std::integral_constant<int, 16>(), std::integral_constant<int, 8>());
        default: return f(std::integral_constant<int, 16>(), std::integral_constant<int, 16>());
    }
}

struct Plan {
    int shape, parts;
};
inline Plan in_parts(int64_t V, int shape) { return Plan{shape, (int)((V + kShapes[shape].cols() - 1) / kShapes[shape].cols())}; }
// Parts of the first of the given shapes that makes no more than kPartsMax of them.
inline Plan in_parts(int64_t V, std::initializer_list<int> shapes) {
    Plan p{};
    for (int s : shapes) {
        p = in_parts(V, s);
        if (p.parts <= kPartsMax) break;
    }
    return p;
}
// The smallest shape for a whole row of up to 16384 columns.
inline Plan short_row(int64_t V) {
    int s = k512;
    while (V > kShapes[s].cols()) s++;
    return Plan{s, 1};
}

// Whole rows need no second launch (3 us), parts of fewer registers leave more of them on a CU.  Both ways in us, whole and in parts
// (of 16384 columns in 16 bits, of 8192 in 32):  16 bits, 32000 columns, 1000 rows 20.2, 23.7; 40000 columns, 60 rows 9.2, 11.2, 300
// 17.0, 16.1, 1000 33.2, 28.5; 60000 columns, 300 rows 19.8, 18.4;  32 bits, 32000 columns, 300 rows 16.3, 16.9, 1000 33.2, 29.3, 4000 125,
// 104; 60000 columns, 60 rows 10.3, 12.4, 300 23.7, 22.5.  Which parts, of 4096, 8192 and 16384: 100000 columns in 16 bits, 1 row
// 9.4, 10.5, 10.5, 60 12.6, 12.6, 12.4, 1000 79, 56, 56; in 32 bits, 60 rows 14.0, 14.5, 14.2, 300 29.8, 27.4, 27.4, 1000 85, 74, 75.
constexpr int64_t few_rows(int type) { return type != NITI_F32 ? 48 : 96; }
Plan logprobs_plan(int64_t M, int64_t V, int type) {
    if (V <= 16384) return short_row(V);
    const bool half = type != NITI_F32;
    if (V <= 32768 && (half || M <= 512)) return Plan{k32768w, 1};
    if (V > 32768 && V <= 65536 && M <= 256) return Plan{k65536, 1};
    if (M <= few_rows(type)) return in_parts(V, {k4096, k8192, k16384, k32768w, k65536});
    return half ? in_parts(V, {k16384, k32768w, k65536}) : in_parts(V, {k8192, k16384, k32768w, k65536});
}

// With the gradient a second reading costs more than the registers of a whole row: parts only where those do not hold it (77 x
// 128001 in 32 bits: parts of 8192 30 us, of 65536 37), or for few rows of more than 65536 (1 x 128000 in 16 bits 14.7 for 20; 1000 of them
// 127 for 102).  32768 columns by eight waves: 4096 x 32000 in 16 bits 102 us, by sixteen 106; in 32 bits 1000 x 32000 56 us, by sixteen 66, but
// 4000 x 32000 240 and 222.
Plan distill_plan(int64_t M, int64_t V, int type) {
    if (V <= 16384) return short_row(V);
    if (V <= 32768) return Plan{k32768, 1};
    if (V <= 65536) return Plan{k65536, 1};
    if (V <= 131072 && type != NITI_F32 && M >= 64) return Plan{k131072, 1};
    return in_parts(V, {k8192, k16384, k32768, k65536});
}

// A launch holds fewer than 2^32 threads: very many rows go in slabs.
constexpr int64_t kSlab = (int64_t)1 << 21;

size_t log_space(int64_t M, int parts, int64_t top) {
    return parts > 1 ? up256((size_t)M * parts * sizeof(Stat)) + up256((size_t)M * parts * (size_t)top * 8) : 0;
}

template <typename T>
hipError_t run_logprobs(LogArgs a, const Plan& plan, char* ws, hipStream_t stream) {
    a.parts = plan.parts;
    const int64_t M = a.M, slab = kSlab / plan.parts;
    if (plan.parts > 1) {
        a.stat = (Stat*)ws;
        a.ranks = (uint64_t*)(ws + up256((size_t)M * a.parts * sizeof(Stat)));
    }
    for (int64_t m0 = 0; m0 < M; m0 += slab) {
        a.M = M - m0 < slab ? M - m0 : slab;
        hipError_t e = by_shape(plan.shape, [&](auto nw, auto vpt) {
            constexpr int NW = decltype(nw)::value, VPT = decltype(vpt)::value;
            if constexpr (VPT == 1)
                if (a.V < CH) {
                    hipLaunchKernelGGL((logprobs_kernel<T, NW, VPT, true>), dim3((unsigned)a.M), dim3(64 * NW), 0, stream, a);
                    return hipGetLastError();
                }
            if constexpr (!(NW == 8 && VPT == 8) && VPT <= 8)
                hipLaunchKernelGGL((logprobs_kernel<T, NW, VPT, false>), dim3((unsigned)(a.M * a.parts)), dim3(64 * NW), 0, stream, a);
            return hipGetLastError();
        });
        if (e == hipSuccess && a.parts > 1) {
            hipLaunchKernelGGL((logprobs_join_kernel<T>), dim3((unsigned)a.M), dim3(256), 0, stream, a);
            e = hipGetLastError();
        }
        if (e != hipSuccess) return e;
        a.x = (const T*)a.x + slab * a.ldx;
        if (a.tokens) a.tokens += slab;
        if (a.logp) a.logp += slab;
        if (a.lse) a.lse += slab;
        if (a.entropy) a.entropy += slab;
        if (a.top_logp) a.top_logp += slab * a.top;
        if (a.top_idx) a.top_idx += slab * a.top;
    }
    return hipSuccess;
}

template <typename T>
void next_slab(DistArgs& a, int64_t slab) {
    a.x = (const T*)a.x + slab * a.ldx;
    a.t_val = (const char*)a.t_val + slab * a.ldt * (int64_t)type_size(a.t_type);
    a.t_idx += slab * a.ldi;
    if (a.loss) a.loss += slab;
    if (a.lse) a.lse += slab;
    if (a.lse_in) a.lse_in += slab;
    if (a.dloss && a.g_step) a.dloss += slab;
    if (a.dx) a.dx = (T*)a.dx + slab * a.lddx;
    if (a.stat) a.stat += slab * a.stats;
}

// Whether a gradient goes past the caches: more than the eight L2 hold would only push out what is still to be read (4096 x 32000 in
// 16 bits, with the loss 119 -> 102 us, alone 112 -> 89).
inline int32_t streams(int64_t M, int64_t V, size_t size) { return M * V * (int64_t)size > ((int64_t)32 << 20); }

template <typename T, bool JOINED>
hipError_t run_distill_bwd(DistArgs a, hipStream_t stream) {
    // 4096 columns a workgroup where rows are longer than 512
    const int shape = a.V <= 512 ? k512 : k4096;
    a.parts = in_parts(a.V, shape).parts;
    a.stream = streams(a.M, a.V, sizeof(T));
    const int64_t M = a.M, slab = kSlab / a.parts;
    for (int64_t m0 = 0; m0 < M; m0 += slab) {
        a.M = M - m0 < slab ? M - m0 : slab;
        const hipError_t e = by_shape(shape, [&](auto nw, auto vpt) {
            constexpr int NW = decltype(nw)::value, VPT = decltype(vpt)::value;
            if constexpr (VPT == 1 && !JOINED)
                if (a.V < CH) {
                    hipLaunchKernelGGL((distill_bwd_kernel<T, NW, VPT, true, false>), dim3((unsigned)a.M), dim3(64 * NW), 0, stream, a);
                    return hipGetLastError();
                }
            if constexpr ((NW == 1 && VPT == 1 && !JOINED) || (NW == 4 && VPT == 2))   // (split rows are long ones)
                hipLaunchKernelGGL((distill_bwd_kernel<T, NW, VPT, false, JOINED>), dim3((unsigned)(a.M * a.parts)), dim3(64 * NW), 0, stream, a);
            return hipGetLastError();
        });
        if (e != hipSuccess) return e;
        next_slab<T>(a, slab);
    }
    return hipSuccess;
}

template <typename T>
hipError_t run_distill(DistArgs a, const Plan& plan, char* ws, hipStream_t stream) {
    a.parts = plan.parts;
    a.stream = streams(a.M, a.V, sizeof(T));
    a.stats = plan.parts;
    if (plan.parts > 1) a.stat = (Stat*)ws;
    const DistArgs whole = a;
    const int64_t M = a.M, slab = kSlab / plan.parts;
    const bool grad = a.dx && plan.parts == 1;
    for (int64_t m0 = 0; m0 < M; m0 += slab) {
        a.M = M - m0 < slab ? M - m0 : slab;
        hipError_t e = by_shape(plan.shape, [&](auto nw, auto vpt) {
            constexpr int NW = decltype(nw)::value, VPT = decltype(vpt)::value;
            const dim3 grid((unsigned)(a.M * a.parts)), block(64 * NW);
            if constexpr (VPT == 1)
                if (a.V < CH) {
                    if (grad) hipLaunchKernelGGL((distill_kernel<T, NW, VPT, true, true>), grid, block, 0, stream, a);
                    else hipLaunchKernelGGL((distill_kernel<T, NW, VPT, true, false>), grid, block, 0, stream, a);
                    return hipGetLastError();
                }
            if constexpr (!(NW == 16 && VPT == 4) && sizeof(T) * VPT <= 32) {
                if (grad) hipLaunchKernelGGL((distill_kernel<T, NW, VPT, false, true>), grid, block, 0, stream, a);
                else hipLaunchKernelGGL((distill_kernel<T, NW, VPT, false, false>), grid, block, 0, stream, a);
            }
            return hipGetLastError();
        });
        if (e == hipSuccess && a.parts > 1) {
            hipLaunchKernelGGL((distill_join_kernel<T>), dim3((unsigned)a.M), dim3(256), 0, stream, a);
            e = hipGetLastError();
        }
        if (e != hipSuccess) return e;
        next_slab<T>(a, slab);
    }
    if (!whole.dx || grad) return hipSuccess;
    return run_distill_bwd<T, true>(whole, stream);
}

// (scale log2 e is finite up to here: an infinite one times a difference of 0 is a NaN)
inline bool fine_scale(float s) { return s > 0.f && s <= 0x1p127f; }

}  // namespace

// For either type's plan: the caller's sizes do not say which.
// (Few rows may be in more parts than many, and take more: there is room for any number of rows up to M.)
size_t logprobs_workspace(int64_t M, int64_t V, int64_t top) {
    if (M < 1 || V < 1 || top < 0 || top > kTopMax || top > V || M >= kMaxDim || V >= kMaxLd) return 0;
    size_t need = 0;
    for (int type : {NITI_F32, NITI_BF16})
        for (int64_t m : {M, std::min(M, few_rows(type))}) need = std::max(need, log_space(m, logprobs_plan(m, V, type).parts, top));
    return need;
}
size_t distill_workspace(int64_t M, int64_t V) {
    if (M < 1 || V < 1 || M >= kMaxDim || V >= kMaxLd) return 0;
    const int wide = distill_plan(M, V, NITI_F32).parts, half = distill_plan(M, V, NITI_BF16).parts;
    const int parts = wide > half ? wide : half;
    return parts > 1 ? up256((size_t)M * parts * sizeof(Stat)) : 0;
}

}  // namespace niti

using namespace niti;

extern "C" {

niti_status niti_token_logprobs(const void* x, int64_t ldx, const int32_t* tokens, float* logp, float* lse, float* entropy,
                                float* top_logp, int32_t* top_idx, int64_t M, int64_t V, int64_t top, float scale, int type,
                                void* ws, size_t ws_bytes, void* stream) {
    if (M < 0 || V < 1 || top < 0 || top > V) return NITI_ERR_SHAPE;
    if (!valid_type(type) || !fine_scale(scale)) return NITI_ERR_ARG;
    if (M >= kMaxDim || V >= kMaxLd || top > kTopMax) return NITI_ERR_UNSUPPORTED;
    if (M == 0) return NITI_OK;
    if (!x || (logp != nullptr) != (tokens != nullptr) || ((top_logp || top_idx) != (top > 0))) return NITI_ERR_NULL;
    if (bad_ld(M > 1 ? ldx : V, V, false)) return NITI_ERR_SHAPE;
    const Plan plan = logprobs_plan(M, V, type);
    if (plan.parts > 1) {
        if (!ws || ws_bytes < log_space(M, plan.parts, top)) return NITI_ERR_WORKSPACE;
        if ((uintptr_t)ws & 15) return NITI_ERR_ARG;
    }
    LogArgs a{};
    a.x = x, a.ldx = M > 1 ? ldx : V, a.tokens = tokens, a.logp = logp, a.lse = lse, a.entropy = entropy;
    a.top_logp = top_logp, a.top_idx = top_idx, a.M = M, a.V = V, a.top = (int32_t)top;
    a.scale = scale, a.c2 = (float)((double)scale * 1.44269504088896340736);
    return by_type(type, [&](auto t) { return run_logprobs<decltype(t)>(a, plan, (char*)ws, (hipStream_t)stream); }) == hipSuccess
               ? NITI_OK : NITI_ERR_HIP;
}

niti_status niti_distill_fwd(const void* x, int64_t ldx, const void* t_val, int64_t ldt, int t_type, const int32_t* t_idx, int64_t ldi,
                             float* loss, float* lse, const float* dloss, int64_t dloss_n, void* dx, int64_t lddx, int64_t M, int64_t V,
                             int64_t top, float scale, int type, void* ws, size_t ws_bytes, void* stream) {
    if (M < 0 || V < 1 || top < 1) return NITI_ERR_SHAPE;
    if (!valid_type(type) || !valid_type(t_type) || !fine_scale(scale)) return NITI_ERR_ARG;
    if (M >= kMaxDim || V >= kMaxLd || top > kListMax) return NITI_ERR_UNSUPPORTED;
    if (M == 0) return NITI_OK;
    if (!x || !t_val || !t_idx || !loss || (dloss && !dx)) return NITI_ERR_NULL;
    if (bad_ld(M > 1 ? ldx : V, V, false) || bad_ld(M > 1 ? ldt : top, top, false) || bad_ld(M > 1 ? ldi : top, top, false) ||
        (dx && bad_ld(M > 1 ? lddx : V, V, true)) || (dloss && dloss_n != 1 && dloss_n != M))
        return NITI_ERR_SHAPE;
    const Plan plan = distill_plan(M, V, type);
    if (plan.parts > 1) {
        if (!ws || ws_bytes < distill_workspace(M, V)) return NITI_ERR_WORKSPACE;
        if ((uintptr_t)ws & 15) return NITI_ERR_ARG;
    }
    DistArgs a{};
    a.x = x, a.ldx = M > 1 ? ldx : V, a.t_val = t_val, a.ldt = M > 1 ? ldt : top, a.t_type = t_type, a.t_idx = t_idx;
    a.ldi = M > 1 ? ldi : top, a.loss = loss, a.lse = lse, a.dloss = dloss, a.g_step = dloss_n == 1 ? 0 : 1;
    a.dx = dx, a.lddx = M > 1 ? lddx : V, a.M = M, a.V = V, a.top = (int32_t)top;
    a.scale = scale, a.c2 = (float)((double)scale * 1.44269504088896340736);
    return by_type(type, [&](auto t) { return run_distill<decltype(t)>(a, plan, (char*)ws, (hipStream_t)stream); }) == hipSuccess
               ? NITI_OK : NITI_ERR_HIP;
}

niti_status niti_distill_bwd(const void* x, int64_t ldx, const void* t_val, int64_t ldt, int t_type, const int32_t* t_idx, int64_t ldi,
                             const float* lse, const float* dloss, int64_t dloss_n, void* dx, int64_t lddx, int64_t M, int64_t V,
                             int64_t top, float scale, int type, void* stream) {
    if (M < 0 || V < 1 || top < 1) return NITI_ERR_SHAPE;
    if (!valid_type(type) || !valid_type(t_type) || !fine_scale(scale)) return NITI_ERR_ARG;
    if (M >= kMaxDim || V >= kMaxLd || top > kListMax) return NITI_ERR_UNSUPPORTED;
    if (M == 0) return NITI_OK;
    if (!x || !t_val || !t_idx || !lse || !dx) return NITI_ERR_NULL;
    if (bad_ld(M > 1 ? ldx : V, V, false) || bad_ld(M > 1 ? ldt : top, top, false) || bad_ld(M > 1 ? ldi : top, top, false) ||
        bad_ld(M > 1 ? lddx : V, V, true) || (dloss && dloss_n != 1 && dloss_n != M))
        return NITI_ERR_SHAPE;
    DistArgs a{};
    a.x = x, a.ldx = M > 1 ? ldx : V, a.t_val = t_val, a.ldt = M > 1 ? ldt : top, a.t_type = t_type, a.t_idx = t_idx;
    a.ldi = M > 1 ? ldi : top, a.lse_in = lse, a.dloss = dloss, a.g_step = dloss_n == 1 ? 0 : 1;
    a.dx = dx, a.lddx = M > 1 ? lddx : V, a.M = M, a.V = V, a.top = (int32_t)top;
    a.scale = scale, a.c2 = (float)((double)scale * 1.44269504088896340736);
    return by_type(type, [&](auto t) { return run_distill_bwd<decltype(t), false>(a, (hipStream_t)stream); }) == hipSuccess
               ? NITI_OK : NITI_ERR_HIP;
}

}  // extern "C"
