// What the logits of a language model are read for: log probabilities of given
// tokens with the entropy and the top alternatives, and the divergence from a
// teacher's top logits with its gradient.
//
// With u_v = x_v - max x:  S = sum exp(scale u_v), W = sum u_v exp(scale u_v),
//   lse = scale max + ln S,  log p_v = scale u_v - ln S,  entropy = ln S - scale W / S,
//   dx_v = dloss scale (exp(scale u_v) / S - sum of the p_j of v).
// A row is read once: it stays in the registers of one workgroup (up to 64K columns in 32 bits, 128K
// in 16) as it was loaded, the maximum is found first and the sums next, so
// that every element costs one exponential; longer rows, and few of them, are split over
// workgroups whose parts a second launch joins.  The fused gradient writes from the same registers.
//
// The k largest of a row: 64 groups of threads have a maximum each, and the k-th
// largest of those is a bound that at least k logits reach.  Logits that reach it
// (some 25 where k is 20) are collected in any order and placed by counting,
// for each, those before it: larger, or equal with a lower column.  Where more than kCand reach the bound
// (masked rows whose bound is minus infinity, many equal ones) the k-th value is found by bisection on its bits, and
// the last column of its equals by bisection on the column.
#include "linear.h"

#include <math.h>

#include <type_traits>

namespace niti {

namespace {

constexpr int kTopMax = 64;     // alternatives of a row
constexpr int kListMax = 256;   // teacher's logits of a row
constexpr int kCand = 512;      // collected logits of a row
constexpr float kLog2e = 1.44269504088896341f;
constexpr uint32_t kNegInf = 0xFF800000u;

__device__ __forceinline__ float neg_inf() { return __uint_as_float(kNegInf); }
__device__ __forceinline__ float quiet_nan() { return __uint_as_float(0x7FC00000u); }

// Integers of the order of floats (no NaN among them; both zeros alike).
__device__ __forceinline__ uint32_t order_key(float v) {
    const uint32_t b = __float_as_uint(v + 0.f);
    return b ^ (b >> 31 ? 0xFFFFFFFFu : 0x80000000u);
}

// Eight logits from column c on, as they are loaded (in no branch where a row has eight).
template <typename T>
__device__ __forceinline__ Piece<T> load_logits(const T* row, int c, int V) {
    Piece<T> p;
    if (V >= CH) {
        const int from = min(c, V - CH);
        __builtin_memcpy(p.w, row + from, sizeof(p.w));
        return p;
    }
    T t[CH];
#pragma unroll
    for (int e = 0; e < CH; e++) t[e] = row[min(c + e, V - 1)];
    __builtin_memcpy(p.w, t, sizeof(t));
    return p;
}
// Set right where the row ends: minus infinity past it.
template <typename T>
__device__ __forceinline__ void end_logits(Piece<T>& p, int c, int V) {
    if (c + CH <= V) return;
    constexpr int W = CH * sizeof(T) / 4, PER = 4 / sizeof(T);
    const uint32_t none = sizeof(T) == 4 ? kNegInf : (__is_same(T, bf16) ? 0xFF80FF80u : 0xFC00FC00u);
    const int down = V < CH ? 0 : min(c - (V - CH), CH);   // elements to move down; CH: the whole piece is past the row
    if (PER == 2 && (down & 1)) {
#pragma unroll
        for (int i = 0; i < W; i++) p.w[i] = p.w[i] >> 16 | (i + 1 < W ? p.w[i + 1 < W ? i + 1 : i] : none) << 16;
    }
#pragma unroll
    for (int b = 1; b <= W; b *= 2) {
        const bool move = (down / PER) & b;
#pragma unroll
        for (int i = 0; i < W; i++) p.w[i] = move ? (i + b < W ? p.w[i + b < W ? i + b : i] : none) : p.w[i];
    }
    if (V < CH) {
        T t[CH];
        __builtin_memcpy(t, p.w, sizeof(t));
#pragma unroll
        for (int e = 0; e < CH; e++)
            if (c + e >= V) t[e] = from_f<T>(neg_inf());
        __builtin_memcpy(p.w, t, sizeof(t));
    }
}
template <typename T>
__device__ __forceinline__ void logit_values(const Piece<T>& p, float (&v)[CH]) {
    T t[CH];
    __builtin_memcpy(t, p.w, sizeof(t));
#pragma unroll
    for (int e = 0; e < CH; e++) v[e] = to_f(t[e]);
}

__device__ __forceinline__ float wave_max_f32(float v) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, kWave));
    return v;
}

// A row's (or a part's) statistics.
struct Stat {
    float m, s, w;   // max x, S, W; a row of minus infinities: -inf, 0, 0
};
// What exponents are taken from: the maximum, or 0 where there is none.
__device__ __forceinline__ float base_of(float m) { return m == neg_inf() ? 0.f : m; }
// A NaN or an infinity in the row leaves a NaN in S.
__device__ __forceinline__ float log_of(const Stat& st) { return logf(st.s); }
__device__ __forceinline__ float lse_of(const Stat& st, float scale, float logs) { return st.m == neg_inf() && st.s == 0.f ? neg_inf() : scale * base_of(st.m) + logs; }
__device__ __forceinline__ float logp_of(const Stat& st, float scale, float logs, float x) {
    return st.m == neg_inf() && st.s == 0.f ? neg_inf() : scale * (x - base_of(st.m)) - logs;
}

// Sums of exp(scale u) and u exp(scale u) over a thread's pieces.
template <typename T, int VPT>
__device__ __forceinline__ void exp_sums(const Piece<T> (&p)[VPT], float base, float c2, float& s, float& w) {
    s = w = 0.f;
#pragma unroll
    for (int i = 0; i < VPT; i++) {
        float v[CH];
        logit_values(p[i], v);
#pragma unroll
        for (int e = 0; e < CH; e++) {
            const float u = v[e] - base;
            const float x = __builtin_amdgcn_exp2f(u * c2);
            s += x;
            w = __builtin_fmaf(x, fmaxf(u, -0x1p100f), w);   // (minus infinity times 0)
        }
    }
}

struct LogArgs {
    const void* x;
    const int32_t* tokens;
    float *logp, *lse, *entropy, *top_logp;
    int32_t* top_idx;
    int64_t ldx, M, V;
    int32_t top, parts;
    float scale, c2;
    // Parts of split rows: [M][parts] statistics, [M][parts][top] logits and columns in order (past the last: column -1).
    Stat* stat;
    float* val;
    int32_t* col;
};

// A row's scalars, by one thread.
__device__ __forceinline__ void put_scalars(const LogArgs& a, int64_t m, const Stat& st, float logs, int tok, float x) {
    if (a.logp) a.logp[m] = (uint32_t)tok < (uint64_t)a.V ? logp_of(st, a.scale, logs, x) : 0.f;
    if (a.lse) a.lse[m] = lse_of(st, a.scale, logs);
    if (a.entropy) a.entropy[m] = st.m == neg_inf() && st.s == 0.f ? 0.f : logs - a.scale * st.w / st.s;
}
__device__ __forceinline__ void put_top(const LogArgs& a, int64_t m, int r, const Stat& st, float logs, float v, int col) {
    const bool bad = !(st.s == st.s);
    if (a.top_logp) a.top_logp[m * a.top + r] = bad ? quiet_nan() : logp_of(st, a.scale, logs, v);
    if (a.top_idx) a.top_idx[m * a.top + r] = bad ? -1 : col;
}

// The bound: the largest of 64 values that at least k of them reach.
__device__ __forceinline__ float bound_of(float g, int k) {
    int above = 0;
#pragma unroll
    for (int j = 0; j < 64; j++)
        above += __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(g), j)) >= g ? 1 : 0;
    return wave_max_f32(above >= k ? g : neg_inf());
}

struct Cand {
    float v[kCand];
    int col[kCand];
    int n;
};
// Whether candidate i stands before one of key and column.
__device__ __forceinline__ bool before(const Cand& c, int i, uint32_t key, int col) {
    const uint32_t k = order_key(c.v[i]);
    return k > key || (k == key && c.col[i] < col);
}

template <typename T, int NW, int VPT>
__global__ __launch_bounds__(64 * NW) void logprobs_kernel(LogArgs a) {
    constexpr int NT = 64 * NW, LEN = NT * VPT * CH;
    __shared__ float red_m[NW], red_s[NW], red_w[NW], group[64], tau_s;
    __shared__ int red_c[2][NW];
    __shared__ Cand cand;
    const int t = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int64_t m = blockIdx.x / (uint32_t)a.parts;
    const int part = blockIdx.x % (uint32_t)a.parts, V = (int)a.V, c0 = part * LEN;
    const T* row = (const T*)a.x + m * a.ldx;
    Piece<T> p[VPT];
#pragma unroll
    for (int i = 0; i < VPT; i++) p[i] = load_logits(row, c0 + (i * NT + t) * CH, V);
    const int tok = a.parts == 1 && a.tokens ? a.tokens[m] : -1;
    const float x_tok = to_f(row[(uint32_t)tok < (uint32_t)V ? tok : 0]);
    if (t == 0) cand.n = 0;
    float mx = neg_inf();
#pragma unroll
    for (int i = 0; i < VPT; i++) {
        end_logits(p[i], c0 + (i * NT + t) * CH, V);
        float v[CH];
        logit_values(p[i], v);
#pragma unroll
        for (int e = 0; e < CH; e++) mx = fmaxf(mx, v[e]);
    }
    // 64 groups of NW neighbouring threads
    float gm = mx;
#pragma unroll
    for (int o = 1; o < NW; o *= 2) gm = fmaxf(gm, __shfl_xor(gm, o, kWave));
    if (t % NW == 0) group[t / NW] = gm;
    const float wm = wave_max_f32(gm);
    if ((t & 63) == 0) red_m[wave] = wm;
    __syncthreads();
    Stat st;
    st.m = red_m[0];
#pragma unroll
    for (int i = 1; i < NW; i++) st.m = fmaxf(st.m, red_m[i]);
    if (a.top && wave == 0) {
        const float tau = bound_of(group[t], a.top);
        if (t == 0) tau_s = tau;
    }
    exp_sums<T, VPT>(p, base_of(st.m), a.c2, st.s, st.w);
    st.s = wave_sum_f32(st.s);
    st.w = wave_sum_f32(st.w);
    if ((t & 63) == 0) red_s[wave] = st.s, red_w[wave] = st.w;
    __syncthreads();
    st.s = red_s[0], st.w = red_w[0];
#pragma unroll
    for (int i = 1; i < NW; i++) st.s += red_s[i], st.w += red_w[i];
    const float logs = log_of(st);
    if (t == 0) {
        if (a.parts == 1) put_scalars(a, m, st, logs, tok, x_tok);
        else a.stat[m * a.parts + part] = st;
    }
    if (!a.top) return;
    const float tau = tau_s;
    auto each = [&](auto f) {   // f(value, column) of this thread's logits
#pragma unroll
        for (int i = 0; i < VPT; i++) {
            float v[CH];
            logit_values(p[i], v);
            const int c = c0 + (i * NT + t) * CH;
#pragma unroll
            for (int e = 0; e < CH; e++)
                if (c + e < V) f(v[e], c + e);
        }
    };
    auto keep = [&](float v, int c) {
        const int at = atomicAdd(&cand.n, 1);
        if (at < kCand) cand.v[at] = v, cand.col[at] = c;
    };
    if (mx >= tau) each([&](float v, int c) {
        if (v >= tau) keep(v, c);
    });
    __syncthreads();
    int n = cand.n;
    if (n > kCand) {   // (the same for all threads)
        int turn = 0;
        auto count = [&](auto pred) {
            int k = 0;
            each([&](float v, int c) { k += v == v && pred(order_key(v), c) ? 1 : 0; });
#pragma unroll
            for (int o = 32; o >= 1; o >>= 1) k += __shfl_xor(k, o, kWave);
            if ((t & 63) == 0) red_c[turn][wave] = k;
            __syncthreads();
            k = 0;
#pragma unroll
            for (int i = 0; i < NW; i++) k += red_c[turn][i];
            turn ^= 1;   // a wave that is a count ahead writes the other half
            return k;
        };
        uint32_t kth = 0;   // the key of the top-th largest
        for (int b = 31; b >= 0; b--) {
            const uint32_t want = kth | 1u << b;
            if (count([&](uint32_t k, int) { return k >= want; }) >= a.top) kth = want;
        }
        const int more = a.top - count([&](uint32_t k, int) { return k > kth; });
        int last = 0;       // the largest column with fewer than `more` equals before it
        for (int b = 22; b >= 0; b--) {
            const int want = last | 1 << b;
            if (count([&](uint32_t k, int c) { return k == kth && c < want; }) < more) last = want;
        }
        if (t == 0) cand.n = 0;
        __syncthreads();
        each([&](float v, int c) {
            const uint32_t k = order_key(v);
            if (v == v && (k > kth || (k == kth && c <= last))) keep(v, c);
        });
        __syncthreads();
        n = min(cand.n, kCand);
    }
    for (int j = t; j < n; j += NT) {
        const float v = cand.v[j];
        const uint32_t key = order_key(v);
        const int col = cand.col[j];
        int r = 0;
        for (int i = 0; i < n; i++) r += before(cand, i, key, col) ? 1 : 0;
        if (r >= a.top) continue;
        if (a.parts == 1) {
            put_top(a, m, r, st, logs, v, col);
        } else {
            const int64_t at = (m * a.parts + part) * a.top + r;
            a.val[at] = v;
            a.col[at] = col;
        }
    }
    for (int r = n + t; r < a.top; r += NT) {   // fewer logits than that in this part, or NaNs among them
        if (a.parts == 1) {
            put_top(a, m, r, st, logs, quiet_nan(), -1);
        } else {
            const int64_t at = (m * a.parts + part) * a.top + r;
            a.val[at] = neg_inf();
            a.col[at] = -1;
        }
    }
}

// Statistics of a row from those of its parts, by all 64 lanes of a wave, in an order fixed by the number of parts.
__device__ __forceinline__ Stat join_stats(const Stat* parts, int n, float c2) {
    const int lane = threadIdx.x & 63;
    float m = neg_inf();
    for (int i = lane; i < n; i += 64) m = fmaxf(m, parts[i].m);
    Stat st;
    st.m = wave_max_f32(m);
    const float base = base_of(st.m);
    st.s = st.w = 0.f;
    for (int i = lane; i < n; i += 64) {
        const Stat p = parts[i];
        const float d = base_of(p.m) - base;   // W = f (W_i + d S_i) with f = exp(scale d)
        const float f = p.s == 0.f ? 0.f : __builtin_amdgcn_exp2f(d * c2);
        st.s += f * p.s;
        st.w += f * (p.w + fmaxf(d, -0x1p100f) * p.s);
    }
    st.s = wave_sum_f32(st.s);
    st.w = wave_sum_f32(st.w);
    return st;
}

constexpr int kPartsMax = 64;   // parts of a row

// Joins a row's parts: 256 threads.  Every part's k candidates are in order, so the (r + 1)-st of
// each of j parts with j (r + 1) >= k bounds the k-th of the row.
template <typename T>
__global__ __launch_bounds__(256) void logprobs_join_kernel(LogArgs a) {
    __shared__ float val[kPartsMax * kTopMax];
    __shared__ int col[kPartsMax * kTopMax];
    __shared__ float tau_s;
    __shared__ int n_s;
    const int t = threadIdx.x;
    const int64_t m = blockIdx.x;
    const int top = a.top, parts = a.parts;
    const int tok = a.tokens ? a.tokens[m] : -1;
    const float x_tok = to_f(((const T*)a.x + m * a.ldx)[(uint32_t)tok < (uint32_t)a.V ? tok : 0]);
    const float* v = a.val + m * parts * top;
    const int32_t* c = a.col + m * parts * top;
    if (t == 0) n_s = 0;
    if (top && t < 64) {
        const int r = (top + parts - 1) / parts - 1, j = (top + r) / (r + 1);
        const float tau = bound_of(t < parts ? v[t * top + r] : neg_inf(), j);
        if (t == 0) tau_s = tau;
    }
    const Stat st = join_stats(a.stat + m * parts, parts, a.c2);
    const float logs = log_of(st);
    if (t == 0) put_scalars(a, m, st, logs, tok, x_tok);
    if (!top) return;
    __syncthreads();
    const float tau = tau_s;
    for (int i = t; i < parts * top; i += 256) {
        const float x = v[i];
        const int k = c[i];
        if (k >= 0 && x >= tau) {
            const int at = atomicAdd(&n_s, 1);
            val[at] = x;
            col[at] = k;
        }
    }
    __syncthreads();
    const int n = n_s;
    for (int j = t; j < n; j += 256) {
        const uint32_t key = order_key(val[j]);
        const int mine = col[j];
        int r = 0;
        for (int i = 0; i < n; i++) {
            const uint32_t k = order_key(val[i]);
            r += k > key || (k == key && col[i] < mine) ? 1 : 0;
        }
        if (r < top) put_top(a, m, r, st, logs, val[j], mine);
    }
    for (int r = n + t; r < top; r += 256) put_top(a, m, r, st, logs, quiet_nan(), -1);
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
    int32_t top, t_type, parts, g_step;
    float scale, c2;
    Stat* stat;
};

// Entry j of the teacher's list of a row: its logit, minus infinity for a column outside the row.
struct Listed {
    float t;
    int col;
};
__device__ __forceinline__ Listed load_listed(const DistArgs& a, int64_t m, int j) {
    Listed l;
    l.col = a.t_idx[m * a.ldi + j];
    float v[1];
    load_typed(a.t_val, a.t_type, m * a.ldt + j, 1, v);
    const bool in = (uint32_t)l.col < (uint64_t)a.V;
    l.t = in ? v[0] : neg_inf();
    l.col = in ? l.col : -1;
    return l;
}

// Sum and maximum over a workgroup of NW waves; red: NW values that no one else uses.
template <int NW>
__device__ __forceinline__ float block_sum(float v, float* red) {
    v = wave_sum_f32(v);
    if (NW == 1) return v;
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = red[0];
#pragma unroll
    for (int i = 1; i < NW; i++) v += red[i];
    return v;
}
template <int NW>
__device__ __forceinline__ float block_max(float v, float* red) {
    v = wave_max_f32(v);
    if (NW == 1) return v;
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = red[0];
#pragma unroll
    for (int i = 1; i < NW; i++) v = fmaxf(v, red[i]);
    return v;
}

// The teacher's distribution over its list: KPT entries a thread.
template <int NW, int KPT>
struct Teacher {
    Listed l[KPT];
    float p[KPT], logp[KPT];
    bool any;     // whether the list has a probability
    float unit;   // 1; NaN for a list with a NaN or an infinity
    __device__ __forceinline__ void load(const DistArgs& a, int64_t m) {
#pragma unroll
        for (int i = 0; i < KPT; i++) {
            const int j = i * 64 * NW + threadIdx.x;
            l[i] = j < a.top ? load_listed(a, m, j) : Listed{neg_inf(), -1};
        }
    }
    __device__ __forceinline__ void form(const DistArgs& a, float* red0, float* red1) {
        float mx = neg_inf(), s = 0.f;
#pragma unroll
        for (int i = 0; i < KPT; i++) mx = fmaxf(mx, l[i].t);
        mx = block_max<NW>(mx, red0);
        const float base = base_of(mx);
#pragma unroll
        for (int i = 0; i < KPT; i++) {
            p[i] = __builtin_amdgcn_exp2f((l[i].t - base) * a.c2);
            s += p[i];
        }
        s = block_sum<NW>(s, red1);
        any = s != 0.f;
        unit = s / s;
        const float logs = logf(s);
#pragma unroll
        for (int i = 0; i < KPT; i++) {
            p[i] = any ? p[i] / s : 0.f;
            logp[i] = a.scale * (l[i].t - base) - logs;
        }
    }
};

// A row's loss from its statistics: the threads' terms, to be summed.  z: the row's logits at the listed columns.
template <int NW, int KPT>
__device__ __forceinline__ float loss_terms(const DistArgs& a, const Teacher<NW, KPT>& t, const float (&z)[KPT], const Stat& st, float logs) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < KPT; i++) {
        const float term = t.p[i] * (t.logp[i] - logp_of(st, a.scale, logs, z[i]));
        s += t.p[i] == 0.f ? 0.f : term;
    }
    return s;
}

template <int KPT>
__device__ __forceinline__ void put_list(int* col, float* p, const Listed (&l)[KPT], const float (&q)[KPT], int n) {
#pragma unroll
    for (int i = 0; i < KPT; i++) {
        const int j = i * (int)blockDim.x + threadIdx.x;
        if (j < n) col[j] = l[i].col, p[j] = q[i];
    }
}
// The listed columns' own gradients, from c0 to c1, after the whole row's: a column that is listed twice has both probabilities.
template <typename T, int KPT>
__device__ __forceinline__ void put_listed(const DistArgs& a, T* dx, const int* col, const float* p, const Listed (&l)[KPT],
                                           const float (&q)[KPT], float g, int c0, int c1) {
#pragma unroll
    for (int i = 0; i < KPT; i++) {
        const int mine = l[i].col;
        if (mine < c0 || mine >= c1 || mine < 0) continue;
        float s = 0.f;
        for (int j = 0; j < a.top; j++) s += col[j] == mine ? p[j] : 0.f;
        dx[mine] = from_f<T>(g * (q[i] - s));
    }
}

constexpr int list_per_thread(int nw) { return nw >= 4 ? 1 : 4; }

// Loss of a row (GRAD: and its gradient) by one workgroup, or a part's statistics.
template <typename T, int NW, int VPT, bool GRAD>
__global__ __launch_bounds__(64 * NW) void distill_kernel(DistArgs a) {
    constexpr int NT = 64 * NW, LEN = NT * VPT * CH, KPT = list_per_thread(NW);
    __shared__ float red_m[NW], red_s[NW], red_t[NW], red_u[NW], red_l[NW];
    __shared__ int col[kListMax];
    __shared__ float prob[kListMax];
    const int t = threadIdx.x;
    const int64_t m = blockIdx.x / (uint32_t)a.parts;
    const int part = blockIdx.x % (uint32_t)a.parts, V = (int)a.V, c0 = part * LEN;
    const T* row = (const T*)a.x + m * a.ldx;
    Piece<T> p[VPT];
#pragma unroll
    for (int i = 0; i < VPT; i++) p[i] = load_logits(row, c0 + (i * NT + t) * CH, V);
    Teacher<NW, KPT> teach;
    float z[KPT];
    if (a.parts == 1) {
        teach.load(a, m);
#pragma unroll
        for (int i = 0; i < KPT; i++) z[i] = to_f(row[max(teach.l[i].col, 0)]);
    }
    float mx = neg_inf();
#pragma unroll
    for (int i = 0; i < VPT; i++) {
        end_logits(p[i], c0 + (i * NT + t) * CH, V);
        float v[CH];
        logit_values(p[i], v);
#pragma unroll
        for (int e = 0; e < CH; e++) mx = fmaxf(mx, v[e]);
    }
    Stat st;
    st.m = block_max<NW>(mx, red_m);
    const float base = base_of(st.m);
    exp_sums<T, VPT>(p, base, a.c2, st.s, st.w);
    st.s = block_sum<NW>(st.s, red_s);
    if (a.parts > 1) {
        st.w = 0.f;
        if (t == 0) a.stat[m * a.parts + part] = st;
        return;
    }
    const float logs = log_of(st);
    teach.form(a, red_t, red_u);
    if (GRAD) put_list(col, prob, teach.l, teach.p, a.top);
    const float loss = block_sum<NW>(loss_terms(a, teach, z, st, logs), red_l);   // (its barrier is the list's too)
    if (NW == 1) __syncthreads();
    if (t == 0) {
        a.loss[m] = loss;
        if (a.lse) a.lse[m] = lse_of(st, a.scale, logs);
    }
    if constexpr (GRAD) {
        const float g = (a.dloss ? a.dloss[a.g_step ? m : 0] : 1.f) * a.scale * teach.unit;
        T* dx = (T*)a.dx + m * a.lddx;
        const float inv = st.s == 0.f ? 0.f : 1.f / st.s;
        float q[KPT];
#pragma unroll
        for (int i = 0; i < KPT; i++) q[i] = __builtin_amdgcn_exp2f((z[i] - base) * a.c2) * inv;
#pragma unroll
        for (int i = 0; i < VPT; i++) {
            const int c = (i * NT + t) * CH;
            if (c >= V) continue;
            float v[CH];
            logit_values(p[i], v);
#pragma unroll
            for (int e = 0; e < CH; e++) v[e] = teach.any ? g * (__builtin_amdgcn_exp2f((v[e] - base) * a.c2) * inv) : 0.f;
            store_some(dx + c, V - c, v);
        }
        if (!teach.any) return;
        __syncthreads();   // the row's stores before the listed columns'
        put_listed(a, dx, col, prob, teach.l, q, g, 0, V);
    }
}

// Joins a row's parts: 256 threads.
template <typename T>
__global__ __launch_bounds__(256) void distill_join_kernel(DistArgs a) {
    __shared__ float red_t[4], red_u[4], red_l[4];
    const int64_t m = blockIdx.x;
    const T* row = (const T*)a.x + m * a.ldx;
    Teacher<4, 1> teach;
    teach.load(a, m);
    const float z[1] = {to_f(row[max(teach.l[0].col, 0)])};
    const Stat st = join_stats(a.stat + m * a.parts, a.parts, a.c2);
    const float logs = log_of(st);
    teach.form(a, red_t, red_u);
    const float loss = block_sum<4>(loss_terms(a, teach, z, st, logs), red_l);
    if (threadIdx.x == 0) {
        a.loss[m] = loss;
        if (a.lse) a.lse[m] = lse_of(st, a.scale, logs);
    }
}

// The gradient from lse: a part of a row each.  The whole part is loaded before any of it is stored, and so are its
// listed columns: dx may be x.  (What a row's last piece reads of the part before is moved out of it.)
template <typename T, int NW, int VPT>
__global__ __launch_bounds__(64 * NW) void distill_bwd_kernel(DistArgs a) {
    constexpr int NT = 64 * NW, LEN = NT * VPT * CH, KPT = list_per_thread(NW);
    __shared__ float red_t[NW], red_u[NW];
    __shared__ int col[kListMax];
    __shared__ float prob[kListMax];
    const int t = threadIdx.x;
    const int64_t m = blockIdx.x / (uint32_t)a.parts;
    const int part = blockIdx.x % (uint32_t)a.parts, V = (int)a.V, c0 = part * LEN, c1 = min(c0 + LEN, V);
    const T* row = (const T*)a.x + m * a.ldx;
    Piece<T> p[VPT];
#pragma unroll
    for (int i = 0; i < VPT; i++) p[i] = load_logits(row, c0 + (i * NT + t) * CH, V);
    Teacher<NW, KPT> teach;
    teach.load(a, m);
    float z[KPT], q[KPT];
#pragma unroll
    for (int i = 0; i < KPT; i++) {
        const int k = teach.l[i].col;
        z[i] = to_f(row[k >= c0 && k < c1 ? k : c0]);
    }
    const float lse = a.lse_in[m];
    float g = (a.dloss ? a.dloss[a.g_step ? m : 0] : 1.f) * a.scale;
    teach.form(a, red_t, red_u);
    g *= teach.unit;
    put_list(col, prob, teach.l, teach.p, a.top);
    auto share = [&](float x) {
        const float d = __builtin_fmaf(x, a.scale, -lse);
        return lse == neg_inf() ? 0.f : __builtin_amdgcn_exp2f(d * kLog2e);
    };
#pragma unroll
    for (int i = 0; i < KPT; i++) q[i] = share(z[i]);
    T* dx = (T*)a.dx + m * a.lddx;
#pragma unroll
    for (int i = 0; i < VPT; i++) end_logits(p[i], c0 + (i * NT + t) * CH, V);
    __syncthreads();   // every load of the part has returned
#pragma unroll
    for (int i = 0; i < VPT; i++) {
        const int c = c0 + (i * NT + t) * CH;
        if (c >= V) continue;
        float v[CH];
        logit_values(p[i], v);
#pragma unroll
        for (int e = 0; e < CH; e++) v[e] = teach.any ? g * share(v[e]) : 0.f;
        store_some(dx + c, V - c, v);
    }
    if (!teach.any) return;
    __syncthreads();
    put_listed(a, dx, col, prob, teach.l, q, g, c0, c1);
}

// ---------------------------------------------------------------- choice
// Kernels by the columns that a workgroup holds.
struct Shape {
    int nw, vpt;
    constexpr int cols() const { return 64 * nw * vpt * CH; }
};
constexpr Shape kShapes[] = {{1, 1}, {1, 4}, {4, 2}, {4, 4}, {16, 2}, {16, 4}, {16, 8}, {16, 16}};
constexpr int kShapeCount = 8;

// Calls f with the shape's sizes as constants.
template <typename F>
hipError_t by_shape(int shape, F f) {
    switch (shape) {
        case 0: return f(std::integral_constant<int, 1>(), std::integral_constant<int, 1>());
        case 1: return f(std::integral_constant<int, 1>(), std::integral_constant<int, 4>());
        case 2: return f(std::integral_constant<int, 4>(), std::integral_constant<int, 2>());
        case 3: return f(std::integral_constant<int, 4>(), std::integral_constant<int, 4>());
        case 4: return f(std::integral_constant<int, 16>(), std::integral_constant<int, 2>());
        case 5: return f(std::integral_constant<int, 16>(), std::integral_constant<int, 4>());
        case 6: return f(std::integral_constant<int, 16>(), std::integral_constant<int, 8>());
        default: return f(std::integral_constant<int, 16>(), std::integral_constant<int, 16>());
    }
}

struct Plan {
    int shape, parts;
};
// The smallest shape that holds a whole row; a longer row in parts of the largest.
Plan whole_rows(int64_t V, int type) {
    const int most = type == NITI_F32 ? 6 : 7;   // (16 pieces of 32 bits a thread are all the registers there are)
    for (int i = 0; i <= most; i++)
        if (V <= kShapes[i].cols()) return Plan{i, 1};
    return Plan{most, (int)((V + kShapes[most].cols() - 1) / kShapes[most].cols())};
}
// Few long rows: parts for all CUs.
Plan split_rows(int64_t M, int64_t V, int type) {
    Plan p = whole_rows(V, type);
    while (p.shape > 2 && M * p.parts < 128 && (V + kShapes[p.shape].cols() / 2 - 1) / (kShapes[p.shape].cols() / 2) <= kPartsMax && V > 32768) {
        p.shape--;
        p.parts = (int)((V + kShapes[p.shape].cols() - 1) / kShapes[p.shape].cols());
    }
    return p;
}

// A launch holds fewer than 2^32 threads: very many rows go in slabs.
constexpr int64_t kSlab = (int64_t)1 << 21;

inline size_t up256(size_t v) { return (v + 255) / 256 * 256; }

size_t log_space(int64_t M, int parts, int64_t top) {
    return parts > 1 ? up256((size_t)M * parts * sizeof(Stat)) + 2 * up256((size_t)M * parts * (size_t)top * 4) : 0;
}

template <typename T>
hipError_t run_logprobs(LogArgs a, const Plan& plan, char* ws, hipStream_t stream) {
    a.parts = plan.parts;
    const int64_t M = a.M, slab = kSlab / plan.parts;
    if (plan.parts > 1) {
        a.stat = (Stat*)ws;
        a.val = (float*)(ws + up256((size_t)M * a.parts * sizeof(Stat)));
        a.col = (int32_t*)((char*)a.val + up256((size_t)M * a.parts * a.top * 4));
    }
    for (int64_t m0 = 0; m0 < M; m0 += slab) {
        a.M = M - m0 < slab ? M - m0 : slab;
        hipError_t e = by_shape(plan.shape, [&](auto nw, auto vpt) {
            constexpr int NW = decltype(nw)::value, VPT = decltype(vpt)::value;
            if constexpr (sizeof(T) * VPT <= 32)
                hipLaunchKernelGGL((logprobs_kernel<T, NW, VPT>), dim3((unsigned)(a.M * a.parts)), dim3(64 * NW), 0, stream, a);
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
}

template <typename T>
hipError_t run_distill_bwd(DistArgs a, hipStream_t stream) {
    // 8192 columns a workgroup where rows are longer than that
    int shape = 0;
    while (shape < 3 && a.V > kShapes[shape].cols()) shape++;
    a.parts = (int)((a.V + kShapes[shape].cols() - 1) / kShapes[shape].cols());
    const int64_t M = a.M, slab = kSlab / a.parts;
    for (int64_t m0 = 0; m0 < M; m0 += slab) {
        a.M = M - m0 < slab ? M - m0 : slab;
        const hipError_t e = by_shape(shape, [&](auto nw, auto vpt) {
            constexpr int NW = decltype(nw)::value, VPT = decltype(vpt)::value;
            if constexpr (NW <= 4)
                hipLaunchKernelGGL((distill_bwd_kernel<T, NW, VPT>), dim3((unsigned)(a.M * a.parts)), dim3(64 * NW), 0, stream, a);
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
    const DistArgs whole = a;
    const int64_t M = a.M, slab = kSlab / plan.parts;
    const bool grad = a.dx && plan.parts == 1;
    if (plan.parts > 1) {
        a.stat = (Stat*)ws;
        if (a.dx && !a.lse) a.lse = (float*)(ws + up256((size_t)M * a.parts * sizeof(Stat)));
    }
    const float* lse = a.lse;
    for (int64_t m0 = 0; m0 < M; m0 += slab) {
        a.M = M - m0 < slab ? M - m0 : slab;
        hipError_t e = by_shape(plan.shape, [&](auto nw, auto vpt) {
            constexpr int NW = decltype(nw)::value, VPT = decltype(vpt)::value;
            if constexpr (sizeof(T) * VPT <= 32) {
                if (grad)
                    hipLaunchKernelGGL((distill_kernel<T, NW, VPT, true>), dim3((unsigned)(a.M * a.parts)), dim3(64 * NW), 0, stream, a);
                else
                    hipLaunchKernelGGL((distill_kernel<T, NW, VPT, false>), dim3((unsigned)(a.M * a.parts)), dim3(64 * NW), 0, stream, a);
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
    DistArgs b = whole;
    b.lse_in = lse;
    return run_distill_bwd<T>(b, stream);
}

inline bool fine_scale(float s) { return s > 0.f && s < INFINITY; }

}  // namespace

// For either type's plan: the caller's sizes do not say which.
size_t logprobs_workspace(int64_t M, int64_t V, int64_t top) {
    if (M < 1 || V < 1 || top < 0 || top > kTopMax || top > V || M >= kMaxDim || V >= kMaxLd) return 0;
    const size_t wide = log_space(M, split_rows(M, V, NITI_F32).parts, top), half = log_space(M, split_rows(M, V, NITI_BF16).parts, top);
    return wide > half ? wide : half;
}
size_t distill_workspace(int64_t M, int64_t V) {
    if (M < 1 || V < 1 || M >= kMaxDim || V >= kMaxLd) return 0;
    const int wide = whole_rows(V, NITI_F32).parts, half = whole_rows(V, NITI_BF16).parts;
    const int parts = wide > half ? wide : half;
    return parts > 1 ? up256((size_t)M * parts * sizeof(Stat)) + up256((size_t)M * 4) : 0;
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
    const Plan plan = split_rows(M, V, type);
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
    const Plan plan = whole_rows(V, type);
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
    return by_type(type, [&](auto t) { return run_distill_bwd<decltype(t)>(a, (hipStream_t)stream); }) == hipSuccess
               ? NITI_OK : NITI_ERR_HIP;
}

}  // extern "C"
