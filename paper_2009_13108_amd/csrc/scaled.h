// Shared pieces of the operators on int8 rows with one scale each: element
// types, int8 codes of a float row, stochastic draws, activations.
//
// A row x is held as codes q and a scale: x ~ q * scale with
//   top = max(max |x|, 2^-100), scale = top / 127, q = round(x * (127 / top)),
// so that a row of zeros has a scale like any other and nothing divides by
// zero.  A row with an infinity or a NaN has the scale NaN and codes 0: what
// is computed from it is NaN, as it would be without the codes.
#pragma once

#include "niti_internal.h"

namespace niti {

typedef _Float16 f16;
typedef float v4f __attribute__((ext_vector_type(4)));

constexpr float kTopMin = 0x1p-100f;
constexpr uint32_t kInfBits = 0x7F800000u;

struct bf16 {
    uint16_t bits;
};

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(f16 v) { return (float)v; }
__device__ __forceinline__ float to_f(bf16 v) { return __uint_as_float((uint32_t)v.bits << 16); }

// Results are held in 32 bits up to the store, which rounds once, to nearest even.
template <typename T>
__device__ __forceinline__ T from_f(float v);
template <>
__device__ __forceinline__ float from_f<float>(float v) { return v; }
template <>
__device__ __forceinline__ f16 from_f<f16>(float v) { return (f16)v; }
template <>
__device__ __forceinline__ bf16 from_f<bf16>(float v) {
    return __builtin_bit_cast(bf16, (__bf16)v);
}

// N consecutive elements from any address (see load16_any).
template <typename T, int N>
__device__ __forceinline__ void load_n(const T* p, float (&v)[N]) {
    T t[N];
    __builtin_memcpy(t, p, sizeof(t));
#pragma unroll
    for (int i = 0; i < N; i++) v[i] = to_f(t[i]);
}
template <typename T, int N>
__device__ __forceinline__ void store_n(T* p, const float (&v)[N]) {
    T t[N];
#pragma unroll
    for (int i = 0; i < N; i++) t[i] = from_f<T>(v[i]);
    __builtin_memcpy(p, t, sizeof(t));
}
// The first n of them (n >= N: all), zero for the others.
template <typename T, int N>
__device__ __forceinline__ void load_some(const T* p, int n, float (&v)[N]) {
    if (n >= N) {
        load_n(p, v);
        return;
    }
#pragma unroll
    for (int i = 0; i < N; i++) v[i] = i < n ? to_f(p[i]) : 0.f;
}
template <typename T, int N>
__device__ __forceinline__ void store_some(T* p, int n, const float (&v)[N]) {
    if (n >= N) {
        store_n(p, v);
        return;
    }
#pragma unroll
    for (int i = 0; i < N; i++)
        if (i < n) p[i] = from_f<T>(v[i]);
}

// Eight elements as they are loaded.  A load inside a branch is waited for where the
// branch ends, so a kernel that is to have many in flight has none of them in a
// branch: a piece past the row's end is loaded from inside it and set to zeros,
// a row's last, partial piece as the row's last eight elements, moved down.
// WHOLE: the row's length is a multiple of 8, and there are no partial pieces.
constexpr int CH = 8;
template <typename T>
struct Piece {
    uint32_t w[CH * sizeof(T) / 4];
};
template <typename T, bool WHOLE>
__device__ __forceinline__ Piece<T> load_piece(const T* row, int c, int D) {   // D >= 8
    const int from = min(c, D - CH);
    Piece<T> p;
    __builtin_memcpy(p.w, row + from, sizeof(p.w));
    return p;
}
// The piece's values once it is used: those of column c on, zeros past D.
template <typename T, bool WHOLE>
__device__ __forceinline__ void piece_values(Piece<T> p, int c, int D, float (&v)[CH]) {
    constexpr int W = CH * sizeof(T) / 4, PER = 4 / sizeof(T);   // words, elements of a word
    const bool out = c >= D;
    if (!WHOLE) {
        const int down = out ? 0 : c - min(c, D - CH);   // elements, 0..7
        if (PER == 2) {
            const bool odd = down & 1;
#pragma unroll
            for (int i = 0; i < W; i++) p.w[i] = odd ? p.w[i] >> 16 | (i + 1 < W ? p.w[i + 1 < W ? i + 1 : i] << 16 : 0u) : p.w[i];
        }
#pragma unroll
        for (int b = 1; b < W; b *= 2) {
            const bool move = (down / PER) & b;
#pragma unroll
            for (int i = 0; i < W; i++) p.w[i] = move ? (i + b < W ? p.w[i + b < W ? i + b : i] : 0u) : p.w[i];
        }
    }
#pragma unroll
    for (int i = 0; i < W; i++) p.w[i] = out ? 0u : p.w[i];
    T t[CH];
    __builtin_memcpy(t, p.w, sizeof(t));
#pragma unroll
    for (int i = 0; i < CH; i++) v[i] = to_f(t[i]);
}

// Elements i .. i+N-1 of a vector of a type known at run time (gains and
// biases, which are small; uniform).
template <int N>
__device__ __forceinline__ void load_typed(const void* p, int type, int64_t i, int n, float (&v)[N]) {
    if (type == NITI_F32)
        load_some((const float*)p + i, n, v);
    else if (type == NITI_BF16)
        load_some((const bf16*)p + i, n, v);
    else
        load_some((const f16*)p + i, n, v);
}

inline size_t type_size(int type) { return type == NITI_F32 ? 4 : 2; }
template <typename T>
constexpr int type_id() { return sizeof(T) == 4 ? NITI_F32 : (__is_same(T, bf16) ? NITI_BF16 : NITI_F16); }
inline bool valid_type(int type) { return type == NITI_F32 || type == NITI_BF16 || type == NITI_F16; }

// |v| as an integer of the same order; every NaN is above infinity, so that a
// maximum of these keeps what a floating maximum drops.
__device__ __forceinline__ uint32_t mag_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

// Codes of one row (or column): the scale, and the factor that forms them.
struct RowScale {
    float scale;   // NaN for a row that is not finite
    float inv;     // 0 for such a row
};
__device__ __forceinline__ RowScale row_scale(uint32_t top_bits) {
    RowScale r;
    const bool bad = top_bits >= kInfBits;
    const float top = fmaxf(__uint_as_float(top_bits), kTopMin);
    r.scale = bad ? __uint_as_float(0x7FC00000u) : top / 127.f;
    r.inv = bad ? 0.f : 127.f / top;
    return r;
}

// Codes as floats that begin at kCode = 1.5 * 2^23: there a step of a float is 1,
// so that adding it rounds v * inv to the nearest integer, ties to even, and
// leaves the code as the float's lowest byte.  The product is rounded first: of
// 16-bit values many lie half way between two codes (half a row's largest is 63.5
// steps), where the rounding takes back that of inv; one multiply-add would go by
// inv's error there (a fifth more distance from the exact codes).  For a
// finite row |v * inv| is at most 127 and a rounding error, which rounds to 127.  Rows that
// are not finite (inv 0) may leave anything: their words are masked (see code_mask).
constexpr float kCode = 12582912.f;
__device__ __forceinline__ float code_rtn(float v, float inv) {
#pragma clang fp contract(off)
    const float r = v * inv;
    return r + kCode;
}
// Stochastically: floor(v * inv + u) is v * inv on average over u in [0, 1).
__device__ __forceinline__ float code_sr(float v, float inv, float u) {
#pragma clang fp contract(off)
    const float r = v * inv;
    return __builtin_amdgcn_fmed3f(floorf(r + u), -127.f, 127.f) + kCode;
}
__device__ __forceinline__ float code_value(float c) { return c - kCode; }
// All bits for a row with codes, none for one without.
__device__ __forceinline__ uint32_t code_mask(float inv) { return inv > 0.f ? ~0u : 0u; }
// Four codes in a word, lowest first.
__device__ __forceinline__ uint32_t pack4(float a, float b, float c, float d) {
    const uint32_t lo = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x0C0C0400);
    const uint32_t hi = __builtin_amdgcn_perm(__float_as_uint(d), __float_as_uint(c), 0x04000C0C);
    return lo | hi;
}
// Consecutive draws idx, idx + 1, ... of sr_draw: its first product is carried as a sum.
struct DrawStream {
    uint64_t z;
    __device__ __forceinline__ DrawStream(uint64_t seed, uint32_t call, uint64_t idx)
        : z(seed + ((((uint64_t)call) << 40) + idx) * 0x9E3779B97F4A7C15ull) {}
    __device__ __forceinline__ uint64_t next() {
        z += 0x9E3779B97F4A7C15ull;
        uint64_t x = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
        x = (x ^ (x >> 27)) * 0x94D049BB133111EBull;
        return x ^ (x >> 31);
    }
};

// Uniform fractions of 24 bits from a draw.
__device__ __forceinline__ float draw_hi(uint64_t r) { return (float)(uint32_t)(r >> 40) * 0x1p-24f; }
__device__ __forceinline__ float draw_lo(uint64_t r) { return (float)((uint32_t)(r >> 8) & 0xFFFFFFu) * 0x1p-24f; }

__device__ __forceinline__ float wave_sum_f32(float v) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o, kWave);
    return v;
}

// exp(x) for |x| <= 80 by the hardware's power of two.  The rounding of x log2(e)
// leaves a relative error of |x| 2^-24: in a sigmoid that is at most s (1 - s) |x| 2^-24 <
// 0.23 * 2^-24.  SiLU in 32 bits is up to 1.2e-6 off (z near 12), as the plain form is, and up to 9e-7 of
// its value, z / (1 + exp(-z)) with the library's expf 1.6e-7.  That and an IEEE division cost ten
// instructions each; with them the slopes alone bounded the passes over a gradient.
__device__ __forceinline__ float exp_mid(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504088896341f); }
__device__ __forceinline__ float sigmoid_mid(float x) { return __builtin_amdgcn_rcpf(1.f + exp_mid(-x)); }

__device__ __forceinline__ float half_exp(float s) { return __builtin_amdgcn_exp2f(s * (-0.5f * 1.44269504088896341f)); }   // exp(-s / 2)

// The normal distribution function at z >= -12.5 from s = z^2 and e = exp(-s / 2): about 0
// it is 1/2 + z P(z^2), beyond that the tail outside |z| is e Q(t) with t = 1 / (1 + 0.4 |z|),
// which keeps its relative error however small it is.  P and Q are fitted in 64
// bits for the least largest error: P within 2.1e-9 of the function for |z| < 1.25, Q within 9e-9
// of the tail, relative, from there to 12.5.  In 32 bits GELU is then nowhere further from
// its exact value than z (1 + erf(z / sqrt 2)) / 2 is, which loses the tail of negative z.
// A five-term error function costs less (4096 x 4096 x 512 to bf16 39.9 us for 42.5 on the same card,
// 1000 x 1500 x 1111 in 32 bits 15.4 for 15.5) and was up to 3e-2 of the value off there.
__device__ __forceinline__ float normal_cdf(float z, float s, float e) {
    float p = __builtin_fmaf(s, -6.66287769e-06f, 0.000110409092f);
    p = __builtin_fmaf(s, p, -0.00118284649f);
    p = __builtin_fmaf(s, p, 0.00997160375f);
    p = __builtin_fmaf(s, p, -0.0664900169f);
    p = __builtin_fmaf(s, p, 0.398942262f);
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(fabsf(z), 0.4f, 1.f));
    float q = __builtin_fmaf(t, 0.0714648142f, -0.195115626f);
    q = __builtin_fmaf(t, q, 0.11459253f);
    q = __builtin_fmaf(t, q, 0.0503757186f);
    q = __builtin_fmaf(t, q, 0.140635118f);
    q = __builtin_fmaf(t, q, 0.158810765f);
    q = __builtin_fmaf(t, q, 0.159622088f);
    q = __builtin_fmaf(t, q, -9.34627906e-07f);
    q *= e;   // the tail beyond |z|
    const float far = z < 0.f ? q : 1.f - q;
    return fabsf(z) < 1.25f ? __builtin_fmaf(z, p, 0.5f) : far;
}

// Activations and their derivatives.  Arguments are held where a sigmoid or a
// tail is below 2^-115, so that an infinity gives the limit and no NaN.
__device__ __forceinline__ float act_value(int act, float z) {
    if (act == NITI_ACT_RELU) return z < 0.f ? 0.f : z;
    if (act == NITI_ACT_GELU) {
        const float c = z < -12.5f ? -12.5f : z;   // (upwards the tail ends at 0 by itself)
        return c * normal_cdf(c, c * c, half_exp(c * c));
    }
    if (act == NITI_ACT_SILU) {
        const float c = z < -80.f ? -80.f : z;
        return c * sigmoid_mid(c > 80.f ? 80.f : c);
    }
    return z;
}
__device__ __forceinline__ float act_slope(int act, float z) {
    if (act == NITI_ACT_RELU) return z > 0.f ? 1.f : (z <= 0.f ? 0.f : z);
    if (act == NITI_ACT_GELU) {
        const float c = z < -12.5f ? -12.5f : (z > 12.5f ? 12.5f : z);
        const float e = half_exp(c * c);
        return normal_cdf(c, c * c, e) + c * e * 0.39894228040143268f;
    }
    if (act == NITI_ACT_SILU) {
        const float c = z < -80.f ? -80.f : (z > 80.f ? 80.f : z);
        const float s = sigmoid_mid(c);
        return s * (1.f + c * (1.f - s));
    }
    return 1.f;
}
// The same of several values: the choice is made once.
template <int N>
__device__ __forceinline__ void act_values(int act, float (&v)[N]) {
    if (act == NITI_ACT_RELU) {
#pragma unroll
        for (int e = 0; e < N; e++) v[e] = act_value(NITI_ACT_RELU, v[e]);
    } else if (act == NITI_ACT_GELU) {
#pragma unroll
        for (int e = 0; e < N; e++) v[e] = act_value(NITI_ACT_GELU, v[e]);
    } else if (act == NITI_ACT_SILU) {
#pragma unroll
        for (int e = 0; e < N; e++) v[e] = act_value(NITI_ACT_SILU, v[e]);
    }
}
constexpr int64_t kMaxLd = (int64_t)1 << 22;   // row strides are below this
constexpr int64_t kMaxDim = (int64_t)1 << 31;
constexpr int64_t kMaxSum = (int64_t)1 << 17;   // shorter sums of int8 products stay in int32

// A row stride: 0 only for operands that are read.
inline bool bad_ld(int64_t ld, int64_t cols, bool out) {
    return ld >= kMaxLd || ld < 0 || (ld < cols && (out || ld != 0));
}

// The slopes of several values, in their place.
template <int N>
__device__ __forceinline__ void act_slopes(int act, float (&v)[N]) {
    if (act == NITI_ACT_RELU) {
#pragma unroll
        for (int e = 0; e < N; e++) v[e] = act_slope(NITI_ACT_RELU, v[e]);
    } else if (act == NITI_ACT_GELU) {
#pragma unroll
        for (int e = 0; e < N; e++) v[e] = act_slope(NITI_ACT_GELU, v[e]);
    } else if (act == NITI_ACT_SILU) {
#pragma unroll
        for (int e = 0; e < N; e++) v[e] = act_slope(NITI_ACT_SILU, v[e]);
    }
}

// Calls f(T()) with the element type.
template <typename F>
inline hipError_t by_type(int type, F f) {
    if (type == NITI_F32) return f(float());
    if (type == NITI_BF16) return f(bf16());
    return f(f16());
}

}  // namespace niti
