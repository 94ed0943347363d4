// Kernels of the product of int8 rows, which linear.hip launches as they are and
// gated.hip with pairs of columns (G).
//
// A gated product has the weights of both projections in one operand of 2 N rows, a
// column n of the result from rows n (the gate) and n + N of it.  A tile of BN
// weight rows takes 32 (few products: 16) gates and then their 32 partners, and so
// on, so that the wave that has a gate's sum has its partner's in the same
// registers and lane: the activation and the product cost no exchange.
#pragma once

#include "linear.h"

#include <math.h>

#include <type_traits>
#include <utility>

namespace niti {

namespace {

// ---------------------------------------------------------------- epilogue
// Accumulators are 32 x 32 tiles acc[a][b] (channels a, rows b): element 4 j + i
// of a lane is channel 32 a + 8 j + 4 (lane / 32) + i of row 32 b + lane % 32.  The
// epilogue works on them where they are (a lane has one row scale per b, and
// four channels at a time), rounds, and turns the tile through LDS, so that
// whole 16-byte pieces of rows are stored.  The residual comes the other way:
// its tile is loaded into the same LDS places, by direct-to-LDS loads all in
// flight at once where its rows are aligned, and each lane adds its four values
// and puts the sums back.
//
// All tiles of a wave share one copy of this code (the accumulators are picked
// by uniform branches): with the loops unrolled, the activations' code outgrew
// the instruction cache and a 256 x 256 tile's epilogue took 16 us alone.
template <typename T, int BM, int BN, int WGM, int WGN, int ROOM>
struct Stage {
    static constexpr int NT = 64 * WGM * WGN;
    static constexpr int WTM = BM / WGM, WTN = BN / WGN, FM = WTM / 32, FN = WTN / 32;
    static constexpr int PPR = BN * (int)sizeof(T) / 16;     // pieces of a row
    static constexpr int EPP = 16 / (int)sizeof(T);          // elements of a piece
    // row tiles b of a wave that are turned at a time: what ROOM bytes hold
    static constexpr int BG = BM * BN * (int)sizeof(T) <= ROOM ? FM : (BM * BN * (int)sizeof(T) <= 2 * ROOM ? FM / 2 : FM / 4);
    static_assert(BG >= 1 && BG * FN >= 1, "room for one row tile of each wave");
    static constexpr int ROWS = 32 * BG * WGM;
    static constexpr int PIECES = ROWS * PPR;
    static_assert(PIECES % (64 * WGM * WGN) == 0, "whole load instructions");
    // LDS piece of piece p of row r: rows that a lane group takes one column of hit distinct banks
    static __device__ __forceinline__ int at(int r, int p) { return r * PPR + (p ^ (r & (PPR < 32 ? PPR - 1 : 31))); }
    // row of the tile that row r of the turned rows is, for the group from b0 on
    static __device__ __forceinline__ int tile_row(int r, int b0) { return r / (32 * BG) * WTM + b0 * 32 + r % (32 * BG); }
};

// x = acc[want] by uniform branches over constant indices: the accumulators stay in registers.
template <int FN, int FM, int... I>
__device__ __forceinline__ void pick(v16i (&acc)[FN][FM], int want, v16i& x, std::integer_sequence<int, I...>) {
    ((want == I ? (void)(x = acc[I / FM][I % FM]) : (void)0), ...);
}

// Operands of the epilogue that a call may not have are read from these, so that
// no load is in a branch, where it would be waited for.
__device__ const float kOnes[1] = {1.f};
__device__ const float kZeros[1] = {0.f};

// One bias as loaded, of a type known at run time: from one of two places, the other gives zero.
struct BiasLoad {
    uint32_t wide;
    uint16_t narrow;
    __device__ __forceinline__ void load(const LinArgs& A, int64_t n) {
        const bool f32 = A.bias && A.bias_type == NITI_F32, f16 = A.bias && A.bias_type != NITI_F32;
        wide = (f32 ? (const uint32_t*)A.bias : (const uint32_t*)kZeros)[f32 ? n : 0];
        narrow = (f16 ? (const uint16_t*)A.bias : (const uint16_t*)kZeros)[f16 ? n : 0];
    }
    __device__ __forceinline__ float get(const LinArgs& A) const {
        const uint16_t h = narrow;
        const float half = A.bias_type == NITI_F16 ? to_f(__builtin_bit_cast(f16, h)) : to_f(bf16{h});
        return A.bias_type == NITI_F32 ? __uint_as_float(wide) : half;
    }
};
__device__ __forceinline__ float load_scale(const float* s, int step, int64_t i) { return (s ? s : kOnes)[s && step ? i : 0]; }

// Row of a tile's weights among those of its gates, or of their partners (blocks of 1 << SH in turn).
template <int SH>
__device__ __forceinline__ int pair_row(int v) { return (v >> (SH + 1) << SH) + (v & ((1 << SH) - 1)); }
template <int SH>
__device__ __forceinline__ int pair_half(int v) { return v >> SH & 1; }

// Scales and biases of a tile's columns and scales of its rows, to LDS before
// the sum begins: loaded in the epilogue they cost it two memory round trips.
template <int BM, int BN, int NT, bool G = false>
__device__ __forceinline__ void load_params(const LinArgs& A, float* par, int64_t m0, int64_t n0) {
    static_assert(NT >= BM && NT >= BN, "one column and one row a thread");
    const int t = threadIdx.x, v = t % BN;
    const int64_t n = G ? min(n0 + pair_row<5>(v), A.N - 1) + pair_half<5>(v) * A.N : min(n0 + v, A.N - 1);
    const int64_t m = min(m0 + t % BM, A.M - 1);
    BiasLoad bias;
    bias.load(A, n);
    const float sb = load_scale(A.s_b, A.b_step, n), sa = load_scale(A.s_a, A.a_step, m);
    if (t < BN) {
        par[t] = sb;
        par[BN + t] = bias.get(A);
    }
    if (t < BM) par[2 * BN + t] = sa;
}

// A workgroup's part of a split sum: its stretch of K, and its place in the sums (int32_t).
template <typename T>
__device__ __forceinline__ void take_part(LinArgs& A) {
    if constexpr (__is_same(T, int32_t)) {
        const int64_t k0 = (int64_t)blockIdx.y * A.klen;
        A.a += k0;
        A.b += k0;
        A.K = min((int64_t)A.klen, A.K - k0);
        A.out = (int32_t*)A.out + blockIdx.y * A.part;
    }
}

// T: the result's type, or int32_t for a part of a split sum, which is stored as it is.
template <typename T, int BM, int BN, int WGM, int WGN, int ROOM>
__device__ __forceinline__ void epilogue(const LinArgs& A, v16i (&acc)[BN / WGN / 32][BM / WGM / 32], int8_t* lds, const float* par,
                                         int64_t m0, int64_t n0) {
    using S = Stage<T, BM, BN, WGM, WGN, ROOM>;
    constexpr int FM = S::FM, FN = S::FN, BG = S::BG;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave % WGM, wn = wave / WGM;
    const int rows = (int)min((int64_t)BM, A.M - m0), ncol = (int)min((int64_t)BN, A.N - n0);
#pragma unroll 1
    for (int b0 = 0; b0 < FM; b0 += BG) {
#pragma unroll 1
        for (int kind = A.z ? 0 : 1; kind < 2; kind++) {   // z, then out
            const bool add = kind == 1 && A.res;
            if (add && A.res_dma) {
                // The descriptor's range is checked by 32-bit words, and a word that it cuts loads zeros: it ends after
                // the word that holds the last element (the residual's address is a multiple of 16).
                const u32x4 rs = raw_rsrc((const T*)A.res + m0 * A.ldres + n0,
                                          (uint32_t)(((int64_t)(rows - 1) * A.ldres + ncol) * (int64_t)sizeof(T) + 3) & ~3u);
                const uint32_t base = lds_address(lds);
#pragma unroll 4
                for (int i = 0; i < S::PIECES / S::NT; i++) {
                    const int slot = (i * (S::NT / 64) + wave) * 64 + lane;
                    const int r = slot / S::PPR, p = S::at(r, slot % S::PPR) - r * S::PPR;
                    lds_dma16(rs, base + (uint32_t)((i * (S::NT / 64) + wave) * 1024),
                              (uint32_t)S::tile_row(r, b0) * (uint32_t)(A.ldres * (int64_t)sizeof(T)) + (uint32_t)(p * 16), 0);
                }
                __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt 0
            } else if (add) {
                for (int slot = threadIdx.x; slot < S::PIECES; slot += S::NT) {
                    const int r = slot / S::PPR, p = slot % S::PPR;
                    const int m = min(S::tile_row(r, b0), rows - 1), nv = ncol - p * S::EPP;
                    const T* src = (const T*)A.res + (m0 + m) * A.ldres + n0 + p * S::EPP;
                    T v[S::EPP] = {};
                    if (nv >= S::EPP) {
                        __builtin_memcpy(v, src, 16);
                    } else {
#pragma unroll
                        for (int e = 0; e < S::EPP; e++)
                            if (e < nv) v[e] = src[e];
                    }
                    __builtin_memcpy(lds + S::at(r, p) * 16, v, 16);
                }
            }
            __syncthreads();
#pragma unroll 1
            for (int t = 0; t < FN * BG; t++) {
                const int ta = t / BG, tb = t % BG;
                v16i x = acc[0][0];
                pick(acc, ta * FM + b0 + tb, x, std::make_integer_sequence<int, FN * FM>());
                const int row = tb * 32 + (lane & 31);                    // of the wave's turned rows
                const int r = wm * 32 * BG + row;
                const int c0 = wn * S::WTN + ta * 32 + 4 * (lane >> 5);   // this lane's columns: c0 + 8 j + e
                T* at[4];
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    const int c = c0 + 8 * j;
                    at[j] = (T*)(lds + S::at(r, c / S::EPP) * 16) + c % S::EPP;
                }
                if constexpr (__is_same(T, int32_t)) {
#pragma unroll
                    for (int j = 0; j < 4; j++) *(v4i*)at[j] = v4i{x[4 * j], x[4 * j + 1], x[4 * j + 2], x[4 * j + 3]};
                } else {
                    const float sa = par[2 * BN + wm * S::WTM + b0 * 32 + row];
                    v4f sb[4], bias[4];
#pragma unroll
                    for (int j = 0; j < 4; j++) {
                        sb[j] = *(const v4f*)(par + c0 + 8 * j);
                        bias[j] = *(const v4f*)(par + BN + c0 + 8 * j);
                    }
                    float v[16];
#pragma unroll
                    for (int e = 0; e < 16; e++) v[e] = (float)x[e] * sb[e >> 2][e & 3] * sa + bias[e >> 2][e & 3];
                    if (kind == 1 && A.act != NITI_ACT_NONE) act_values(A.act, v);
                    if (add) {
                        float res[4][4];
#pragma unroll
                        for (int j = 0; j < 4; j++) load_n(at[j], res[j]);
#pragma unroll
                        for (int e = 0; e < 16; e++) v[e] += res[e >> 2][e & 3];
                    }
#pragma unroll
                    for (int j = 0; j < 4; j++) {
                        const float w[4] = {v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]};
                        store_n(at[j], w);
                    }
                }
            }
            __syncthreads();
            T* out = (T*)(kind ? A.out : A.z) + m0 * (kind ? A.ldout : A.ldz) + n0;
            const int64_t ld = kind ? A.ldout : A.ldz;
#pragma unroll 4
            for (int i = 0; i < S::PIECES / S::NT; i++) {
                const int slot = i * S::NT + threadIdx.x;
                const int r = slot / S::PPR, p = slot % S::PPR;
                const int m = S::tile_row(r, b0), nv = ncol - p * S::EPP;
                const uint4 v = *(const uint4*)(lds + S::at(r, p) * 16);
                if (m >= rows || nv <= 0) continue;
                T* dst = out + m * ld + p * S::EPP;
                if (nv >= S::EPP) {
                    store16_any(dst, v);
                } else {
                    T e[S::EPP];
                    __builtin_memcpy(e, &v, 16);
#pragma unroll
                    for (int k = 0; k < S::EPP; k++)
                        if (k < nv) dst[k] = e[k];
                }
            }
            if (kind == 0 || b0 + BG < FM) __syncthreads();
        }
    }
}

// The same for pairs: z's gates, z's partners and act(gate) * partner, each turned through LDS
// as a tile of BN / 2 columns.
template <typename T, int BM, int BN, int WGM, int WGN, int ROOM>
__device__ __forceinline__ void gated_epilogue(const LinArgs& A, v16i (&acc)[BN / WGN / 32][BM / WGM / 32], int8_t* lds, const float* par,
                                               int64_t m0, int64_t n0) {
    using S = Stage<T, BM, BN / 2, WGM, WGN, ROOM>;
    constexpr int FM = S::FM, FN = S::FN, BG = S::BG;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave % WGM, wn = wave / WGM;
    const int rows = (int)min((int64_t)BM, A.M - m0), ncol = (int)min((int64_t)(BN / 2), A.N - n0);
#pragma unroll 1
    for (int b0 = 0; b0 < FM; b0 += BG) {
#pragma unroll 1
        for (int kind = A.z ? 0 : 2; kind < 3; kind++) {
#pragma unroll 1
            for (int t = 0; t < FN * BG; t++) {
                const int ta = t / BG, tb = t % BG;
                v16i x = acc[0][0], y = acc[1][0];
                pick(acc, 2 * ta * FM + b0 + tb, x, std::make_integer_sequence<int, 2 * FN * FM>());
                pick(acc, (2 * ta + 1) * FM + b0 + tb, y, std::make_integer_sequence<int, 2 * FN * FM>());
                const int row = tb * 32 + (lane & 31);
                const int r = wm * 32 * BG + row;
                const int c0 = wn * S::WTN + ta * 32 + 4 * (lane >> 5);       // this lane's columns: c0 + 8 j + e
                const int v0 = wn * 2 * S::WTN + ta * 64 + 4 * (lane >> 5);   // their gates' places in par
                const float sa = par[2 * BN + wm * S::WTM + b0 * 32 + row];
                float gate[16], up[16];
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    const v4f sg = *(const v4f*)(par + v0 + 8 * j), bg = *(const v4f*)(par + BN + v0 + 8 * j);
                    const v4f su = *(const v4f*)(par + v0 + 32 + 8 * j), bu = *(const v4f*)(par + BN + v0 + 32 + 8 * j);
#pragma unroll
                    for (int e = 0; e < 4; e++) {
                        gate[4 * j + e] = (float)x[4 * j + e] * sg[e] * sa + bg[e];
                        up[4 * j + e] = (float)y[4 * j + e] * su[e] * sa + bu[e];
                    }
                }
                if (kind == 2) {
                    act_values(A.act, gate);
#pragma unroll
                    for (int e = 0; e < 16; e++) gate[e] *= up[e];
                }
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    const int c = c0 + 8 * j;
                    float w[4];
#pragma unroll
                    for (int e = 0; e < 4; e++) w[e] = kind == 1 ? up[4 * j + e] : gate[4 * j + e];
                    store_n((T*)(lds + S::at(r, c / S::EPP) * 16) + c % S::EPP, w);
                }
            }
            __syncthreads();
            const int64_t ld = kind == 2 ? A.ldout : A.ldz;
            T* out = (T*)(kind == 2 ? A.out : A.z) + m0 * ld + n0 + (kind == 1 ? A.N : 0);
#pragma unroll 4
            for (int i = 0; i < S::PIECES / S::NT; i++) {
                const int slot = i * S::NT + threadIdx.x;
                const int r = slot / S::PPR, p = slot % S::PPR;
                const int m = S::tile_row(r, b0), nv = ncol - p * S::EPP;
                const uint4 v = *(const uint4*)(lds + S::at(r, p) * 16);
                if (m >= rows || nv <= 0) continue;
                T* dst = out + m * ld + p * S::EPP;
                if (nv >= S::EPP) {
                    if (kind < 2 && A.z_stream) __builtin_nontemporal_store(any_u32x4{v.x, v.y, v.z, v.w}, (any_u32x4*)dst);
                    else store16_any(dst, v);
                } else {
                    T e[S::EPP];
                    __builtin_memcpy(e, &v, 16);
#pragma unroll
                    for (int k = 0; k < S::EPP; k++)
                        if (k < nv) dst[k] = e[k];
                }
            }
            if (kind < 2 || b0 + BG < FM) __syncthreads();
        }
    }
}

// ---------------------------------------------------------------- any operands
// 16 bytes k .. k+15 of a row of K at any address, zeros past K.  A row's last,
// partial piece is read as the row's last 16 bytes and shifted.
__device__ __forceinline__ v4i row_piece(const int8_t* row, int k, int K) {
    if (k + 16 <= K) return __builtin_bit_cast(v4i, load16_any(row + k));
    if (k >= K) return v4i{0, 0, 0, 0};
    unsigned __int128 x = 0;
    if (K >= 16) {
        x = __builtin_bit_cast(unsigned __int128, load16_any(row + K - 16)) >> (8 * (k + 16 - K));
    } else {
        for (int i = K - 1; i >= k; i--) x = x << 8 | (uint8_t)row[i];
    }
    return __builtin_bit_cast(v4i, x);
}

// 64 x 64 tiles, four waves of 32 x 32, K steps of 128 bytes through two LDS
// stages, a thread's pieces of three steps in registers: with those of one step
// a step took a memory round trip, with steps of 64 bytes twice the barriers
// (1000 x 1500 x 1111 18.8 and 16.9 us).  The loads are in no branch, where
// each would be waited for: past a row's last whole piece they read that one, and
// the last step sets right what they gave.
constexpr int GT = 64, GK = 128, GA = 3;

__device__ __forceinline__ int gswz(int row) { return (row >> 1) & 7; }

// The piece at k of a row, as loaded from min(k, K - 16): zeros past K.
__device__ __forceinline__ v4i cut_piece(v4i v, int k, int K) {
    if (k + 16 <= K) return v;
    if (k >= K) return v4i{0, 0, 0, 0};
    return __builtin_bit_cast(v4i, __builtin_bit_cast(unsigned __int128, v) >> (8 * (k + 16 - K)));
}

template <typename T, bool G = false>
__global__ __launch_bounds__(256) void linear_any_kernel(LinArgs A, int tiles_n) {
    take_part<T>(A);
    __shared__ __attribute__((aligned(16))) int8_t lds[2][2 * GT * GK];
    __shared__ __attribute__((aligned(16))) float par[3 * GT];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t m0 = (int64_t)(blockIdx.x / tiles_n) * GT, n0 = (int64_t)(blockIdx.x % tiles_n) * (G ? GT / 2 : GT);
    // two pieces of each operand a thread, 64 bytes apart: rows past the edge read row 0, whose products are not stored
    const int row = threadIdx.x >> 2, pc = threadIdx.x & 3;
    const int8_t* ra = A.a + (m0 + row < A.M ? (m0 + row) * A.lda : 0);
    const int64_t nb = G ? n0 + pair_row<5>(row) : n0 + row;
    const int8_t* rb = A.b + (nb < A.N ? nb + (G ? pair_half<5>(row) * A.N : 0) : 0) * A.ldb;
    const int K = (int)A.K, nk = (K + GK - 1) / GK;
    v16i acc[1][1];
    acc[0][0] = v16i{};
    const int wm = wave & 1, wn = wave >> 1;
    auto put = [&](int8_t* st, int h, v4i a, v4i b) {
        const int at = row * GK + (((pc + 4 * h) ^ gswz(row)) << 4);
        *(v4i*)(st + at) = a;
        *(v4i*)(st + GT * GK + at) = b;
    };
    auto products = [&](const int8_t* st) {
        v4i fa[4], fb[4];
#pragma unroll
        for (int ks = 0; ks < 4; ks++) {
            const int kp = (lane >> 5) + 2 * ks, r = lane & 31;
            fa[ks] = *(const v4i*)(st + (wm * 32 + r) * GK + ((kp ^ gswz(r)) << 4));
            fb[ks] = *(const v4i*)(st + GT * GK + (wn * 32 + r) * GK + ((kp ^ gswz(r)) << 4));
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int ks = 0; ks < 4; ks++) acc[0][0] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fb[ks], fa[ks], acc[0][0], 0, 0, 0);
    };
    if (K >= 16) {
        v4i pa[GA][2], pb[GA][2];
        auto load = [&](int kt, int s) {
#pragma unroll
            for (int h = 0; h < 2; h++) {
                const int k = min(kt * GK + h * 64 + pc * 16, K - 16);
                pa[s][h] = __builtin_bit_cast(v4i, load16_any(ra + k));
                pb[s][h] = __builtin_bit_cast(v4i, load16_any(rb + k));
            }
        };
#pragma unroll
        for (int s = 0; s < GA; s++) load(s, s);
        load_params<GT, GT, 256, G>(A, par, m0, n0);
        // a step's barrier is its only one: a wave writes this stage again two steps on, after the barrier in between
        int k0 = 0, stage = 0;
        for (; k0 + GA < nk; k0 += GA) {
#pragma unroll
            for (int s = 0; s < GA; s++) {
                int8_t* st = lds[0] + stage;
#pragma unroll
                for (int h = 0; h < 2; h++) put(st, h, pa[s][h], pb[s][h]);
                __syncthreads();
                load(k0 + s + GA, s);
                products(st);
                stage ^= 2 * GT * GK;
            }
        }
#pragma unroll
        for (int s = 0; s < GA; s++) {   // what is left, the last step among it
            if (k0 + s >= nk) break;
            int8_t* st = lds[0] + stage;
#pragma unroll
            for (int h = 0; h < 2; h++) {
                const int k = (k0 + s) * GK + h * 64 + pc * 16;
                put(st, h, cut_piece(pa[s][h], k, K), cut_piece(pb[s][h], k, K));
            }
            __syncthreads();
            products(st);
            stage ^= 2 * GT * GK;
        }
    } else {
        load_params<GT, GT, 256, G>(A, par, m0, n0);
        if (K > 0) {
#pragma unroll
            for (int h = 0; h < 2; h++) put(lds[0], h, row_piece(ra, h * 64 + pc * 16, K), row_piece(rb, h * 64 + pc * 16, K));
            __syncthreads();
            products(lds[0]);
        }
    }
    __syncthreads();
    if constexpr (G) {
        // gates and partners are in different waves here: the sums go through LDS, then eight columns of a row a thread
        constexpr int PITCH = GT + 4;
        static_assert(sizeof(lds) >= GT * PITCH * 4, "room for the sums");
        int32_t* sums = (int32_t*)lds[0];
#pragma unroll
        for (int j = 0; j < 4; j++)
            *(v4i*)(sums + (wm * 32 + (lane & 31)) * PITCH + wn * 32 + 8 * j + 4 * (lane >> 5)) =
                v4i{acc[0][0][4 * j], acc[0][0][4 * j + 1], acc[0][0][4 * j + 2], acc[0][0][4 * j + 3]};
        __syncthreads();
        const int r = threadIdx.x >> 2, c = (threadIdx.x & 3) * 8;
        const int64_t m = m0 + r, n = n0 + c;
        if (m >= A.M || n >= A.N) return;
        const int left = (int)min((int64_t)8, A.N - n);
        const float sa = par[2 * GT + r];
        float gate[8], up[8];
#pragma unroll
        for (int e = 0; e < 8; e++) {
            gate[e] = (float)sums[r * PITCH + c + e] * par[c + e] * sa + par[GT + c + e];
            up[e] = (float)sums[r * PITCH + 32 + c + e] * par[32 + c + e] * sa + par[GT + 32 + c + e];
        }
        if (A.z) {
            store_first((T*)A.z + m * A.ldz + n, left, gate);
            store_first((T*)A.z + m * A.ldz + A.N + n, left, up);
        }
        act_values(A.act, gate);
#pragma unroll
        for (int e = 0; e < 8; e++) gate[e] *= up[e];
        store_first((T*)A.out + m * A.ldout + n, left, gate);
    } else {
        epilogue<T, GT, GT, 2, 2, sizeof(lds)>(A, acc, lds[0], par, m0, n0);
    }
}

// Timing record of a launch (NITI_TIMING_KERNEL, or the sum of parts), closed by timing_end.
template <typename T>
const char* type_name() { return __is_same(T, int32_t) ? "i32" : (__is_same(T, float) ? "f32" : (__is_same(T, bf16) ? "bf16" : "f16")); }
template <typename... V>
int time_launch(int family, hipStream_t stream, const char* fmt, V... v) {
    return timing_on() ? timing_begin(family, stream, kernel_label(fmt, v...)) : -1;
}

template <typename T, bool G = false>
hipError_t run_any(const LinArgs& A, hipStream_t stream) {
    const int64_t tm = (A.M + GT - 1) / GT, tn = G ? (A.N + GT / 2 - 1) / (GT / 2) : (A.N + GT - 1) / GT;
    const dim3 grid((unsigned)(tm * tn), A.klen ? (unsigned)((A.K + A.klen - 1) / A.klen) : 1);
    const int tk = time_launch(NITI_TIMING_KERNEL, stream, G ? "linear_any_kernel<%s,pairs>" : "linear_any_kernel<%s>", type_name<T>());
    hipLaunchKernelGGL((linear_any_kernel<T, G>), grid, dim3(256), 0, stream, A, (int)tn);
    timing_end(tk, stream);
    return hipGetLastError();
}

// ---------------------------------------------------------------- few products
// Tiles of 16 FM rows x 16 FN channels; the workgroup's eight waves split the
// sum, so that a tile's operands are in flight all at once, straight from
// memory into MFMA registers, and join through LDS.  A step of a wave is 128
// bytes of each row (two 16 x 16 x 64 MFMAs): whole cache lines.  Any strides and
// addresses.  One token by 4096 x 4096 is 256 such tiles: every CU streams 64 KB
// of weights.
// 16 bytes as they are loaded.  BYTES: from an address that is no multiple of 4.
// The hardware takes such loads apart where the lanes beside one read other rows
// (one token by 4096 x 4097 took 10.9 us, with aligned words 7.1, by 4096 x 4100 5.8; the kernel above,
// whose lanes read a row four by four, loses by the shifts), so the aligned words that hold the bytes are loaded, five
// where the address is not aligned, and shifted when they are used.  Every word
// read holds a byte of the piece.
template <bool BYTES>
struct Raw16 {
    v4i v;
    uint32_t next;
    uint32_t shift;
    __device__ __forceinline__ void load(const int8_t* p) {
        if (BYTES) {
            shift = (uint32_t)(uintptr_t)p & 3u;
            const int8_t* q = p - shift;
            __builtin_memcpy(&v, __builtin_assume_aligned(q, 4), 16);
            __builtin_memcpy(&next, __builtin_assume_aligned(q + (shift ? 16 : 12), 4), 4);
        } else {
            __builtin_memcpy(&v, __builtin_assume_aligned(p, 4), 16);
        }
    }
    __device__ __forceinline__ v4i get() const {
        if (!BYTES) return v;
        return v4i{(int)__builtin_amdgcn_alignbyte((uint32_t)v[1], (uint32_t)v[0], shift),
                   (int)__builtin_amdgcn_alignbyte((uint32_t)v[2], (uint32_t)v[1], shift),
                   (int)__builtin_amdgcn_alignbyte((uint32_t)v[3], (uint32_t)v[2], shift),
                   (int)__builtin_amdgcn_alignbyte(next, (uint32_t)v[3], shift)};
    }
};
// Whether rows begin at multiples of 4.
inline bool word_rows(const LinArgs& A) { return A.lda % 4 == 0 && A.ldb % 4 == 0 && (((uintptr_t)A.a | (uintptr_t)A.b) & 3) == 0 && A.K % 4 == 0; }

constexpr int SW = 8;

template <typename T, int FM, int FN, bool BYTES, bool G = false>
__device__ __forceinline__ void small_tile(const LinArgs& A, int tiles_n, int block) {
    static_assert(!G || FN % 2 == 0, "gates and partners");
    constexpr int TM = 16 * FM, TN = 16 * FN, PITCH = TN + 4, CN = G ? FN / 2 : FN;   // CN: column tiles of the result
    constexpr int KB = FM + FN <= 2 ? 4 : (FM + FN <= 3 ? 2 : 1);   // steps in flight of a wave
    __shared__ __attribute__((aligned(16))) int32_t red[SW * TM * PITCH];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t m0 = (int64_t)(block / tiles_n) * TM, n0 = (int64_t)(block % tiles_n) * (16 * CN);
    // the epilogue's operands of the threads that end a row's four channels, ahead of the sum
    const int row = threadIdx.x / (4 * CN), col = threadIdx.x % (4 * CN) * 4;
    const int64_t m = m0 + row, n = n0 + col;
    const int left = row < TM && m < A.M && n < A.N ? (int)min((int64_t)4, A.N - n) : 0;
    // (in a branch, and so waited for, but by the waves of those threads alone)
    float sa = 0.f, sb[4], bias[4] = {0.f, 0.f, 0.f, 0.f}, res[4] = {0.f, 0.f, 0.f, 0.f};
    float sb2[4], bias2[4] = {0.f, 0.f, 0.f, 0.f};   // of the partners
    if (left > 0) {
        if constexpr (G) {
#pragma unroll
            for (int e = 0; e < 4; e++) sb2[e] = A.s_b[A.b_step ? A.N + n + min(e, left - 1) : 0];
            if (A.bias) load_typed(A.bias, A.bias_type, A.N + n, left, bias2);
        }
        sa = A.s_a ? A.s_a[A.a_step ? m : 0] : 1.f;
#pragma unroll
        for (int e = 0; e < 4; e++) sb[e] = A.s_b ? A.s_b[A.b_step ? n + min(e, left - 1) : 0] : 1.f;
        if (A.bias) load_typed(A.bias, A.bias_type, n, left, bias);
        if (!G && A.res) load_some((const T*)A.res + m * A.ldres + n, left, res);
    }
    // rows past the edge read row 0: what they give is not stored
    const int r16 = lane & 15, kq = (lane >> 4) * 16;
    const int8_t *ra[FM], *rb[FN];
#pragma unroll
    for (int i = 0; i < FM; i++) ra[i] = A.a + (m0 + 16 * i + r16 < A.M ? (m0 + 16 * i + r16) * A.lda : 0);
#pragma unroll
    for (int i = 0; i < FN; i++) {
        const int64_t nb = n0 + 16 * (G ? i / 2 : i) + r16;
        rb[i] = A.b + (nb < A.N ? nb + (G ? (i & 1) * A.N : 0) : 0) * A.ldb;
    }
    const int K = (int)A.K;
    v4i acc[FN][FM];
#pragma unroll
    for (int a = 0; a < FN; a++)
#pragma unroll
        for (int b = 0; b < FM; b++) acc[a][b] = v4i{0, 0, 0, 0};
    auto mma = [&](v4i (&w)[FN], v4i (&x)[FM]) {
#pragma unroll
        for (int a = 0; a < FN; a++)
#pragma unroll
            for (int b = 0; b < FM; b++) acc[a][b] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[a], x[b], acc[a][b], 0, 0, 0);
    };
    // NS steps of this wave from step s on, their loads all in flight and none of them in a branch: past a
    // row's last whole piece they read that one, and the sum's last step sets right what they gave.
    const int last = (K - 1) >> 7;
    auto steps = [&](int s, auto count) {
        constexpr int NS = decltype(count)::value;
        Raw16<BYTES> rw[2 * NS][FN], rx[2 * NS][FM];
#pragma unroll
        for (int j = 0; j < 2 * NS; j++) {
            const int k = min((s + (j >> 1) * SW) * 128 + (j & 1) * 64 + kq, K - 16);
#pragma unroll
            for (int i = 0; i < FN; i++) rw[j][i].load(rb[i] + k);
#pragma unroll
            for (int i = 0; i < FM; i++) rx[j][i].load(ra[i] + k);
        }
#pragma unroll
        for (int j = 0; j < 2 * NS; j++) {
            const int at = s + (j >> 1) * SW, k = at * 128 + (j & 1) * 64 + kq;
            v4i w[FN], x[FM];
#pragma unroll
            for (int i = 0; i < FN; i++) w[i] = rw[j][i].get();
#pragma unroll
            for (int i = 0; i < FM; i++) x[i] = rx[j][i].get();
            if (at == last) {
#pragma unroll
                for (int i = 0; i < FN; i++) w[i] = cut_piece(w[i], k, K);
#pragma unroll
                for (int i = 0; i < FM; i++) x[i] = cut_piece(x[i], k, K);
            }
            mma(w, x);
        }
    };
    if (K >= 16) {
        int s = wave;
        for (; s + (KB - 1) * SW <= last; s += KB * SW) steps(s, std::integral_constant<int, KB>());
        if (KB > 2 && s + SW <= last) {
            steps(s, std::integral_constant<int, 2>());
            s += 2 * SW;
        }
        if (KB > 1 && s <= last) steps(s, std::integral_constant<int, 1>());
    } else if (wave == 0 && K > 0) {
        v4i w[FN], x[FM];
#pragma unroll
        for (int i = 0; i < FN; i++) w[i] = row_piece(rb[i], kq, K);
#pragma unroll
        for (int i = 0; i < FM; i++) x[i] = row_piece(ra[i], kq, K);
        mma(w, x);
    }
    // element i of acc[a][b]: channel 16 a + 4 (lane / 16) + i of row 16 b + lane % 16
#pragma unroll
    for (int a = 0; a < FN; a++)
#pragma unroll
        for (int b = 0; b < FM; b++)
            *(v4i*)(red + (wave * TM + 16 * b + r16) * PITCH + 16 * a + 4 * (lane >> 4)) = acc[a][b];
    __syncthreads();
    if (left <= 0) return;
    const int at = G ? col / 16 * 32 + col % 16 : col;
    v4i sum = *(const v4i*)(red + row * PITCH + at);
#pragma unroll
    for (int i = 1; i < SW; i++) sum += *(const v4i*)(red + (i * TM + row) * PITCH + at);
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; e++) v[e] = (float)sum[e] * sb[e] * sa + bias[e];
    if constexpr (G) {
        v4i two = *(const v4i*)(red + row * PITCH + at + 16);
#pragma unroll
        for (int i = 1; i < SW; i++) two += *(const v4i*)(red + (i * TM + row) * PITCH + at + 16);
        float up[4];
#pragma unroll
        for (int e = 0; e < 4; e++) up[e] = (float)two[e] * sb2[e] * sa + bias2[e];
        if (A.z) {
            store_some((T*)A.z + m * A.ldz + n, left, v);
            store_some((T*)A.z + m * A.ldz + A.N + n, left, up);
        }
        act_values(A.act, v);
#pragma unroll
        for (int e = 0; e < 4; e++) v[e] *= up[e];
        store_some((T*)A.out + m * A.ldout + n, left, v);
        return;
    }
    if (A.z) store_some((T*)A.z + m * A.ldz + n, left, v);
    act_values(A.act, v);
#pragma unroll
    for (int e = 0; e < 4; e++) v[e] += res[e];
    store_some((T*)A.out + m * A.ldout + n, left, v);
}

template <typename T, int FM, int FN, bool BYTES, bool G = false>
__global__ __launch_bounds__(64 * SW) void linear_small_kernel(LinArgs A, int tiles_n) {
    small_tile<T, FM, FN, BYTES, G>(A, tiles_n, blockIdx.x);
}

// Two products in one launch (word-aligned rows).
struct LinPair {
    LinArgs a[2];
    int tiles_n[2];
    int blocks;   // tiles of the first
};

template <typename T, int FM, int FN>
__global__ __launch_bounds__(64 * SW) void linear_small_pair_kernel(LinPair P) {
    const int i = (int)blockIdx.x < P.blocks ? 0 : 1;
    small_tile<T, FM, FN, false>(P.a[i], P.tiles_n[i], (int)blockIdx.x - i * P.blocks);
}

template <typename T, int FM, int FN, bool G = false>
hipError_t run_small(const LinArgs& A, hipStream_t stream) {
    constexpr int CN = G ? FN / 2 : FN;
    const int64_t tm = (A.M + 16 * FM - 1) / (16 * FM), tn = (A.N + 16 * CN - 1) / (16 * CN);
    const bool words = word_rows(A);
    const int tk = time_launch(NITI_TIMING_KERNEL, stream, G ? "linear_small_kernel<%s,%d,%d,%d,pairs>" : "linear_small_kernel<%s,%d,%d,%d>", type_name<T>(), FM, FN, !words);
    if (words)
        hipLaunchKernelGGL((linear_small_kernel<T, FM, FN, false, G>), dim3((unsigned)(tm * tn)), dim3(64 * SW), 0, stream, A, (int)tn);
    else
        hipLaunchKernelGGL((linear_small_kernel<T, FM, FN, true, G>), dim3((unsigned)(tm * tn)), dim3(64 * SW), 0, stream, A, (int)tn);
    timing_end(tk, stream);
    return hipGetLastError();
}

// ---------------------------------------------------------------- ring
// Tiles of BM x BN from an LDS ring of NS stages of KS bytes a row, filled by
// direct-to-LDS loads.  Needs K, strides and addresses in whole 16 bytes.
// 256 x 256 tiles read the least from L2 and LDS for a product (4096 x 4096 x 2048 44 us, by
// 128 x 128 50), smaller ones give more CUs work (2048 x 4096 x 4096 by 128 x 128 44, by 256 x 256 58).
constexpr uint32_t kOut = 0x80000000u;   // an offset past any tile: loads zeros

template <int N>
__device__ __forceinline__ void wait_loads() {   // vmcnt <= N and this wave's LDS reads done
    static_assert(N < 64, "vmcnt");
    __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | 0x0070);
}

template <int BM, int BN, int NS, int WGM, int WGN, int KS>
struct Ring {
    static constexpr int NW = WGM * WGN, NT = 64 * NW;
    static constexpr int RPB = 1024 / KS;          // rows of a 1 KiB block (one load instruction)
    static constexpr int LPR = KS / 16;            // lanes of a row
    static constexpr int ND = KS / 32;             // MFMA depths of a step
    static constexpr int WTM = BM / WGM, WTN = BN / WGN;
    static constexpr int FM = WTM / 32, FN = WTN / 32;
    static constexpr int LA = BM / RPB / NW, LB = BN / RPB / NW;   // loads of a wave and stage
    static_assert(LA * RPB * NW == BM && LB * RPB * NW == BN, "loads split over the waves");
    static_assert(NW % 2 == 0, "one swizzle parity per wave");
    static constexpr int STAGE = (BM + BN) * KS;
    static constexpr int LDS = NS * STAGE + (2 * BN + BM) * 4;   // the ring, and the tile's scales and biases
    // 16-byte piece c of row r is stored at piece c ^ swz(r): the 32 rows that a
    // fragment read takes one piece of then hit distinct banks
    static __device__ __forceinline__ int swz(int row) { return KS == 64 ? ((row >> 1) ^ (row >> 2)) & 3 : (row >> 1) & 7; }
};

template <typename T, int BM, int BN, int NS, int WGM, int WGN, int KS, bool G = false>
__device__ __forceinline__ void ring_tile(const LinArgs& A, int tiles_n, int block) {
    using R = Ring<BM, BN, NS, WGM, WGN, KS>;
    static_assert(!G || R::WTN % 64 == 0, "a wave has gates and their partners");
    extern __shared__ __attribute__((aligned(1024))) int8_t ring[];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave % WGM, wn = wave / WGM;
    const int64_t m0 = (int64_t)(block / tiles_n) * BM, n0 = (int64_t)(block % tiles_n) * (G ? BN / 2 : BN);
    const int rows_a = (int)min((int64_t)BM, A.M - m0), rows_b = (int)min((int64_t)(G ? BN / 2 : BN), A.N - n0);
    const int K = (int)A.K, nk = (K + KS - 1) / KS;
    // Offsets from the tile's first row; rows past the operand lie past the descriptor's end and load zeros.
    const uint32_t lda = (uint32_t)A.lda, ldb = (uint32_t)A.ldb;
    const u32x4 rs_a = raw_rsrc(A.a + m0 * A.lda, (uint32_t)(rows_a - 1) * lda + (uint32_t)K);
    // Pairs: a load instruction's rows are all gates or all partners, which have a descriptor each (even and odd loads of a wave).
    u32x4 rs_b[2];
#pragma unroll
    for (int i = 0; i < 2; i++) {
        const int half = G ? pair_half<5>((wave + i * R::NW) * R::RPB) : 0;
        rs_b[i] = raw_rsrc(A.b + (n0 + half * A.N) * A.ldb, (uint32_t)(rows_b - 1) * ldb + (uint32_t)K);
    }
    static_assert(!G || (32 % R::RPB == 0 && 2 * R::NW * R::RPB % 64 == 0), "loads two apart are of the same half");
    const int lrow = lane / R::LPR;
    const uint32_t kpo = (uint32_t)(((lane % R::LPR) ^ R::swz((wave & 1) * R::RPB + lrow)) << 4);
    const uint32_t lds0 = lds_address(ring);
    uint32_t oa[R::LA], ob[R::LB], da[R::LA], db[R::LB];
#pragma unroll
    for (int i = 0; i < R::LA; i++) {
        const int blk = wave + i * R::NW;
        oa[i] = (uint32_t)(blk * R::RPB + lrow) * lda + kpo;
        da[i] = __builtin_amdgcn_readfirstlane(lds0 + (uint32_t)blk * 1024u);
    }
#pragma unroll
    for (int i = 0; i < R::LB; i++) {
        const int blk = wave + i * R::NW;
        ob[i] = (uint32_t)(G ? pair_row<5>(blk * R::RPB + lrow) : blk * R::RPB + lrow) * ldb + kpo;
        db[i] = __builtin_amdgcn_readfirstlane(lds0 + (uint32_t)(BM * KS) + (uint32_t)blk * 1024u);
    }
    const uint32_t kend = (uint32_t)(K - (nk - 1) * KS);   // bytes of the last step
    int left = nk - 1;                                     // whole steps to load
    uint32_t koff = 0, slot = 0;
    // Loads of the next step.  Past the last one they go on as zeros: the wait counts stay constant.
    auto begin_step = [&]() {
        if (left <= 0) {
            const bool out = left < 0 || kpo >= kend;
#pragma unroll
            for (int i = 0; i < R::LA; i++) oa[i] = out ? kOut : oa[i];
#pragma unroll
            for (int i = 0; i < R::LB; i++) ob[i] = out ? kOut : ob[i];
        }
        left = __builtin_amdgcn_readfirstlane(left - 1);
    };
    auto end_step = [&]() {
        koff += KS;
        slot = slot + R::STAGE == (uint32_t)(NS * R::STAGE) ? 0u : slot + R::STAGE;
    };
    // load i of the step, of LA + LB
    auto load = [&](int i) {
        if (i < R::LA)
            lds_dma16_at(rs_a, da[i], slot, oa[i], koff);
        else
            lds_dma16_at(rs_b[G ? (i - R::LA) & 1 : 0], db[i - R::LA], slot, ob[i - R::LA], koff);
    };

    v16i acc[R::FN][R::FM];
#pragma unroll
    for (int a = 0; a < R::FN; a++)
#pragma unroll
        for (int b = 0; b < R::FM; b++) acc[a][b] = v16i{};
    int a_at[R::FM], b_at[R::FN], a_sw[R::FM], b_sw[R::FN];
#pragma unroll
    for (int i = 0; i < R::FM; i++) {
        const int row = wm * R::WTM + i * 32 + (lane & 31);
        a_at[i] = row * KS;
        a_sw[i] = R::swz(row & 15);
    }
#pragma unroll
    for (int i = 0; i < R::FN; i++) {
        const int row = wn * R::WTN + i * 32 + (lane & 31);
        b_at[i] = BM * KS + row * KS;
        b_sw[i] = R::swz(row & 15);
    }
    float* par = (float*)(ring + NS * R::STAGE);
#pragma unroll
    for (int s = 0; s < NS - 1; s++) {
        begin_step();
#pragma unroll
        for (int i = 0; i < R::LA + R::LB; i++) load(i);
        end_step();
    }
    load_params<BM, BN, R::NT, G>(A, par, m0, n0);   // behind the ring's first loads, whose latency it shares
    v4i fa[2][R::FM], fb[2][R::FN];
    auto read = [&](const int8_t* st, int d, int i) {   // fragment i of FN + FM of a depth
        const int kp = (lane >> 5) + 2 * d;
        if (i < R::FN)
            fb[d & 1][i] = *(const v4i*)(st + b_at[i] + ((kp ^ b_sw[i]) << 4));
        else
            fa[d & 1][i - R::FN] = *(const v4i*)(st + a_at[i - R::FN] + ((kp ^ a_sw[i - R::FN]) << 4));
    };
    // The MFMAs of depth d, with the reads of a next depth and loads from..to-1 spread between them: a wave
    // that issues its loads and reads at once keeps its matrix core waiting meanwhile.
    constexpr int NM = R::FN * R::FM, NR = R::FN + R::FM;
    auto depth = [&](int d, const int8_t* rd_st, int rd, int from, int to) {
#pragma unroll
        for (int i = 0; i < NM; i++) {
            const int a = i / R::FM, b = i % R::FM;
            acc[a][b] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fb[d & 1][a], fa[d & 1][b], acc[a][b], 0, 0, 0);
#pragma unroll
            for (int r = i * NR / NM; r < (i + 1) * NR / NM; r++) read(rd_st, rd, r);
#pragma unroll
            for (int l = from + i * (to - from) / NM; l < from + (i + 1) * (to - from) / NM; l++) load(l);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // Fragments are double buffered over the depths: one depth's are read while the previous one's MFMAs run,
    // the next stage's first right after the barrier.  Before a barrier a wave waits for its own fragment reads,
    // so no read of the stage that the next loads overwrite is in flight behind it.
    constexpr int NL = R::LA + R::LB;
    constexpr int LD = NS > 2 || R::ND < 4 ? R::ND - 1 : R::ND - 2;   // depths that loads are issued in
    wait_loads<(NS - 2) * NL>();
    __builtin_amdgcn_s_barrier();
#pragma unroll
    for (int i = 0; i < NR; i++) read(ring, 0, i);
    int cur = 0;
    for (int kt = 0; kt < nk; kt++) {
        const int8_t* st = ring + cur;
        begin_step();
#pragma unroll
        for (int d = 0; d + 1 < R::ND; d++)
            depth(d, st, d + 1, d < LD ? d * NL / LD : NL, d < LD ? (d + 1) * NL / LD : NL);
        end_step();
        wait_loads<(NS - 2) * NL>();
        __builtin_amdgcn_s_barrier();
        cur = cur + R::STAGE == NS * R::STAGE ? 0 : cur + R::STAGE;
        depth(R::ND - 1, ring + cur, 0, NL, NL);   // (after the last step it reads zeros that no MFMA uses)
    }
    wait_loads<0>();   // the loads past the end, before the ring is reused
    __builtin_amdgcn_s_barrier();
    if constexpr (G)
        gated_epilogue<T, BM, BN, WGM, WGN, NS * R::STAGE>(A, acc, ring, par, m0, n0);
    else
        epilogue<T, BM, BN, WGM, WGN, NS * R::STAGE>(A, acc, ring, par, m0, n0);
}

template <typename T, int BM, int BN, int NS, int WGM, int WGN, int KS, bool G = false>
__global__ __launch_bounds__(64 * WGM * WGN, BM * BN / (WGM * WGN) <= 8192 ? 2 : 1) void linear_ring_kernel(LinArgs A, int tiles_n) {
    take_part<T>(A);
    ring_tile<T, BM, BN, NS, WGM, WGN, KS, G>(A, tiles_n, blockIdx.x);
}

// Two products in one launch.
template <typename T, int BM, int BN, int NS, int WGM, int WGN, int KS>
__global__ __launch_bounds__(64 * WGM * WGN, BM * BN / (WGM * WGN) <= 8192 ? 2 : 1) void linear_ring_pair_kernel(LinPair P) {
    const int i = (int)blockIdx.x < P.blocks ? 0 : 1;
    ring_tile<T, BM, BN, NS, WGM, WGN, KS>(P.a[i], P.tiles_n[i], (int)blockIdx.x - i * P.blocks);
}

template <typename T, int BM, int BN, int NS, int WGM, int WGN, int KS, bool G = false>
hipError_t run_ring(const LinArgs& A, hipStream_t stream) {
    using R = Ring<BM, BN, NS, WGM, WGN, KS>;
    constexpr auto kernel = linear_ring_kernel<T, BM, BN, NS, WGM, WGN, KS, G>;
    constexpr int CN = G ? BN / 2 : BN;
    const hipError_t e = allow_lds<kernel, R::LDS>();
    if (e != hipSuccess) return e;
    const int64_t tm = (A.M + BM - 1) / BM, tn = (A.N + CN - 1) / CN;
    const int tk = time_launch(NITI_TIMING_KERNEL, stream,
                               G ? "linear_ring_kernel<%s,%d,%d,%d,%d,%d,%d,pairs>" : "linear_ring_kernel<%s,%d,%d,%d,%d,%d,%d>", type_name<T>(), BM, BN, NS, WGM, WGN, KS);
    hipLaunchKernelGGL(kernel, dim3((unsigned)(tm * tn), A.klen ? (unsigned)((A.K + A.klen - 1) / A.klen) : 1), dim3(R::NT), R::LDS,
                       stream, A, (int)tn);
    timing_end(tk, stream);
    return hipGetLastError();
}

bool ring_takes(const LinArgs& A) {
    return A.K > 0 && A.K % 16 == 0 && A.lda % 16 == 0 && A.ldb % 16 == 0 && (((uintptr_t)A.a | (uintptr_t)A.b) & 15) == 0;
}

// ---------------------------------------------------------------- what the choice of a kernel goes by
// The kernels, and what a product takes in each (us), with t = tiles / 256 CUs and
// k = K / 1000:
//   kSpread  start + round * max(1, t) + k * (step + more * max(0, t - 1))
//   kTwo     start + round * max(1, t) + k * (step * ceil(t / 2) + more * max(1, t))   (two tiles or more a CU at a time)
//   kRounds  start + ceil(t) * (round + k * step) + k * more * min(1, t)               (one tile a CU at a time)
enum CostForm { kSpread, kTwo, kRounds };
struct Cost {
    int bm, bn;
    CostForm form;
    float start, round, step, more;
};
float cost(const Cost& c, int64_t M, int64_t N, int64_t K, int parts = 1) {
    const float t = (float)((M + c.bm - 1) / c.bm) * (float)((N + c.bn - 1) / c.bn) * (float)parts / 256.f;
    const float k = (float)K / 1000.f / (float)parts, one = fmaxf(1.f, t);
    if (c.form == kRounds) return c.start + ceilf(t) * (c.round + c.step * k) + fminf(t, 1.f) * c.more * k;
    if (c.form == kTwo) return c.start + c.round * one + k * (c.step * ceilf(0.5f * t) + c.more * one);
    return c.start + c.round * one + k * (c.step + c.more * (one - 1.f));
}

// What the operands' rows are made of, aligned.
enum Rows { kOfBytes, kOfWords, kOfPieces };

inline int64_t up16(int64_t v) { return (v + 15) / 16 * 16; }
// Copies of both operands, where K leaves their rows no whole pieces (whole rows at odd
// strides go without: the workspace is sized before strides are known); less than 2^32 pieces.
constexpr int64_t kPackBytes = (int64_t)1 << 34;
inline size_t pack_bytes(int64_t M, int64_t N, int64_t K) {
    const int64_t Kp = up16(K);
    return K < 16 || K % 16 == 0 || M > kPackBytes / Kp || N > kPackBytes / Kp ? 0 : (size_t)((M + N) * Kp + 255) / 256 * 256;
}

// Both operands' rows, at any addresses, to rows of Kp = ppr * 16 bytes, a's and then b's; zeros past K.
__global__ __launch_bounds__(256) void linear_pack_kernel(LinArgs A, uint32_t ppr, uint32_t pieces, int8_t* out) {
    const uint32_t i = blockIdx.x * 256 + threadIdx.x;
    if (i >= pieces) return;
    const int64_t r = i / ppr;
    const int k = (int)(i % ppr) * 16, K = (int)A.K;
    const int8_t* row = r < A.M ? A.a + r * A.lda : A.b + (r - A.M) * A.ldb;
    *(v4i*)(out + (int64_t)i * 16) = cut_piece(__builtin_bit_cast(v4i, load16_any(row + min(k, K - 16))), k, K);
}

}  // namespace

}  // namespace niti
