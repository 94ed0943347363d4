// Product of int8 rows with its epilogue:
//
//   z[m][n] = s_a[m] s_b[n] sum_k a[m][k] b[n][k] + bias[n],  out = act(z) + res
//
// The sum is exact in int32 (int8 MFMA); everything after it is in 32-bit
// floats, rounded once at the store.  The epilogue runs in the kernel that
// forms the sum: z, the activation and the residual cost no pass of their own.
//
// Four kinds of kernel.  Whole aligned pieces: LDS rings of 64 x 64, 128 x 128 or
// 256 x 256 tiles.  Any addresses: 64 x 64 tiles through registers, or rows copied to
// whole pieces first.  Few products: small tiles straight from memory.  Long
// sums of few products: parts side by side in the workspace.
//
// Measured: 8192 x 8192 x 8192 to bf16 484 to 491 us, 2.24 to 2.27 POPS, bound by power (the
// clock falls to 1.55 to 1.73 GHz with the MFMAs busy 65 to 60% of it); one token by 4096 x 4096
// 6.1 us, 2.8 TB/s of weights; 1000 x 1500 x 1111 in 32 bits with every operand 15.
#include "linear.h"

#include <math.h>

#include <atomic>
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

// Scales and biases of a tile's columns and scales of its rows, to LDS before
// the sum begins: loaded in the epilogue they cost it two memory round trips.
template <int BM, int BN, int NT>
__device__ __forceinline__ void load_params(const LinArgs& A, float* par, int64_t m0, int64_t n0) {
    static_assert(NT >= BM && NT >= BN, "one column and one row a thread");
    const int t = threadIdx.x;
    const int64_t n = min(n0 + t % BN, A.N - 1), m = min(m0 + t % BM, A.M - 1);
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

template <typename T>
__global__ __launch_bounds__(256) void linear_any_kernel(LinArgs A, int tiles_n) {
    take_part<T>(A);
    __shared__ __attribute__((aligned(16))) int8_t lds[2][2 * GT * GK];
    __shared__ __attribute__((aligned(16))) float par[3 * GT];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t m0 = (int64_t)(blockIdx.x / tiles_n) * GT, n0 = (int64_t)(blockIdx.x % tiles_n) * GT;
    // two pieces of each operand a thread, 64 bytes apart: rows past the edge read row 0, whose products are not stored
    const int row = threadIdx.x >> 2, pc = threadIdx.x & 3;
    const int8_t* ra = A.a + (m0 + row < A.M ? (m0 + row) * A.lda : 0);
    const int8_t* rb = A.b + (n0 + row < A.N ? (n0 + row) * A.ldb : 0);
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
        load_params<GT, GT, 256>(A, par, m0, n0);
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
        load_params<GT, GT, 256>(A, par, m0, n0);
        if (K > 0) {
#pragma unroll
            for (int h = 0; h < 2; h++) put(lds[0], h, row_piece(ra, h * 64 + pc * 16, K), row_piece(rb, h * 64 + pc * 16, K));
            __syncthreads();
            products(lds[0]);
        }
    }
    __syncthreads();
    epilogue<T, GT, GT, 2, 2, sizeof(lds)>(A, acc, lds[0], par, m0, n0);
}

// Timing record of a launch (NITI_TIMING_KERNEL, or the sum of parts), closed by timing_end.
template <typename T>
const char* type_name() { return __is_same(T, int32_t) ? "i32" : (__is_same(T, float) ? "f32" : (__is_same(T, bf16) ? "bf16" : "f16")); }
template <typename... V>
int time_launch(int family, hipStream_t stream, const char* fmt, V... v) {
    return timing_on() ? timing_begin(family, stream, kernel_label(fmt, v...)) : -1;
}

template <typename T>
hipError_t run_any(const LinArgs& A, hipStream_t stream) {
    const int64_t tm = (A.M + GT - 1) / GT, tn = (A.N + GT - 1) / GT;
    const dim3 grid((unsigned)(tm * tn), A.klen ? (unsigned)((A.K + A.klen - 1) / A.klen) : 1);
    const int tk = time_launch(NITI_TIMING_KERNEL, stream, "linear_any_kernel<%s>", type_name<T>());
    hipLaunchKernelGGL((linear_any_kernel<T>), grid, dim3(256), 0, stream, A, (int)tn);
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

template <typename T, int FM, int FN, bool BYTES>
__device__ __forceinline__ void small_tile(const LinArgs& A, int tiles_n, int block) {
    constexpr int TM = 16 * FM, TN = 16 * FN, PITCH = TN + 4;
    constexpr int KB = FM + FN <= 2 ? 4 : (FM + FN <= 3 ? 2 : 1);   // steps in flight of a wave
    __shared__ __attribute__((aligned(16))) int32_t red[SW * TM * PITCH];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t m0 = (int64_t)(block / tiles_n) * TM, n0 = (int64_t)(block % tiles_n) * TN;
    // the epilogue's operands of the threads that end a row's four channels, ahead of the sum
    const int row = threadIdx.x / (4 * FN), col = threadIdx.x % (4 * FN) * 4;
    const int64_t m = m0 + row, n = n0 + col;
    const int left = row < TM && m < A.M && n < A.N ? (int)min((int64_t)4, A.N - n) : 0;
    // (in a branch, and so waited for, but by the waves of those threads alone)
    float sa = 0.f, sb[4], bias[4] = {0.f, 0.f, 0.f, 0.f}, res[4] = {0.f, 0.f, 0.f, 0.f};
    if (left > 0) {
        sa = A.s_a ? A.s_a[A.a_step ? m : 0] : 1.f;
#pragma unroll
        for (int e = 0; e < 4; e++) sb[e] = A.s_b ? A.s_b[A.b_step ? n + min(e, left - 1) : 0] : 1.f;
        if (A.bias) load_typed(A.bias, A.bias_type, n, left, bias);
        if (A.res) load_some((const T*)A.res + m * A.ldres + n, left, res);
    }
    // rows past the edge read row 0: what they give is not stored
    const int r16 = lane & 15, kq = (lane >> 4) * 16;
    const int8_t *ra[FM], *rb[FN];
#pragma unroll
    for (int i = 0; i < FM; i++) ra[i] = A.a + (m0 + 16 * i + r16 < A.M ? (m0 + 16 * i + r16) * A.lda : 0);
#pragma unroll
    for (int i = 0; i < FN; i++) rb[i] = A.b + (n0 + 16 * i + r16 < A.N ? (n0 + 16 * i + r16) * A.ldb : 0);
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
    v4i sum = *(const v4i*)(red + row * PITCH + col);
#pragma unroll
    for (int i = 1; i < SW; i++) sum += *(const v4i*)(red + (i * TM + row) * PITCH + col);
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; e++) v[e] = (float)sum[e] * sb[e] * sa + bias[e];
    if (A.z) store_some((T*)A.z + m * A.ldz + n, left, v);
    act_values(A.act, v);
#pragma unroll
    for (int e = 0; e < 4; e++) v[e] += res[e];
    store_some((T*)A.out + m * A.ldout + n, left, v);
}

template <typename T, int FM, int FN, bool BYTES>
__global__ __launch_bounds__(64 * SW) void linear_small_kernel(LinArgs A, int tiles_n) {
    small_tile<T, FM, FN, BYTES>(A, tiles_n, blockIdx.x);
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

template <typename T, int FM, int FN>
hipError_t run_small(const LinArgs& A, hipStream_t stream) {
    const int64_t tm = (A.M + 16 * FM - 1) / (16 * FM), tn = (A.N + 16 * FN - 1) / (16 * FN);
    const bool words = word_rows(A);
    const int tk = time_launch(NITI_TIMING_KERNEL, stream, "linear_small_kernel<%s,%d,%d,%d>", type_name<T>(), FM, FN, !words);
    if (words)
        hipLaunchKernelGGL((linear_small_kernel<T, FM, FN, false>), dim3((unsigned)(tm * tn)), dim3(64 * SW), 0, stream, A, (int)tn);
    else
        hipLaunchKernelGGL((linear_small_kernel<T, FM, FN, true>), dim3((unsigned)(tm * tn)), dim3(64 * SW), 0, stream, A, (int)tn);
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

template <typename T, int BM, int BN, int NS, int WGM, int WGN, int KS>
__device__ __forceinline__ void ring_tile(const LinArgs& A, int tiles_n, int block) {
    using R = Ring<BM, BN, NS, WGM, WGN, KS>;
    extern __shared__ __attribute__((aligned(1024))) int8_t ring[];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave % WGM, wn = wave / WGM;
    const int64_t m0 = (int64_t)(block / tiles_n) * BM, n0 = (int64_t)(block % tiles_n) * BN;
    const int rows_a = (int)min((int64_t)BM, A.M - m0), rows_b = (int)min((int64_t)BN, A.N - n0);
    const int K = (int)A.K, nk = (K + KS - 1) / KS;
    // Offsets from the tile's first row; rows past the operand lie past the descriptor's end and load zeros.
    const uint32_t lda = (uint32_t)A.lda, ldb = (uint32_t)A.ldb;
    const u32x4 rs_a = raw_rsrc(A.a + m0 * A.lda, (uint32_t)(rows_a - 1) * lda + (uint32_t)K);
    const u32x4 rs_b = raw_rsrc(A.b + n0 * A.ldb, (uint32_t)(rows_b - 1) * ldb + (uint32_t)K);
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
        ob[i] = (uint32_t)(blk * R::RPB + lrow) * ldb + kpo;
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
            lds_dma16_at(rs_b, db[i - R::LA], slot, ob[i - R::LA], koff);
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
    load_params<BM, BN, R::NT>(A, par, m0, n0);   // behind the ring's first loads, whose latency it shares
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
    epilogue<T, BM, BN, WGM, WGN, NS * R::STAGE>(A, acc, ring, par, m0, n0);
}

template <typename T, int BM, int BN, int NS, int WGM, int WGN, int KS>
__global__ __launch_bounds__(64 * WGM * WGN, BM * BN / (WGM * WGN) <= 8192 ? 2 : 1) void linear_ring_kernel(LinArgs A, int tiles_n) {
    take_part<T>(A);
    ring_tile<T, BM, BN, NS, WGM, WGN, KS>(A, tiles_n, blockIdx.x);
}

// Two products in one launch.
template <typename T, int BM, int BN, int NS, int WGM, int WGN, int KS>
__global__ __launch_bounds__(64 * WGM * WGN, BM * BN / (WGM * WGN) <= 8192 ? 2 : 1) void linear_ring_pair_kernel(LinPair P) {
    const int i = (int)blockIdx.x < P.blocks ? 0 : 1;
    ring_tile<T, BM, BN, NS, WGM, WGN, KS>(P.a[i], P.tiles_n[i], (int)blockIdx.x - i * P.blocks);
}

// Once for each kernel and device, from any thread: it may have more than 64 KiB of LDS.
template <auto kernel, int LDS>
hipError_t allow_lds() {
    static std::atomic<uint64_t> done{0};   // a bit for each of the first 64 devices
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    const uint64_t bit = dev < 64 ? (uint64_t)1 << dev : 0;
    if (done.load(std::memory_order_relaxed) & bit) return hipSuccess;
    e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
    if (e == hipSuccess) done.fetch_or(bit, std::memory_order_relaxed);
    return e;
}

template <typename T, int BM, int BN, int NS, int WGM, int WGN, int KS>
hipError_t run_ring(const LinArgs& A, hipStream_t stream) {
    using R = Ring<BM, BN, NS, WGM, WGN, KS>;
    constexpr auto kernel = linear_ring_kernel<T, BM, BN, NS, WGM, WGN, KS>;
    const hipError_t e = allow_lds<kernel, R::LDS>();
    if (e != hipSuccess) return e;
    const int64_t tm = (A.M + BM - 1) / BM, tn = (A.N + BN - 1) / BN;
    const int tk = time_launch(NITI_TIMING_KERNEL, stream, "linear_ring_kernel<%s,%d,%d,%d,%d,%d,%d>", type_name<T>(), BM, BN, NS, WGM, WGN, KS);
    hipLaunchKernelGGL(kernel, dim3((unsigned)(tm * tn), A.klen ? (unsigned)((A.K + A.klen - 1) / A.klen) : 1), dim3(R::NT), R::LDS,
                       stream, A, (int)tn);
    timing_end(tk, stream);
    return hipGetLastError();
}

bool ring_takes(const LinArgs& A) {
    return A.K > 0 && A.K % 16 == 0 && A.lda % 16 == 0 && A.ldb % 16 == 0 && (((uintptr_t)A.a | (uintptr_t)A.b) & 15) == 0;
}

// ---------------------------------------------------------------- split sums
// Few tiles and a long sum: each part of the sum has workgroups of its own, which
// leave int32 sums in the workspace, and a second launch adds the parts up
// (integers: their order does not matter) and does the epilogue, eight columns
// a thread.
template <typename T>
__global__ __launch_bounds__(256) void linear_join_kernel(LinArgs A, const int32_t* sums, int parts, int64_t ld, int groups_n) {
    const int64_t idx = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t m = idx / groups_n;
    if (m >= A.M) return;
    const int64_t n = idx % groups_n * 8;
    const int left = (int)min((int64_t)8, A.N - n);
    const int32_t* p = sums + m * ld + n;   // (ld is a multiple of 8: a row's last piece is whole)
    v4i lo = {0, 0, 0, 0}, hi = {0, 0, 0, 0};
    for (int i = 0; i < parts; i += 4) {   // four parts in flight; past the last, it again, not added
        v4i x[4], y[4];
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const int32_t* q = p + min(i + j, parts - 1) * A.part;
            x[j] = *(const v4i*)q;
            y[j] = *(const v4i*)(q + 4);
        }
#pragma unroll
        for (int j = 0; j < 4; j++) {
            lo += i + j < parts ? x[j] : v4i{0, 0, 0, 0};
            hi += i + j < parts ? y[j] : v4i{0, 0, 0, 0};
        }
    }
    float sb[8], bias[8] = {}, v[8];
    if (A.s_b && A.b_step)
        load_some(A.s_b + n, left, sb);
    else
#pragma unroll
        for (int e = 0; e < 8; e++) sb[e] = A.s_b ? A.s_b[0] : 1.f;
    if (A.bias) load_typed(A.bias, A.bias_type, n, left, bias);
    const float sa = A.s_a ? A.s_a[A.a_step ? m : 0] : 1.f;
#pragma unroll
    for (int e = 0; e < 8; e++) v[e] = (float)(e < 4 ? lo[e & 3] : hi[e & 3]) * sb[e] * sa + bias[e];
    if (A.z) store_some((T*)A.z + m * A.ldz + n, left, v);
    act_values(A.act, v);
    if (A.res) {
        float r[8];
        load_some((const T*)A.res + m * A.ldres + n, left, r);
#pragma unroll
        for (int e = 0; e < 8; e++) v[e] += r[e];
    }
    store_some((T*)A.out + m * A.ldout + n, left, v);
}

// ---------------------------------------------------------------- choice
// The kernels, and what a product takes in each (us), with t = tiles / 256 CUs and
// k = K / 1000:
//   kSpread  start + round * max(1, t) + k * (step + more * max(0, t - 1))
//   kTwo     start + round * max(1, t) + k * (step * ceil(t / 2) + more * max(1, t))   (two tiles or more a CU at a time)
//   kRounds  start + ceil(t) * (round + k * step) + k * more * min(1, t)               (one tile a CU at a time)
// Small tiles give every CU work and split the sum, large ones load less for each
// product; 128 x 128 tiles have a ring of four stages, one a CU, which a
// CU with one tile needs to cover a load's latency (800 x 2880 x 3712, 161 tiles: 25.9 ->
// 19.4 us), or of two, two tiles a CU (2048 x 4096 x 4096: 44 us, 48 with four).  Fitted to
// 500 random products of 1..8192 x 32..9216 x 32..9216 timed with each kernel;
// what the model picks takes 1.4% longer than the fastest of these seven in the
// mean, on 250 others 1.8%; 64 x 64 tiles alone 33% and 36%.
enum CostForm { kSpread, kTwo, kRounds };
struct Cost {
    int bm, bn;
    CostForm form;
    float start, round, step, more;
};
constexpr Cost kSmall11{16, 16, kSpread, 1.93f, 0.56f, 0.58f, 0.81f};
constexpr Cost kSmall12{16, 32, kSpread, 1.92f, 0.61f, 0.95f, 1.33f};
constexpr Cost kSmall22{32, 32, kSpread, 2.06f, 0.75f, 1.18f, 1.90f};
// Rows at odd addresses, from 200 random products, 2.6% from the fastest in the mean; 5.8% without the copies below.
constexpr Cost kBytes11{16, 16, kSpread, 1.88f, 0.64f, 0.78f, 1.73f};
constexpr Cost kBytes12{16, 32, kSpread, 2.01f, 0.59f, 1.23f, 2.45f};
constexpr Cost kBytes22{32, 32, kSpread, 2.02f, 0.86f, 1.39f, 3.48f};
constexpr Cost kRing64{64, 64, kTwo, 2.09f, 1.02f, 0.32f, 2.21f};
constexpr Cost kAny64{64, 64, kSpread, 2.84f, 1.02f, 3.38f, 4.07f};
constexpr Cost kRing128{128, 128, kTwo, 0.96f, 3.17f, 3.79f, 3.45f};
constexpr Cost kDeep128{128, 128, kRounds, 0.12f, 4.49f, 3.72f, 2.33f};
constexpr Cost kRing256{256, 256, kRounds, 0.41f, 11.1f, 9.31f, 5.98f};

float cost(const Cost& c, int64_t M, int64_t N, int64_t K, int parts = 1) {
    const float t = (float)((M + c.bm - 1) / c.bm) * (float)((N + c.bn - 1) / c.bn) * (float)parts / 256.f;
    const float k = (float)K / 1000.f / (float)parts, one = fmaxf(1.f, t);
    if (c.form == kRounds) return c.start + ceilf(t) * (c.round + c.step * k) + fminf(t, 1.f) * c.more * k;
    if (c.form == kTwo) return c.start + c.round * one + k * (c.step * ceilf(0.5f * t) + c.more * one);
    return c.start + c.round * one + k * (c.step + c.more * (one - 1.f));
}

struct Choice {
    enum { kS11, kS12, kS22, k64, k128, k128d, k256 } kernel;
    int parts;       // of the sum
    int64_t klen;    // products of a part, whole steps
    float time;
    bool pack;       // the operands are copied to whole aligned pieces first
};

inline int64_t up16(int64_t v) { return (v + 15) / 16 * 16; }
// Copies of both operands, where K leaves their rows no whole pieces (whole rows at odd
// strides go without: the workspace is sized before strides are known); less than 2^32 pieces.
constexpr int64_t kPackBytes = (int64_t)1 << 34;
inline size_t pack_bytes(int64_t M, int64_t N, int64_t K) {
    const int64_t Kp = up16(K);
    return K < 16 || K % 16 == 0 || M > kPackBytes / Kp || N > kPackBytes / Kp ? 0 : (size_t)((M + N) * Kp + 255) / 256 * 256;
}

constexpr int64_t kPartLen = 512;   // least products of a part
inline int64_t part_ld(int64_t N) { return (N + 7) / 8 * 8; }

// rows: what the operands' rows are made of, aligned; room: bytes of workspace.
enum Rows { kOfBytes, kOfWords, kOfPieces };

Choice choose(int64_t M, int64_t N, int64_t K, Rows rows, size_t room) {
    const bool whole = rows == kOfPieces, words = rows != kOfBytes;
    Choice c{Choice::kS11, 1, 0, cost(words ? kSmall11 : kBytes11, M, N, K), false};
    auto take = [&](decltype(c.kernel) kernel, float time, int parts, int64_t klen) {
        if (time < c.time) c = Choice{kernel, parts, klen, time, false};
    };
    take(Choice::kS12, cost(words ? kSmall12 : kBytes12, M, N, K), 1, 0);
    take(Choice::kS22, cost(words ? kSmall22 : kBytes22, M, N, K), 1, 0);
    const Cost& tile = whole ? kRing64 : kAny64;
    take(Choice::k64, cost(tile, M, N, K), 1, 0);
    if (whole) {
        take(Choice::k128, cost(kRing128, M, N, K), 1, 0);
        // (where tiles outnumber the CUs, two a CU come out a little better than the model has them)
        take(Choice::k128d, cost(kDeep128, M, N, K) * (M * N > 256 * 128 * 128 ? 1.08f : 1.f), 1, 0);
        take(Choice::k256, cost(kRing256, M, N, K), 1, 0);
    }
    // Split sums of 64 x 64 tiles: a second launch (2.3 us), and the parts' sums written and read (8 bytes at 4 TB/s).
    for (int want = 2; want <= 32 && K >= want * kPartLen; want *= 2) {
        const int64_t klen = ((K + want - 1) / want + 127) / 128 * 128;
        const int parts = (int)((K + klen - 1) / klen);
        const double bytes = (double)parts * (double)M * (double)part_ld(N) * 4.;
        if (bytes > (double)room) break;
        take(Choice::k64, cost(tile, M, N, klen * parts, parts) + 2.3f + (float)(bytes * 2. / 4e6), parts, klen);
    }
    // Rows at odd addresses: a launch that copies them to whole pieces, and the kernels for
    // those (4096 x 4096 x 4097: 246 -> 96 us, 2000 x 2000 x 1111: 20 -> 17).
    const size_t copies = whole ? 0 : pack_bytes(M, N, K);
    if (copies > 0 && copies <= room) {
        Choice p = choose(M, N, up16(K), kOfPieces, room - copies);
        p.time += 2.3f + (float)((double)copies * 2. / 3e6);   // (3 TB/s)
        p.pack = true;
        if (p.time < c.time) c = p;
    }
    return c;
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

template <typename T>
hipError_t run_64(const LinArgs& A, bool whole, hipStream_t stream) {
    return whole ? run_ring<T, 64, 64, 3, 2, 2, 128>(A, stream) : run_any<T>(A, stream);
}

template <typename T>
hipError_t run_linear(LinArgs A, void* ws, size_t ws_bytes, hipStream_t stream) {
    const int64_t ld = A.ldres * (int64_t)sizeof(T);
    A.res_dma = A.res && ld % 16 == 0 && ((uintptr_t)A.res & 15) == 0 && ld < ((int64_t)1 << 22);
    A.klen = 0;
    const bool whole = ring_takes(A);
    const Choice c = choose(A.M, A.N, A.K, whole ? kOfPieces : (word_rows(A) ? kOfWords : kOfBytes), ((uintptr_t)ws & 15) == 0 ? ws_bytes : 0);
    if (c.pack) {
        const int64_t Kp = up16(A.K);
        const uint32_t ppr = (uint32_t)(Kp / 16), pieces = (uint32_t)(A.M + A.N) * ppr;
        hipLaunchKernelGGL(linear_pack_kernel, dim3((pieces + 255) / 256), dim3(256), 0, stream, A, ppr, pieces, (int8_t*)ws);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        LinArgs P = A;
        P.a = (const int8_t*)ws, P.b = P.a + A.M * Kp;
        P.lda = P.ldb = P.K = Kp;
        const size_t copies = pack_bytes(A.M, A.N, A.K);
        return run_linear<T>(P, (char*)ws + copies, ws_bytes - copies, stream);
    }
    if (c.parts > 1) {
        LinArgs P = A;   // sums only
        P.s_a = P.s_b = nullptr;
        P.bias = P.res = nullptr;
        P.z = nullptr;
        P.res_dma = 0;
        P.out = ws;
        P.ldout = part_ld(A.N);
        P.klen = (int32_t)c.klen;
        P.part = A.M * P.ldout;
        const hipError_t e = run_64<int32_t>(P, whole, stream);
        if (e != hipSuccess) return e;
        A.part = P.part;
        const int64_t groups = (A.N + 7) / 8;
        const int tk = time_launch(NITI_TIMING_SUM, stream, "linear_join_kernel<%s>", type_name<T>());
        hipLaunchKernelGGL((linear_join_kernel<T>), dim3((unsigned)((A.M * groups + 255) / 256)), dim3(256), 0, stream, A,
                           (const int32_t*)ws, c.parts, P.ldout, (int)groups);
        timing_end(tk, stream);
        return hipGetLastError();
    }
    switch (c.kernel) {
        case Choice::kS11: return run_small<T, 1, 1>(A, stream);
        case Choice::kS12: return run_small<T, 1, 2>(A, stream);
        case Choice::kS22: return run_small<T, 2, 2>(A, stream);
        case Choice::k64: return run_64<T>(A, whole, stream);
        case Choice::k128: return run_ring<T, 128, 128, 2, 4, 2, 128>(A, stream);
        case Choice::k128d: return run_ring<T, 128, 128, 4, 4, 2, 128>(A, stream);
        default: return run_ring<T, 256, 256, 4, 2, 4, 64>(A, stream);
    }
}

// Two products that are ready together, in one launch where both are small: a
// launch takes longer than either.
template <typename T, int FM, int FN>
hipError_t run_small_pair(const LinArgs& A, const LinArgs& B, hipStream_t stream) {
    const auto tiles = [](int64_t n, int t) { return (n + t - 1) / t; };
    const int64_t na = tiles(A.N, 16 * FN), nb = tiles(B.N, 16 * FN), ba = tiles(A.M, 16 * FM) * na, bb = tiles(B.M, 16 * FM) * nb;
    const int tk = time_launch(NITI_TIMING_KERNEL, stream, "linear_small_pair_kernel<%s,%d,%d>", type_name<T>(), FM, FN);
    hipLaunchKernelGGL((linear_small_pair_kernel<T, FM, FN>), dim3((unsigned)(ba + bb)), dim3(64 * SW), 0, stream,
                       LinPair{{A, B}, {(int)na, (int)nb}, (int)ba});
    timing_end(tk, stream);
    return hipGetLastError();
}

template <typename T>
hipError_t run_ring64_pair(const LinArgs& A, const LinArgs& B, hipStream_t stream) {
    using R = Ring<64, 64, 3, 2, 2, 128>;
    constexpr auto kernel = linear_ring_pair_kernel<T, 64, 64, 3, 2, 2, 128>;
    const hipError_t e = allow_lds<kernel, R::LDS>();
    if (e != hipSuccess) return e;
    const auto tiles = [](int64_t n) { return (n + 63) / 64; };
    const int64_t na = tiles(A.N), nb = tiles(B.N), ba = tiles(A.M) * na, bb = tiles(B.M) * nb;
    const int tk = time_launch(NITI_TIMING_KERNEL, stream, "linear_ring_pair_kernel<%s,64,64,3,2,2,128>", type_name<T>());
    hipLaunchKernelGGL(kernel, dim3((unsigned)(ba + bb)), dim3(R::NT), R::LDS, stream, LinPair{{A, B}, {(int)na, (int)nb}, (int)ba});
    timing_end(tk, stream);
    return hipGetLastError();
}

constexpr float kLaunch = 2.5f;   // us that a second launch takes at least

}  // namespace

hipError_t linear_run_pair(const LinArgs& a, const LinArgs& b, int type, void* ws, size_t ws_bytes, hipStream_t stream) {
    const bool whole = ring_takes(a) && ring_takes(b) && !a.res && !b.res && a.M < kMaxSum && b.M < kMaxSum;
    if (whole) {
        const Choice ca = choose(a.M, a.N, a.K, kOfPieces, ws_bytes), cb = choose(b.M, b.N, b.K, kOfPieces, ws_bytes);
        const Choice& c = ca.time > cb.time ? ca : cb;
        const bool small_a = ca.parts == 1 && ca.kernel <= Choice::kS22, small_b = cb.parts == 1 && cb.kernel <= Choice::kS22;
        if (small_a && small_b) {
            return by_type(type, [&](auto t) {
                using T = decltype(t);
                if (c.kernel == Choice::kS11) return run_small_pair<T, 1, 1>(a, b, stream);
                if (c.kernel == Choice::kS12) return run_small_pair<T, 1, 2>(a, b, stream);
                return run_small_pair<T, 2, 2>(a, b, stream);
            });
        }
        if (cost(kRing64, a.M, a.N, a.K) + cost(kRing64, b.M, b.N, b.K) < ca.time + cb.time + kLaunch)
            return by_type(type, [&](auto t) { return run_ring64_pair<decltype(t)>(a, b, stream); });
    }
    const hipError_t e = linear_run(a, type, ws, ws_bytes, stream);
    return e == hipSuccess ? linear_run(b, type, ws, ws_bytes, stream) : e;
}

// For copies of the operands and the sums of parts, if that is how this product would go with room for them.
size_t linear_fwd_workspace(int64_t M, int64_t N, int64_t K) {
    if (M < 1 || N < 1 || K < 1 || M >= kMaxDim || N >= kMaxLd || K >= kMaxSum) return 0;
    size_t most = 0;
    for (Rows rows : {kOfBytes, kOfWords, kOfPieces}) {
        const Choice c = choose(M, N, K, rows, SIZE_MAX);
        const size_t need = (c.parts > 1 ? (size_t)c.parts * (size_t)(M * part_ld(N)) * 4 : 0) + (c.pack ? pack_bytes(M, N, K) : 0);
        most = need > most ? need : most;
    }
    return (most + 255) / 256 * 256;
}

// Very many rows go in slabs, so that a launch stays below 2^32 threads.
hipError_t linear_run(const LinArgs& args, int type, void* ws, size_t ws_bytes, hipStream_t stream) {
    LinArgs a = args;
    const int64_t size = (int64_t)type_size(type);
    const int64_t tn = (a.N + GT - 1) / GT;
    int64_t slab = ((int64_t)1 << 22) / tn * GT;   // 2^22 tiles
    if (slab < GT) slab = GT;
    for (int64_t left = args.M; left > 0; left -= slab) {
        a.M = left < slab ? left : slab;
        const hipError_t e = by_type(type, [&](auto t) { return run_linear<decltype(t)>(a, ws, ws_bytes, stream); });
        if (e != hipSuccess) return e;
        a.a += slab * a.lda;
        if (a.a_step) a.s_a += slab;
        if (a.res) a.res = (const char*)a.res + slab * a.ldres * size;
        if (a.z) a.z = (char*)a.z + slab * a.ldz * size;
        a.out = (char*)a.out + slab * a.ldout * size;
    }
    return hipSuccess;
}

}  // namespace niti

using namespace niti;

extern "C" {

niti_status niti_linear_fwd(const int8_t* a, int64_t lda, const float* s_a, int64_t s_a_n, const int8_t* b,
                            int64_t ldb, const float* s_b, int64_t s_b_n, const void* bias, int bias_type, int act,
                            const void* res, int64_t ldres, void* z, int64_t ldz, void* out, int64_t ldout, int64_t M,
                            int64_t N, int64_t K, int type, void* ws, size_t ws_bytes, void* stream) {
    if (M < 0 || N < 0 || K < 0) return NITI_ERR_SHAPE;
    if (!valid_type(type) || (bias && !valid_type(bias_type)) || act < NITI_ACT_NONE || act > NITI_ACT_SILU) return NITI_ERR_ARG;
    if (M >= kMaxDim || N >= kMaxLd || K >= kMaxSum) return NITI_ERR_UNSUPPORTED;
    if (M == 0 || N == 0) return NITI_OK;
    if (!s_a || !s_b || !out || (K > 0 && (!a || !b))) return NITI_ERR_NULL;
    if ((s_a_n != 1 && s_a_n != M) || (s_b_n != 1 && s_b_n != N)) return NITI_ERR_SHAPE;
    if (bad_ld(M > 1 ? lda : K, K, false) || bad_ld(N > 1 ? ldb : K, K, false) ||
        (res && bad_ld(M > 1 ? ldres : N, N, false)) || (z && bad_ld(M > 1 ? ldz : N, N, true)) ||
        bad_ld(M > 1 ? ldout : N, N, true))
        return NITI_ERR_SHAPE;
    if (ws_bytes > 0 && !ws) return NITI_ERR_WORKSPACE;
    const LinArgs A{a, b, s_a, s_b, bias, res, z, out, M > 1 ? lda : K, N > 1 ? ldb : K, ldres, ldz, ldout, M, N, K,
                    s_a_n == 1 ? 0 : 1, s_b_n == 1 ? 0 : 1, bias_type, act};
    return linear_run(A, type, ws, ws_bytes, (hipStream_t)stream) == hipSuccess ? NITI_OK : NITI_ERR_HIP;
}

}  // extern "C"
