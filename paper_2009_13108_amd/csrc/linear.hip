// Product of int8 rows with its epilogue:
//
//   z[m][n] = s_a[m] s_b[n] sum_k a[m][k] b[n][k] + bias[n],  out = act(z) + res
//
// The sum is exact in int32 (int8 MFMA); everything after it is in 32-bit
// floats, rounded once at the store.  The epilogue runs in the kernel that
// forms the sum: z, the activation and the residual cost no pass of their own.
#include "linear.h"

namespace niti {

namespace {

// ---------------------------------------------------------------- epilogue
// A wave's accumulators leave through a strip of LDS, 32 rows at a time, so
// that each lane then holds 8 consecutive columns of a row: whole cache lines
// are loaded (residual) and stored.  WTN: columns of the wave's tile.
template <int WTN>
struct Strip {
    static constexpr int PITCH = WTN + 4;          // ints; lanes of a column hit distinct banks
    static constexpr int INTS = 32 * PITCH;
    static constexpr int LPR = WTN / 8;            // lanes of a row
    static constexpr int RPP = 64 / LPR;           // rows of a pass
};

// What a lane needs of its 8 columns, the same for every row.
struct ColArgs {
    float sb[8], bias[8];
};

template <int WTN>
__device__ __forceinline__ void load_cols(const LinArgs& A, int64_t n0, ColArgs& c) {
    const int64_t n = n0 + (threadIdx.x & 63) % Strip<WTN>::LPR * 8;
    const int left = (int)min((int64_t)8, A.N - n);
#pragma unroll
    for (int e = 0; e < 8; e++) {
        c.sb[e] = A.s_b && left > 0 ? A.s_b[A.b_step ? n + min(e, left - 1) : 0] : 1.f;
        c.bias[e] = 0.f;
    }
    if (A.bias) load_typed(A.bias, A.bias_type, n, left, c.bias);
}

// 32 rows from m0 on, 8 columns a lane, from the strip.
template <typename T, int WTN>
__device__ __forceinline__ void finish_strip(const LinArgs& A, const int32_t* strip, int64_t m0, int64_t n0, const ColArgs& c) {
    using S = Strip<WTN>;
    const int lane = threadIdx.x & 63;
    const int col = lane % S::LPR * 8;
    const int64_t n = n0 + col;
    const int left = (int)min((int64_t)8, A.N - n);
#pragma unroll
    for (int r0 = 0; r0 < 32; r0 += S::RPP) {
        const int row = r0 + lane / S::LPR;
        const int64_t m = m0 + row;
        if (m >= A.M || left <= 0) continue;
        const v4i lo = *(const v4i*)(strip + row * S::PITCH + col);
        const v4i hi = *(const v4i*)(strip + row * S::PITCH + col + 4);
        const float sa = A.s_a ? A.s_a[A.a_step ? m : 0] : 1.f;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; e++) v[e] = (float)(e < 4 ? lo[e & 3] : hi[e & 3]) * (sa * c.sb[e]) + c.bias[e];
        if (A.z) store_some((T*)A.z + m * A.ldz + n, left, v);
        if (A.act != NITI_ACT_NONE) {
#pragma unroll
            for (int e = 0; e < 8; e++) v[e] = act_value(A.act, v[e]);
        }
        if (A.res) {
            float r[8];
            load_some((const T*)A.res + m * A.ldres + n, left, r);
#pragma unroll
            for (int e = 0; e < 8; e++) v[e] += r[e];
        }
        store_some((T*)A.out + m * A.ldout + n, left, v);
    }
}

// Orders a wave's own LDS writes before its reads by other lanes.
__device__ __forceinline__ void wave_lds_fence() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// Accumulators acc[a][b] (32 x 32 tiles: channels a, rows b; element 4 j + i is
// channel 32 a + 8 j + 4 (lane / 32) + i of row 32 b + lane % 32) through the strip.
template <typename T, int FN, int FM>
__device__ __forceinline__ void epilogue(const LinArgs& A, v16i (&acc)[FN][FM], int32_t* strip, int64_t m0, int64_t n0) {
    constexpr int WTN = 32 * FN;
    using S = Strip<WTN>;
    const int lane = threadIdx.x & 63;
    ColArgs c;
    load_cols<WTN>(A, n0, c);
#pragma unroll
    for (int b = 0; b < FM; b++) {
#pragma unroll
        for (int a = 0; a < FN; a++)
#pragma unroll
            for (int j = 0; j < 4; j++)
                *(v4i*)(strip + (lane & 31) * S::PITCH + 32 * a + 8 * j + 4 * (lane >> 5)) =
                    v4i{acc[a][b][4 * j], acc[a][b][4 * j + 1], acc[a][b][4 * j + 2], acc[a][b][4 * j + 3]};
        wave_lds_fence();
        finish_strip<T, WTN>(A, strip, m0 + 32 * b, n0, c);
        wave_lds_fence();
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

// 64 x 64 tiles, four waves of 32 x 32, K steps of 64 bytes through two LDS
// stages; the next step's pieces are in registers while one is computed.  Takes
// any strides and addresses.
constexpr int GT = 64, GK = 64;

__device__ __forceinline__ int gswz(int row) { return ((row >> 1) ^ (row >> 2)) & 3; }

template <typename T>
__global__ __launch_bounds__(256) void linear_any_kernel(LinArgs A, int tiles_n) {
    __shared__ __attribute__((aligned(16))) int8_t lds[2][2 * GT * GK];
    __shared__ __attribute__((aligned(16))) int32_t strips[4][Strip<32>::INTS];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t m0 = (int64_t)(blockIdx.x / tiles_n) * GT, n0 = (int64_t)(blockIdx.x % tiles_n) * GT;
    // one piece of each operand a thread: rows past the edge read row 0, whose products are not stored
    const int row = threadIdx.x >> 2, pc = threadIdx.x & 3;
    const int8_t* ra = A.a + (m0 + row < A.M ? (m0 + row) * A.lda : 0);
    const int8_t* rb = A.b + (n0 + row < A.N ? (n0 + row) * A.ldb : 0);
    const int K = (int)A.K, nk = (K + GK - 1) / GK;
    const int put = row * GK + ((pc ^ gswz(row)) << 4);
    v16i acc[1][1];
    acc[0][0] = v16i{};
    const int wm = wave & 1, wn = wave >> 1;
    v4i pa = row_piece(ra, pc * 16, K), pb = row_piece(rb, pc * 16, K);
    for (int kt = 0; kt < nk; kt++) {
        int8_t* st = lds[kt & 1];
        *(v4i*)(st + put) = pa;
        *(v4i*)(st + GT * GK + put) = pb;
        // one barrier a step: a wave writes this stage again two steps on, after the barrier in between
        __syncthreads();
        if (kt + 1 < nk) {
            pa = row_piece(ra, (kt + 1) * GK + pc * 16, K);
            pb = row_piece(rb, (kt + 1) * GK + pc * 16, K);
        }
#pragma unroll
        for (int ks = 0; ks < 2; ks++) {
            const int kp = (lane >> 5) + 2 * ks;
            const int r = lane & 31;
            const v4i fa = *(const v4i*)(st + (wm * 32 + r) * GK + ((kp ^ gswz(r)) << 4));
            const v4i fb = *(const v4i*)(st + GT * GK + (wn * 32 + r) * GK + ((kp ^ gswz(r)) << 4));
            acc[0][0] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fb, fa, acc[0][0], 0, 0, 0);
        }
    }
    epilogue<T, 1, 1>(A, acc, strips[wave], m0 + wm * 32, n0 + wn * 32);
}

template <typename T>
hipError_t run_any(const LinArgs& A, hipStream_t stream) {
    const int64_t tm = (A.M + GT - 1) / GT, tn = (A.N + GT - 1) / GT;
    hipLaunchKernelGGL((linear_any_kernel<T>), dim3((unsigned)(tm * tn)), dim3(256), 0, stream, A, (int)tn);
    return hipGetLastError();
}

template <typename T>
hipError_t run_linear(const LinArgs& A, void*, size_t, hipStream_t stream) {
    return run_any<T>(A, stream);
}

}  // namespace

size_t linear_fwd_workspace(int64_t M, int64_t N, int64_t K) {
    (void)M;
    (void)N;
    (void)K;
    return 0;
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
