// Root-mean-square norm with the residual's addition and an output in int8
// rows (forward, backward), and the int8 rows of a plain matrix.
//
// Forward, per row of D elements:  h = x + res, rstd = 1 / sqrt(mean h^2 + eps),
// y = h rstd gain, top = max |y|, codes round(y 127 / top).  Two reductions
// (the sum of squares, then the maximum) and every element needed after each:
// the row stays in registers between them, so memory is read once and written
// once, which is what bounds it.  A row of up to 2048 elements belongs to one
// wave (four rows in a workgroup, no barrier), up to 8192 to four waves, up to
// 32768 to sixteen; a longer one is read again for each pass.
//
// Backward: dx = rstd (t - xh mean(t xh)) + dh with t = dy gain, xh = h rstd.  One
// reduction per row, the row in registers as above.  dgain sums dy xh over the
// rows: a workgroup takes every G-th row and keeps its columns' sums in
// registers, writes them once to the workspace, and a second launch adds the G
// partial rows in a fixed order.
//
// Measured, bf16: 4096 x 4096 with residual and codes 30.4 us (151 MB, 5.0 TB/s; a copy
// reaches 5.3), one such row 3.0; codes of 4096 x 9216 35.9 (189 MB, 5.3 TB/s), rounded stochastically
// 50.9: two 64-bit products an element; backward of 4096 x 4096 28.5 (134 MB, 4.7 TB/s) and 4.2 for
// the second launch.  In 32 bits, backward of 1777 x 1111: 8.6 and 3.8, bound by latency with three or
// four rows a workgroup.
#include "scaled.h"

namespace niti {

namespace {

constexpr int NT_LONG = 1024;  // threads of the kernels for longer rows
constexpr int kMaxParts = 512; // partial rows of dgain

struct RowArgs {
    const void* x;
    const void* res;
    const void* gain;
    void* h;
    void* y;
    int8_t* q;
    float* scale;
    float* rstd;
    int64_t ldx, ldres, ldh, ldy, ldq;
    int64_t M, D;
    int64_t m0;      // index of the first row, for the draws
    float eps;
    int gain_type;
    int sr;
    uint64_t seed;
    uint32_t call;
};

// Sum or maximum over the threads of a row: NW waves of a workgroup.
template <int NW>
__device__ __forceinline__ float row_sum(float v, float* red, int wave) {
    v = wave_sum_f32(v);
    if (NW == 1) return v;
    if ((threadIdx.x & 63) == 0) red[wave] = v;
    __syncthreads();
    v = red[0];
#pragma unroll
    for (int i = 1; i < NW; i++) v += red[i];
    return v;
}
template <int NW>
__device__ __forceinline__ uint32_t row_max(uint32_t v, uint32_t* red, int wave) {
    v = wave_max_u32(v);
    if (NW == 1) return v;
    if ((threadIdx.x & 63) == 0) red[wave] = v;
    __syncthreads();
    v = red[0];
#pragma unroll
    for (int i = 1; i < NW; i++) v = max(v, red[i]);
    return v;
}

// Squares of values above 2^64 or so leave the 32-bit range, and those of values
// below 2^-50 its normal part: where the mean of the squares and eps, the smaller of
// which is then lost or inexact, is that large or small, the row is summed again with its elements
// scaled by a power of two (exact), and eps by its square.
constexpr float kDown = 0x1p-80f, kUp = 0x1p100f, kLow = 0x1p-100f;
__device__ __forceinline__ float norm_factor(float ss, float D, float eps) {
    return !(ss < __uint_as_float(kInfBits)) ? kDown : (ss + eps * D < kLow * D ? kUp : 1.f);
}

__device__ __forceinline__ void store_codes(int8_t* q, int n, const float (&c)[CH], uint32_t mask) {
    uint32_t w[2] = {pack4(c[0], c[1], c[2], c[3]) & mask, pack4(c[4], c[5], c[6], c[7]) & mask};
    if (n >= CH) {
        __builtin_memcpy(q, w, CH);
        return;
    }
#pragma unroll
    for (int i = 0; i < CH; i++)
        if (i < n) q[i] = (int8_t)(w[i >> 2] >> (8 * (i & 3)));
}

// Codes, scale and values of a piece at column c of row m.
template <typename T>
__device__ __forceinline__ void put_piece(const RowArgs& a, int64_t m, int64_t c, int n, float (&v)[CH], const RowScale& rs) {
    if (a.q) {
        float code[CH];
        if (a.sr) {
            DrawStream r(a.seed, a.call, (uint64_t)((a.m0 + m) * a.D + c));
#pragma unroll
            for (int e = 0; e < CH; e++) code[e] = code_sr(v[e], rs.inv, draw_hi(r.next()));
        } else {
#pragma unroll
            for (int e = 0; e < CH; e++) code[e] = code_rtn(v[e], rs.inv);
        }
#pragma unroll
        for (int e = 0; e < CH; e++) v[e] = code_value(code[e]) * rs.scale;
        store_codes(a.q + m * a.ldq + c, n, code, code_mask(rs.inv));
    }
    if (a.y) store_some((T*)a.y + m * a.ldy + c, n, v);
}

// NW waves per row, VPT pieces per thread; NORM: the norm, otherwise codes of x.
// TG: type of the gain.  All loads of a row go out together.
template <typename T, typename TG, int NW, int VPT, bool NORM, bool WHOLE>
__global__ __launch_bounds__(NW == 1 ? 256 : 64 * NW) void row_fwd_kernel(RowArgs a) {
    constexpr int NT = 64 * NW;
    __shared__ float red_s[NW], red_t[NW];
    __shared__ uint32_t red_m[NW];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t m = NW == 1 ? (int64_t)blockIdx.x * 4 + wave : (int64_t)blockIdx.x;
    if (m >= a.M) return;   // a whole wave of a workgroup that has no barrier
    const int t = NW == 1 ? (int)(threadIdx.x & 63) : (int)threadIdx.x;
    const int D = (int)a.D;
    const T* x = (const T*)a.x + m * a.ldx;
    const T* res = NORM && a.res ? (const T*)a.res + m * a.ldres : nullptr;
    Piece<T> px[VPT], pr[VPT];
    Piece<TG> pg[VPT];
#pragma unroll
    for (int i = 0; i < VPT; i++) px[i] = load_piece<T, WHOLE>(x, (i * NT + t) * CH, D);
    if constexpr (NORM) {
        // without a residual x again, which costs no traffic, in place of a branch
#pragma unroll
        for (int i = 0; i < VPT; i++) pr[i] = load_piece<T, WHOLE>(res ? res : x, (i * NT + t) * CH, D);
#pragma unroll
        for (int i = 0; i < VPT; i++) pg[i] = load_piece<TG, WHOLE>((const TG*)a.gain, (i * NT + t) * CH, D);
    }
    float v[VPT][CH];
#pragma unroll
    for (int i = 0; i < VPT; i++) piece_values<T, WHOLE>(px[i], (i * NT + t) * CH, D, v[i]);
    if constexpr (NORM) {
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < VPT; i++) {
            float r[CH];
            piece_values<T, WHOLE>(pr[i], (i * NT + t) * CH, D, r);
#pragma unroll
            for (int e = 0; e < CH; e++) {
                v[i][e] = res ? v[i][e] + r[e] : v[i][e];
                ss += v[i][e] * v[i][e];
            }
        }
        if (a.h) {
#pragma unroll
            for (int i = 0; i < VPT; i++) {
                const int c = (i * NT + t) * CH;
                if (c < D) store_some((T*)a.h + m * a.ldh + c, WHOLE ? CH : D - c, v[i]);
            }
        }
        ss = row_sum<NW>(ss, red_s, wave);
        float eps = a.eps;
        const float down = norm_factor(ss, (float)D, eps);   // the same for the whole row
        if (down != 1.f) {
            eps = eps * down * down;
            ss = 0.f;
#pragma unroll
            for (int i = 0; i < VPT; i++)
#pragma unroll
                for (int e = 0; e < CH; e++) ss += (v[i][e] * down) * (v[i][e] * down);
            ss = row_sum<NW>(ss, red_t, wave);
        }
        const float rstd = 1.f / sqrtf(ss / (float)D + eps);
        if (a.rstd && t == 0) a.rstd[m] = rstd * down;
#pragma unroll
        for (int i = 0; i < VPT; i++) {
            float g[CH];
            piece_values<TG, WHOLE>(pg[i], (i * NT + t) * CH, D, g);
#pragma unroll
            for (int e = 0; e < CH; e++) v[i][e] = (v[i][e] * down) * rstd * g[e];
        }
    }
    RowScale rs{0.f, 0.f};
    if (a.q) {
        uint32_t top = 0;   // (elements past the row are zeros)
#pragma unroll
        for (int i = 0; i < VPT; i++)
#pragma unroll
            for (int e = 0; e < CH; e++) top = max(top, mag_bits(v[i][e]));
        rs = row_scale(row_max<NW>(top, red_m, wave));
        if (t == 0) a.scale[m] = rs.scale;
    }
#pragma unroll
    for (int i = 0; i < VPT; i++) {
        const int c = (i * NT + t) * CH;
        if (c < D) put_piece<T>(a, m, c, WHOLE ? CH : D - c, v[i], rs);
    }
}

// Rows of any length, read again for each pass.  A thread reads a piece
// before it writes that piece, so outputs may be the call's own inputs.
template <typename T, bool NORM>
__global__ __launch_bounds__(NT_LONG) void row_fwd_long_kernel(RowArgs a) {
    constexpr int NW = NT_LONG / 64;
    __shared__ float red_s[NW], red_t[NW];
    __shared__ uint32_t red_m[NW];
    const int wave = threadIdx.x >> 6;
    const int64_t m = blockIdx.x;
    const T* x = (const T*)a.x + m * a.ldx;
    const T* res = a.res ? (const T*)a.res + m * a.ldres : nullptr;
    auto load = [&](int64_t c, float (&v)[CH]) {
        const int n = (int)min((int64_t)CH, a.D - c);
        load_some(x + c, n, v);
        if (NORM && res) {
            float r[CH];
            load_some(res + c, n, r);
#pragma unroll
            for (int e = 0; e < CH; e++) v[e] += r[e];
        }
    };
    float down = 1.f, rstd = 1.f;
    if constexpr (NORM) {
        auto squares = [&](float factor) {
            float s = 0.f;
            for (int64_t c = threadIdx.x * CH; c < a.D; c += NT_LONG * CH) {
                float v[CH];
                load(c, v);
#pragma unroll
                for (int e = 0; e < CH; e++) s += (v[e] * factor) * (v[e] * factor);
            }
            return s;
        };
        float s = row_sum<NW>(squares(1.f), red_s, wave), eps = a.eps;
        down = norm_factor(s, (float)a.D, eps);
        if (down != 1.f) {
            eps = eps * down * down;
            s = row_sum<NW>(squares(down), red_t, wave);
        }
        rstd = 1.f / sqrtf(s / (float)a.D + eps);
        if (a.rstd && threadIdx.x == 0) a.rstd[m] = rstd * down;
    }
    auto value = [&](int64_t c, float (&v)[CH]) {
        if constexpr (NORM) {
            float g[CH];
            load_typed(a.gain, a.gain_type, c, (int)min((int64_t)CH, a.D - c), g);
#pragma unroll
            for (int e = 0; e < CH; e++) v[e] = (v[e] * down) * rstd * g[e];
        }
    };
    RowScale rs{0.f, 0.f};
    if (a.q) {
        uint32_t top = 0;
        for (int64_t c = threadIdx.x * CH; c < a.D; c += NT_LONG * CH) {
            float v[CH];
            load(c, v);
            value(c, v);
#pragma unroll
            for (int e = 0; e < CH; e++)
                if (e < a.D - c) top = max(top, mag_bits(v[e]));
        }
        rs = row_scale(row_max<NW>(top, red_m, wave));
        if (threadIdx.x == 0) a.scale[m] = rs.scale;
    }
    for (int64_t c = threadIdx.x * CH; c < a.D; c += NT_LONG * CH) {
        const int n = (int)min((int64_t)CH, a.D - c);
        float v[CH];
        load(c, v);
        if (NORM && a.h) store_some((T*)a.h + m * a.ldh + c, n, v);
        value(c, v);
        put_piece<T>(a, m, c, n, v, rs);
    }
}

struct RowBwdArgs {
    const void* dy;
    const void* h;
    const void* gain;
    const float* rstd;
    const void* dh;
    void* dx;
    float* part;   // [gridDim.x][D], or NULL
    int64_t lddy, ldh, lddh, lddx;
    int64_t M, D;
    int gain_type;
};

template <typename T, typename TG, int NW, int VPT, bool WHOLE>
__global__ __launch_bounds__(NW == 1 ? 256 : 64 * NW) void row_bwd_kernel(RowBwdArgs a) {
    constexpr int NT = 64 * NW;
    constexpr int ROWS = NW == 1 ? 4 : 1;   // rows of a workgroup at a time
    __shared__ float red[2][NW];
    __shared__ float sums[NW == 1 ? 4 : 1][NW == 1 ? 64 * VPT * CH : 1];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int t = NW == 1 ? (int)(threadIdx.x & 63) : (int)threadIdx.x;
    const int D = (int)a.D;
    Piece<TG> pg[VPT];
#pragma unroll
    for (int i = 0; i < VPT; i++) pg[i] = load_piece<TG, WHOLE>((const TG*)a.gain, (i * NT + t) * CH, D);
    // A row's loads go out while the row before it is worked on (past the last row, that one's again);
    // sixteen waves hide them for each other, and have no registers for it.
    constexpr bool AHEAD = NW < 16;
    Piece<T> dyr[VPT], hr[VPT], er[VPT];
    float rstd_r;
    auto load = [&](int64_t m) {
        m = min(m, a.M - 1);
        rstd_r = a.rstd[m];
        const T* dy = (const T*)a.dy + m * a.lddy;
        const T* h = (const T*)a.h + m * a.ldh;
        const T* dh = a.dh ? (const T*)a.dh + m * a.lddh : dy;
#pragma unroll
        for (int i = 0; i < VPT; i++) {
            const int c = (i * NT + t) * CH;
            dyr[i] = load_piece<T, WHOLE>(dy, c, D);
            hr[i] = load_piece<T, WHOLE>(h, c, D);
            er[i] = load_piece<T, WHOLE>(dh, c, D);
        }
    };
    int par = 0;
    const int64_t step = (int64_t)gridDim.x * ROWS;
    int64_t m = (int64_t)blockIdx.x * ROWS + (NW == 1 ? wave : 0);
    if (NW > 1) __builtin_assume(m < a.M);   // (no more workgroups than rows: the first row's loads do not wait for the gain's)
    if (AHEAD) load(m);
    float g[VPT][CH], dg[VPT][CH];
#pragma unroll
    for (int i = 0; i < VPT; i++) {
        piece_values<TG, WHOLE>(pg[i], (i * NT + t) * CH, D, g[i]);
#pragma unroll
        for (int e = 0; e < CH; e++) dg[i][e] = 0.f;
    }
    for (; m < a.M; m += step, par ^= 1) {
        float dy[VPT][CH], xh[VPT][CH], r[VPT][CH];
        if (!AHEAD) load(m);
        const float rstd = rstd_r;
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < VPT; i++) {
            const int c = (i * NT + t) * CH;
            piece_values<T, WHOLE>(dyr[i], c, D, dy[i]);
            piece_values<T, WHOLE>(hr[i], c, D, xh[i]);
            piece_values<T, WHOLE>(er[i], c, D, r[i]);
        }
        if (AHEAD) load(m + step);
#pragma unroll
        for (int i = 0; i < VPT; i++)
#pragma unroll
            for (int e = 0; e < CH; e++) {
                xh[i][e] *= rstd;
                dg[i][e] += dy[i][e] * xh[i][e];
                dy[i][e] *= g[i][e];
                s += dy[i][e] * xh[i][e];
            }
        // the two halves of red alternate: a wave that is a row ahead writes the other
        const float mean = row_sum<NW>(s, red[par], wave) / (float)D;
#pragma unroll
        for (int i = 0; i < VPT; i++) {
            const int c = (i * NT + t) * CH;
            if (c >= D) continue;
#pragma unroll
            for (int e = 0; e < CH; e++) {
                const float d = rstd * (dy[i][e] - xh[i][e] * mean);
                r[i][e] = a.dh ? d + r[i][e] : d;
            }
            store_some((T*)a.dx + m * a.lddx + c, WHOLE ? CH : D - c, r[i]);
        }
    }
    if (!a.part) return;
    float* part = a.part + (int64_t)blockIdx.x * D;
    if constexpr (NW == 1) {   // the four waves hold sums of the same columns
#pragma unroll
        for (int i = 0; i < VPT; i++)
#pragma unroll
            for (int e = 0; e < CH; e++) sums[wave][(i * NT + t) * CH + e] = dg[i][e];
        __syncthreads();
        for (int c = threadIdx.x; c < D; c += 256) part[c] = (sums[0][c] + sums[1][c]) + (sums[2][c] + sums[3][c]);
    } else {
#pragma unroll
        for (int i = 0; i < VPT; i++) {
            const int c = (i * NT + t) * CH;
            if (c < D) store_some(part + c, D - c, dg[i]);
        }
    }
}

// Rows of any length; a workgroup adds its columns' sums up in the workspace.
template <typename T>
__global__ __launch_bounds__(NT_LONG) void row_bwd_long_kernel(RowBwdArgs a) {
    constexpr int NW = NT_LONG / 64;
    __shared__ float red[2][NW];
    const int wave = threadIdx.x >> 6;
    float* part = a.part ? a.part + (int64_t)blockIdx.x * a.D : nullptr;
    int par = 0;
    for (int64_t m = blockIdx.x; m < a.M; m += gridDim.x, par ^= 1) {
        const float rstd = a.rstd[m];
        const T* pdy = (const T*)a.dy + m * a.lddy;
        const T* ph = (const T*)a.h + m * a.ldh;
        float s = 0.f;
        for (int64_t c = threadIdx.x * CH; c < a.D; c += NT_LONG * CH) {
            const int n = (int)min((int64_t)CH, a.D - c);
            float dy[CH], xh[CH], g[CH];
            load_some(pdy + c, n, dy);
            load_some(ph + c, n, xh);
            load_typed(a.gain, a.gain_type, c, n, g);
#pragma unroll
            for (int e = 0; e < CH; e++) s += (dy[e] * g[e]) * (xh[e] * rstd);
        }
        const float mean = row_sum<NW>(s, red[par], wave) / (float)a.D;
        for (int64_t c = threadIdx.x * CH; c < a.D; c += NT_LONG * CH) {
            const int n = (int)min((int64_t)CH, a.D - c);
            float dy[CH], xh[CH], g[CH], r[CH];
            load_some(pdy + c, n, dy);
            load_some(ph + c, n, xh);
            load_typed(a.gain, a.gain_type, c, n, g);
            if (a.dh) load_some((const T*)a.dh + m * a.lddh + c, n, r);
            if (part) {
                float p[CH];
                load_some(part + c, m == blockIdx.x ? 0 : n, p);
#pragma unroll
                for (int e = 0; e < CH; e++) p[e] += dy[e] * (xh[e] * rstd);
                store_some(part + c, n, p);
            }
#pragma unroll
            for (int e = 0; e < CH; e++) {
                const float d = rstd * (dy[e] * g[e] - (xh[e] * rstd) * mean);
                r[e] = a.dh ? d + r[e] : d;
            }
            store_some((T*)a.dx + m * a.lddx + c, n, r);
        }
    }
}

// dgain = the partial rows' sum: 32 columns a workgroup, the partial rows
// shared by 32 groups of threads, eight loads of each in flight, and joined in order.
__global__ __launch_bounds__(1024) void dgain_kernel(const float* part, float* dgain, int64_t parts, int64_t D) {
    __shared__ float s[32][33];
    const int col = threadIdx.x & 31, grp = threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * 32 + col;
    float v = 0.f;
    if (c < D)
        for (int64_t p = grp; p < parts; p += 256) {
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; i++) x[i] = p + 32 * i < parts ? part[(p + 32 * i) * D + c] : 0.f;
#pragma unroll
            for (int i = 0; i < 8; i++) v += x[i];
        }
    s[grp][col] = v;
    __syncthreads();
    // eight partial sums of four groups, then those
    if (threadIdx.x < 256) {
        const int o = threadIdx.x >> 5;
        s[o][col] = (s[o][col] + s[o + 8][col]) + (s[o + 16][col] + s[o + 24][col]);
    }
    __syncthreads();
    if (grp == 0 && c < D) {
        v = s[0][col];
        for (int i = 1; i < 8; i++) v += s[i][col];
        dgain[c] = v;
    }
}

inline int pieces(int64_t D) { return (int)((D + CH - 1) / CH); }

template <typename T, typename TG, int NW, int VPT, bool NORM>
hipError_t launch_fwd(const RowArgs& a, hipStream_t stream) {
    const dim3 grid((unsigned)(NW == 1 ? (a.M + 3) / 4 : a.M)), block(NW == 1 ? 256 : 64 * NW);
    if (a.D % CH == 0)
        hipLaunchKernelGGL((row_fwd_kernel<T, TG, NW, VPT, NORM, true>), grid, block, 0, stream, a);
    else
        hipLaunchKernelGGL((row_fwd_kernel<T, TG, NW, VPT, NORM, false>), grid, block, 0, stream, a);
    return hipGetLastError();
}

template <typename T, typename TG, bool NORM>
hipError_t run_short_rows(const RowArgs& a, hipStream_t stream) {
    const int p = pieces(a.D);
    if (p <= 64) return launch_fwd<T, TG, 1, 1, NORM>(a, stream);
    if (p <= 128) return launch_fwd<T, TG, 1, 2, NORM>(a, stream);
    if (p <= 256) return launch_fwd<T, TG, 1, 4, NORM>(a, stream);
    if (p <= 512) return launch_fwd<T, TG, 4, 2, NORM>(a, stream);
    if (p <= 1024) return launch_fwd<T, TG, 4, 4, NORM>(a, stream);
    if (p <= 2048) return launch_fwd<T, TG, 16, 2, NORM>(a, stream);
    return launch_fwd<T, TG, 16, 4, NORM>(a, stream);
}

// Rows below one piece, above 32768 elements, and a gain of another 16-bit type than x go by the kernel for rows of any length.
template <typename T, bool NORM>
hipError_t run_rows(const RowArgs& a, hipStream_t stream) {
    if (a.D >= CH && a.D <= 32768) {
        if (!NORM || a.gain_type == type_id<T>()) return run_short_rows<T, T, NORM>(a, stream);
        if constexpr (NORM)
            if (a.gain_type == NITI_F32) return run_short_rows<T, float, NORM>(a, stream);
    }
    hipLaunchKernelGGL((row_fwd_long_kernel<T, NORM>), dim3((unsigned)a.M), dim3(NT_LONG), 0, stream, a);
    return hipGetLastError();
}

// A launch holds fewer than 2^32 threads: very many rows go in slabs.
constexpr int64_t kSlab = (int64_t)1 << 21;

template <typename T, bool NORM>
hipError_t run_fwd(RowArgs a, hipStream_t stream) {
    const int64_t M = a.M;
    for (;;) {
        a.M = M - a.m0 < kSlab ? M - a.m0 : kSlab;
        const hipError_t e = run_rows<T, NORM>(a, stream);
        if (e != hipSuccess || a.m0 + a.M >= M) return e;
        a.m0 += kSlab;
        a.x = (const T*)a.x + kSlab * a.ldx;
        if (a.res) a.res = (const T*)a.res + kSlab * a.ldres;
        if (a.h) a.h = (T*)a.h + kSlab * a.ldh;
        if (a.y) a.y = (T*)a.y + kSlab * a.ldy;
        if (a.q) a.q += kSlab * a.ldq, a.scale += kSlab;
        if (a.rstd) a.rstd += kSlab;
    }
}

template <typename T, typename TG, int NW, int VPT>
hipError_t launch_bwd(const RowBwdArgs& a, int64_t parts, hipStream_t stream) {
    const dim3 grid((unsigned)parts), block(NW == 1 ? 256 : 64 * NW);
    if (a.D % CH == 0)
        hipLaunchKernelGGL((row_bwd_kernel<T, TG, NW, VPT, true>), grid, block, 0, stream, a);
    else
        hipLaunchKernelGGL((row_bwd_kernel<T, TG, NW, VPT, false>), grid, block, 0, stream, a);
    return hipGetLastError();
}

template <typename T, typename TG>
hipError_t run_short_bwd(const RowBwdArgs& a, int64_t parts, hipStream_t stream) {
    const int p = pieces(a.D);
    if (p <= 64) return launch_bwd<T, TG, 1, 1>(a, parts, stream);
    if (p <= 128) return launch_bwd<T, TG, 1, 2>(a, parts, stream);
    if (p <= 256) return launch_bwd<T, TG, 4, 1>(a, parts, stream);
    if (p <= 512) return launch_bwd<T, TG, 4, 2>(a, parts, stream);
    if (p <= 1024) return launch_bwd<T, TG, 16, 1>(a, parts, stream);
    return launch_bwd<T, TG, 16, 2>(a, parts, stream);
}

template <typename T>
hipError_t run_bwd(const RowBwdArgs& a, int64_t parts, hipStream_t stream) {
    if (a.D >= CH && a.D <= 16384) {
        if (a.gain_type == type_id<T>()) return run_short_bwd<T, T>(a, parts, stream);
        if (a.gain_type == NITI_F32) return run_short_bwd<T, float>(a, parts, stream);
    }
    hipLaunchKernelGGL((row_bwd_long_kernel<T>), dim3((unsigned)parts), dim3(NT_LONG), 0, stream, a);
    return hipGetLastError();
}

// Workgroups of the backward pass, which is also the number of partial rows.
int64_t bwd_parts(int64_t M, int64_t D) {
    // A few rows go by one workgroup, whose sums are dgain and which saves the second launch.  Both ways (us, one launch
    // and two; bf16, 32 bits in brackets): 16 rows of 512 4.6, 5.1 (4.4, 5.1), of 1000 5.7, 5.7 (6.3, 5.8), 24 of 512 5.6, 5.1;
    // 3 rows of 4096 5.4, 5.9 (6.1, 6.1), 4 of 1111 5.9, 5.5, 4 of 4096 6.4, 6.0; 2 rows of 9216 6.5, 7.2 (8.3, 8.5), 3 8.1, 7.3.
    const int p = pieces(D), few = p <= 128 ? 16 : (p <= 512 ? 3 : 2);
    if (M <= few) return M > 0 ? 1 : 0;
    const int64_t units = p <= 128 ? (M + 3) / 4 : M;
    return units < kMaxParts ? units : kMaxParts;
}


}  // namespace

size_t rmsnorm_bwd_workspace(int64_t M, int64_t D) {
    return M > 0 && D > 0 && M < kMaxDim && D < kMaxLd ? (size_t)(bwd_parts(M, D) * D * 4 + 255) / 256 * 256 : 0;
}

}  // namespace niti

using namespace niti;

extern "C" {

niti_status niti_rmsnorm_fwd(const void* x, int64_t ldx, const void* res, int64_t ldres, const void* gain,
                             int gain_type, void* h, int64_t ldh, void* y, int64_t ldy, int8_t* q, int64_t ldq,
                             float* scale, float* rstd, int64_t M, int64_t D, float eps, int type, void* stream) {
    if (M < 0 || D < 1) return NITI_ERR_SHAPE;
    if (!valid_type(type) || !valid_type(gain_type) || !(eps >= 0.f)) return NITI_ERR_ARG;
    if (M >= kMaxDim || D >= kMaxLd) return NITI_ERR_UNSUPPORTED;
    if (M == 0) return NITI_OK;
    if (!x || !gain || (q == nullptr) != (scale == nullptr)) return NITI_ERR_NULL;
    // (one row has no stride to speak of)
    if (bad_ld(M > 1 ? ldx : D, D, false) || (res && bad_ld(M > 1 ? ldres : D, D, false)) ||
        (h && bad_ld(M > 1 ? ldh : D, D, true)) || (y && bad_ld(M > 1 ? ldy : D, D, true)) ||
        (q && bad_ld(M > 1 ? ldq : D, D, true)))
        return NITI_ERR_SHAPE;
    RowArgs a{x, res, gain, h, y, q, scale, rstd, ldx, ldres, ldh, ldy, ldq, M, D, 0, eps, gain_type, 0, 0, 0};
    return by_type(type, [&](auto t) { return run_fwd<decltype(t), true>(a, (hipStream_t)stream); }) == hipSuccess
               ? NITI_OK : NITI_ERR_HIP;
}

niti_status niti_quantize_rows(const void* x, int64_t ldx, int8_t* q, int64_t ldq, float* scale, void* y,
                               int64_t ldy, int64_t M, int64_t D, niti_round_mode mode, uint64_t seed, uint32_t call,
                               int type, void* stream) {
    if (M < 0 || D < 1) return NITI_ERR_SHAPE;
    if (!valid_type(type) || (mode != NITI_ROUND_RTN && mode != NITI_ROUND_SR)) return NITI_ERR_ARG;
    if (M >= kMaxDim || D >= kMaxLd) return NITI_ERR_UNSUPPORTED;
    if (M == 0) return NITI_OK;
    if (!x || !q || !scale) return NITI_ERR_NULL;
    if (bad_ld(M > 1 ? ldx : D, D, false) || bad_ld(M > 1 ? ldq : D, D, true) || (y && bad_ld(M > 1 ? ldy : D, D, true)))
        return NITI_ERR_SHAPE;
    RowArgs a{x, nullptr, nullptr, nullptr, y, q, scale, nullptr, ldx, 0, 0, ldy, ldq, M, D, 0, 0.f, NITI_F32,
              mode == NITI_ROUND_SR, seed, call};
    return by_type(type, [&](auto t) { return run_fwd<decltype(t), false>(a, (hipStream_t)stream); }) == hipSuccess
               ? NITI_OK : NITI_ERR_HIP;
}

niti_status niti_rmsnorm_bwd(const void* dy, int64_t lddy, const void* h, int64_t ldh, const void* gain,
                             int gain_type, const float* rstd, const void* dh, int64_t lddh, void* dx, int64_t lddx,
                             float* dgain, int64_t M, int64_t D, int type, void* ws, size_t ws_bytes, void* stream) {
    if (M < 0 || D < 1) return NITI_ERR_SHAPE;
    if (!valid_type(type) || !valid_type(gain_type)) return NITI_ERR_ARG;
    if (M >= kMaxDim || D >= kMaxLd) return NITI_ERR_UNSUPPORTED;
    if (M > 0) {
        if (!dy || !h || !gain || !rstd || !dx) return NITI_ERR_NULL;
        if (bad_ld(M > 1 ? lddy : D, D, false) || bad_ld(M > 1 ? ldh : D, D, false) ||
            (dh && bad_ld(M > 1 ? lddh : D, D, false)) || bad_ld(M > 1 ? lddx : D, D, true))
            return NITI_ERR_SHAPE;
        const size_t need = dgain ? rmsnorm_bwd_workspace(M, D) : 0;
        if (need > 0 && (!ws || ws_bytes < need)) return NITI_ERR_WORKSPACE;
        if (need > 0 && ((uintptr_t)ws & 3)) return NITI_ERR_ARG;
    }
    const int64_t parts = bwd_parts(M, D);
    hipStream_t s = (hipStream_t)stream;
    if (M > 0) {
        RowBwdArgs a{dy, h, gain, rstd, dh, dx, !dgain ? nullptr : (parts == 1 ? dgain : (float*)ws), lddy, ldh, lddh, lddx, M, D, gain_type};
        if (by_type(type, [&](auto t) { return run_bwd<decltype(t)>(a, parts, s); }) != hipSuccess) return NITI_ERR_HIP;
    }
    if (dgain && parts != 1) {   // no rows: zeros
        hipLaunchKernelGGL(dgain_kernel, dim3((unsigned)((D + 31) / 32)), dim3(1024), 0, s, (const float*)ws, dgain, parts, D);
        if (hipGetLastError() != hipSuccess) return NITI_ERR_HIP;
    }
    return NITI_OK;
}

}  // extern "C"
