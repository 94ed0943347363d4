// Backward pass of the product of int8 rows, by two int8 products.
//
// With dz = dy act'(z):  dbias = sum_m dz,
//   da[m][k] = r[m] sum_n p[m][n] b[n][k],  codes p and scales r of the rows of dz s_b,
//   db[n][k] = c[n] sum_m q[m][n] a[m][k],  codes q and scales c of the columns of dz s_a.
// Folding b's scale into the rows (it varies along their sum) and a's into the
// columns leaves both sums with integers only.
//
// Four steps.  (1) dy and z are read once for the rows' codes and for each
// column's maximum and sum, which a workgroup keeps in registers over the rows
// it takes and leaves as partial rows; (2) those are joined: c and dbias;
// (3) the columns' codes, transposed, and transposed copies of a and b: the
// products take rows along their sum; (4) the products, by the forward kernels.
#include "linear.h"

namespace niti {

namespace {

constexpr int CH = 8;
constexpr int kParts = 512;      // partial rows of the column statistics
constexpr int64_t kPad = 16;     // sums are padded to whole 16-byte pieces

inline int64_t up(int64_t v, int64_t m) { return (v + m - 1) / m * m; }

struct DzArgs {
    const void* dy;
    const void* z;
    const float* s_a;
    const float* s_b;
    int64_t lddy, ldz;
    int64_t M, N, Mp, Np;
    int32_t a_step, b_step;
    int32_t act, sr;
    uint64_t seed;
    uint32_t call;
    int8_t* p;       // [M][Np] codes of the rows, or NULL
    float* r;        // [M]
    int8_t* q;       // [N][Mp] codes of the columns, transposed, or NULL
    float* c;        // [N]
    float* dbias;    // [N] or NULL
    uint32_t* pmax;  // [parts][N] partial maxima (magnitude bits)
    float* psum;     // [parts][N]
    int64_t parts;
};

// dz of n consecutive elements from (m, c) on; zeros past them.
template <typename T>
__device__ __forceinline__ void load_dz(const DzArgs& a, int64_t m, int64_t c, int n, float (&d)[CH]) {
    load_some((const T*)a.dy + m * a.lddy + c, n, d);
    if (a.act != NITI_ACT_NONE) {
        float z[CH];
        load_some((const T*)a.z + m * a.ldz + c, n, z);
#pragma unroll
        for (int e = 0; e < CH; e++)
            if (e < n) d[e] *= act_slope(a.act, z[e]);
    }
}

// Codes of a piece of a row; the row's padding up to a multiple of 16 is zero.
__device__ __forceinline__ void put_codes(const DzArgs& a, int64_t m, int64_t c, int n, const float (&v)[CH], float inv) {
    float code[CH];
#pragma unroll
    for (int e = 0; e < CH; e++) {
        const float u = a.sr ? draw_hi(sr_draw(a.seed, a.call, (uint64_t)(m * a.N + c + e))) : 0.f;
        code[e] = e < n ? (a.sr ? code_sr(v[e], inv, u) : code_rtn(v[e], inv)) : 0.f;
    }
    const uint32_t w[2] = {pack4(code[0], code[1], code[2], code[3]), pack4(code[4], code[5], code[6], code[7])};
    __builtin_memcpy(a.p + m * a.Np + c, w, CH);
}

// Step 1 for up to 64 NW VPT 8 columns: NW waves a row.
template <typename T, int NW, int VPT>
__global__ __launch_bounds__(64 * NW) void dz_rows_kernel(DzArgs a) {
    constexpr int NT = 64 * NW;
    __shared__ uint32_t red[2][NW];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int N = (int)a.N;
    float sb[VPT][CH], sum[VPT][CH];
    uint32_t mx[VPT][CH];
#pragma unroll
    for (int i = 0; i < VPT; i++)
#pragma unroll
        for (int e = 0; e < CH; e++) {
            const int c = (i * NT + (int)threadIdx.x) * CH + e;
            sb[i][e] = c < N ? a.s_b[a.b_step ? c : 0] : 0.f;
            sum[i][e] = 0.f;
            mx[i][e] = 0;
        }
    int par = 0;
    for (int64_t m = blockIdx.x; m < a.M; m += gridDim.x, par ^= 1) {
        const float sa = a.s_a[a.a_step ? m : 0];
        float d[VPT][CH];
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < VPT; i++) {
            const int c = (i * NT + (int)threadIdx.x) * CH;
            load_dz<T>(a, m, c, N - c, d[i]);
#pragma unroll
            for (int e = 0; e < CH; e++) {
                sum[i][e] += d[i][e];
                mx[i][e] = max(mx[i][e], mag_bits(d[i][e] * sa));
                d[i][e] *= sb[i][e];
                if (c + e < N) top = max(top, mag_bits(d[i][e]));
            }
        }
        if (a.p) {
            top = wave_max_u32(top);
            if ((threadIdx.x & 63) == 0) red[par][wave] = top;
            __syncthreads();   // the halves of red alternate, see the norm's backward pass
#pragma unroll
            for (int i = 0; i < NW; i++) top = max(top, red[par][i]);
            const RowScale rs = row_scale(top);
            if (threadIdx.x == 0) a.r[m] = rs.scale;
#pragma unroll
            for (int i = 0; i < VPT; i++) {
                const int c = (i * NT + (int)threadIdx.x) * CH;
                if (c < (int)a.Np) put_codes(a, m, c, N - c, d[i], rs.inv);
            }
        }
    }
    if (!a.pmax) return;
#pragma unroll
    for (int i = 0; i < VPT; i++)
#pragma unroll
        for (int e = 0; e < CH; e++) {
            const int c = (i * NT + (int)threadIdx.x) * CH + e;
            if (c < N) {
                a.pmax[(int64_t)blockIdx.x * N + c] = mx[i][e];
                a.psum[(int64_t)blockIdx.x * N + c] = sum[i][e];
            }
        }
}

// Step 1 for more columns: each row twice, column statistics in the workspace.
template <typename T>
__global__ __launch_bounds__(1024) void dz_rows_long_kernel(DzArgs a) {
    constexpr int NW = 16;
    __shared__ uint32_t red[2][NW];
    const int wave = threadIdx.x >> 6;
    int par = 0;
    for (int64_t m = blockIdx.x; m < a.M; m += gridDim.x, par ^= 1) {
        const float sa = a.s_a[a.a_step ? m : 0];
        uint32_t top = 0;
        for (int64_t c = threadIdx.x * CH; c < a.N; c += 1024 * CH) {
            const int n = (int)min((int64_t)CH, a.N - c);
            float d[CH];
            load_dz<T>(a, m, c, n, d);
#pragma unroll
            for (int e = 0; e < CH; e++) {
                if (e >= n) continue;
                if (a.pmax) {
                    const int64_t at = (int64_t)blockIdx.x * a.N + c + e;
                    const bool first = m == blockIdx.x;
                    a.pmax[at] = max(first ? 0u : a.pmax[at], mag_bits(d[e] * sa));
                    a.psum[at] = (first ? 0.f : a.psum[at]) + d[e];
                }
                top = max(top, mag_bits(d[e] * a.s_b[a.b_step ? c + e : 0]));
            }
        }
        if (!a.p) continue;
        top = wave_max_u32(top);
        if ((threadIdx.x & 63) == 0) red[par][wave] = top;
        __syncthreads();
        for (int i = 0; i < NW; i++) top = max(top, red[par][i]);
        const RowScale rs = row_scale(top);
        if (threadIdx.x == 0) a.r[m] = rs.scale;
        for (int64_t c = threadIdx.x * CH; c < a.Np; c += 1024 * CH) {
            const int n = (int)max((int64_t)0, min((int64_t)CH, a.N - c));
            float d[CH];
            load_dz<T>(a, m, c, n, d);
#pragma unroll
            for (int e = 0; e < CH; e++)
                if (e < n) d[e] *= a.s_b[a.b_step ? c + e : 0];
            put_codes(a, m, c, n, d, rs.inv);
        }
    }
}

// Step 2: 64 columns a workgroup, partial rows shared by 16 groups and joined in order.
__global__ __launch_bounds__(1024) void dz_cols_kernel(DzArgs a) {
    __shared__ float ssum[16][64];
    __shared__ uint32_t smax[16][64];
    const int col = threadIdx.x & 63, grp = threadIdx.x >> 6;
    const int64_t c = (int64_t)blockIdx.x * 64 + col;
    float s = 0.f;
    uint32_t mx = 0;
    if (c < a.N)
        for (int64_t i = grp; i < a.parts; i += 16) {
            s += a.psum[i * a.N + c];
            mx = max(mx, a.pmax[i * a.N + c]);
        }
    ssum[grp][col] = s;
    smax[grp][col] = mx;
    __syncthreads();
    if (grp == 0 && c < a.N) {
        for (int i = 1; i < 16; i++) {
            s += ssum[i][col];
            mx = max(mx, smax[i][col]);
        }
        if (a.dbias) a.dbias[c] = s;
        a.c[c] = __uint_as_float(mx);   // step 3 forms the scale, and writes it here
    }
}

// Step 3: a 64 x 64 tile of the columns' codes, transposed through LDS.  The
// rows of a tile of column maxima are its last reader, so that the tiles of row 0
// may not replace them with the scales: those go out by dz_scale_kernel.
template <typename T>
__global__ __launch_bounds__(256) void dz_cols_codes_kernel(DzArgs a, int tiles_n) {
    __shared__ int8_t tile[64][64 + 4];
    const int64_t m0 = (int64_t)(blockIdx.x / tiles_n) * 64, n0 = (int64_t)(blockIdx.x % tiles_n) * 64;
    const int col = (threadIdx.x & 7) * CH;
#pragma unroll
    for (int i = 0; i < 2; i++) {
        const int row = (threadIdx.x >> 3) + 32 * i;
        const int64_t m = m0 + row;
        const int n = m < a.M ? (int)max((int64_t)0, min((int64_t)CH, a.N - (n0 + col))) : 0;
        float d[CH];
        if (n > 0) load_dz<T>(a, m, n0 + col, n, d);
        const float sa = n > 0 ? a.s_a[a.a_step ? m : 0] : 0.f;
#pragma unroll
        for (int e = 0; e < CH; e++) {
            float code = 0.f;   // rows past M pad the sums with zeros
            if (e < n) {
                const float inv = row_scale(__float_as_uint(a.c[n0 + col + e])).inv;
                const float v = d[e] * sa;
                code = a.sr ? code_sr(v, inv, draw_lo(sr_draw(a.seed, a.call, (uint64_t)(m * a.N + n0 + col + e)))) : code_rtn(v, inv);
            }
            tile[col + e][row] = (int8_t)(int)code;
        }
    }
    __syncthreads();
    const int row = threadIdx.x >> 2, pc = (threadIdx.x & 3) * 16;
    if (n0 + row < a.N && m0 + pc < a.Mp) {
        uint32_t w[4];
        __builtin_memcpy(w, &tile[row][pc], 16);
        *(uint4*)(a.q + (n0 + row) * a.Mp + m0 + pc) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

__global__ void dz_scale_kernel(float* c, int64_t N) {
    const int64_t n = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (n < N) c[n] = row_scale(__float_as_uint(c[n])).scale;
}

// t[k][r] = x[r][k] for r < R, zeros up to Rp (a multiple of 16).
__global__ __launch_bounds__(256) void transpose_kernel(const int8_t* x, int64_t ldx, int8_t* t, int64_t R, int64_t Rp, int64_t K,
                                                        int tiles_k) {
    __shared__ int8_t tile[64][64 + 4];
    const int64_t r0 = (int64_t)(blockIdx.x / tiles_k) * 64, k0 = (int64_t)(blockIdx.x % tiles_k) * 64;
    const int row = threadIdx.x >> 2, pc = (threadIdx.x & 3) * 16;
    int8_t v[16] = {};
    if (r0 + row < R) {
        const int8_t* src = x + (r0 + row) * ldx + k0 + pc;
        const int n = (int)min((int64_t)16, K - (k0 + pc));
        if (n == 16) {
            __builtin_memcpy(v, src, 16);
        } else {
            for (int i = 0; i < n; i++) v[i] = src[i];
        }
    }
#pragma unroll
    for (int i = 0; i < 16; i++) tile[pc + i][row] = v[i];
    __syncthreads();
    if (k0 + row < K && r0 + pc < Rp) {
        uint32_t w[4];
        __builtin_memcpy(w, &tile[row][pc], 16);
        *(uint4*)(t + (k0 + row) * Rp + r0 + pc) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

template <typename T>
hipError_t run_rows(const DzArgs& a, hipStream_t stream) {
    const unsigned grid = (unsigned)a.parts;
    const int64_t pieces = (a.N + CH - 1) / CH;
    if (pieces <= 256)
        hipLaunchKernelGGL((dz_rows_kernel<T, 4, 1>), dim3(grid), dim3(256), 0, stream, a);
    else if (pieces <= 512)
        hipLaunchKernelGGL((dz_rows_kernel<T, 4, 2>), dim3(grid), dim3(256), 0, stream, a);
    else if (pieces <= 2048)
        hipLaunchKernelGGL((dz_rows_kernel<T, 16, 2>), dim3(grid), dim3(1024), 0, stream, a);
    else
        hipLaunchKernelGGL((dz_rows_long_kernel<T>), dim3(grid), dim3(1024), 0, stream, a);
    return hipGetLastError();
}

hipError_t transpose(const int8_t* x, int64_t ldx, int8_t* t, int64_t R, int64_t Rp, int64_t K, hipStream_t stream) {
    const int64_t tr = (R + 63) / 64, tk = (K + 63) / 64;
    hipLaunchKernelGGL(transpose_kernel, dim3((unsigned)(tr * tk)), dim3(256), 0, stream, x, ldx, t, R, Rp, K, (int)tk);
    return hipGetLastError();
}

struct BwdSpace {
    int64_t Mp, Np, parts;
    int64_t p, q, at, bt, r, c, pmax, psum, total;
};

BwdSpace space(int64_t M, int64_t N, int64_t K) {
    BwdSpace s;
    s.Mp = up(M, kPad);
    s.Np = up(N, kPad);
    s.parts = M < kParts ? M : kParts;
    int64_t at = 0;
    auto take = [&](int64_t bytes) {
        const int64_t o = at;
        at += up(bytes, 256);
        return o;
    };
    s.p = take(M * s.Np);
    s.q = take(N * s.Mp);
    s.at = take(K * s.Mp);
    s.bt = take(K * s.Np);
    s.r = take(M * 4);
    s.c = take(N * 4);
    s.pmax = take(s.parts * N * 4);
    s.psum = take(s.parts * N * 4);
    s.total = at;
    return s;
}

}  // namespace

size_t linear_bwd_workspace(int64_t M, int64_t N, int64_t K) {
    return M > 0 && N > 0 && K >= 0 ? (size_t)space(M, N, K).total : 0;
}

}  // namespace niti

using namespace niti;

extern "C" {

niti_status niti_linear_bwd(const void* dy, int64_t lddy, const void* z, int64_t ldz, int act, const int8_t* a,
                            int64_t lda, const float* s_a, int64_t s_a_n, const int8_t* b, int64_t ldb,
                            const float* s_b, int64_t s_b_n, void* da, int64_t ldda, void* db, int64_t lddb,
                            float* dbias, int64_t M, int64_t N, int64_t K, niti_round_mode mode, uint64_t seed,
                            uint32_t call, int type, void* ws, size_t ws_bytes, void* stream) {
    if (M < 0 || N < 0 || K < 0) return NITI_ERR_SHAPE;
    if (!valid_type(type) || act < NITI_ACT_NONE || act > NITI_ACT_SILU) return NITI_ERR_ARG;
    if (mode != NITI_ROUND_RTN && mode != NITI_ROUND_SR) return NITI_ERR_ARG;
    if (M >= kMaxSum || N >= kMaxSum || K >= kMaxLd) return NITI_ERR_UNSUPPORTED;
    hipStream_t s = (hipStream_t)stream;
    if (K == 0) da = db = nullptr;
    if (M == 0 || N == 0) {   // sums of nothing
        if ((da && M > 0 && bad_ld(M > 1 ? ldda : K, K, true)) || (db && N > 0 && bad_ld(N > 1 ? lddb : K, K, true))) return NITI_ERR_SHAPE;
        LinArgs e{};
        e.a_step = e.b_step = 0;
        e.act = NITI_ACT_NONE;
        if (da && M > 0) {
            e.out = da, e.ldout = ldda, e.M = M, e.N = K;
            if (linear_run(e, type, nullptr, 0, s) != hipSuccess) return NITI_ERR_HIP;
        }
        if (N > 0) {
            if (db) {
                e.out = db, e.ldout = lddb, e.M = N, e.N = K;
                if (linear_run(e, type, nullptr, 0, s) != hipSuccess) return NITI_ERR_HIP;
            }
            if (dbias) {
                e.out = dbias, e.ldout = N, e.M = 1, e.N = N;
                if (linear_run(e, NITI_F32, nullptr, 0, s) != hipSuccess) return NITI_ERR_HIP;
            }
        }
        return NITI_OK;
    }
    if (!dy || !s_a || !s_b || (act != NITI_ACT_NONE && !z) || (db && !a) || (da && !b)) return NITI_ERR_NULL;
    if ((s_a_n != 1 && s_a_n != M) || (s_b_n != 1 && s_b_n != N)) return NITI_ERR_SHAPE;
    if (bad_ld(M > 1 ? lddy : N, N, false) || (act != NITI_ACT_NONE && bad_ld(M > 1 ? ldz : N, N, false)) ||
        (db && bad_ld(M > 1 ? lda : K, K, false)) || (da && bad_ld(N > 1 ? ldb : K, K, false)) ||
        (da && bad_ld(M > 1 ? ldda : K, K, true)) || (db && bad_ld(N > 1 ? lddb : K, K, true)))
        return NITI_ERR_SHAPE;
    const BwdSpace w = space(M, N, K);
    if (!ws || ws_bytes < (size_t)w.total) return NITI_ERR_WORKSPACE;
    if ((uintptr_t)ws & 15) return NITI_ERR_ARG;
    if (!da && !db && !dbias) return NITI_OK;
    char* base = (char*)ws;
    DzArgs d{};
    d.dy = dy, d.z = z, d.s_a = s_a, d.s_b = s_b;
    d.lddy = lddy, d.ldz = ldz;
    d.M = M, d.N = N, d.Mp = w.Mp, d.Np = w.Np;
    d.a_step = s_a_n == 1 ? 0 : 1, d.b_step = s_b_n == 1 ? 0 : 1;
    d.act = act, d.sr = mode == NITI_ROUND_SR, d.seed = seed, d.call = call;
    d.p = da ? (int8_t*)(base + w.p) : nullptr;
    d.r = (float*)(base + w.r);
    d.q = db ? (int8_t*)(base + w.q) : nullptr;
    d.c = (float*)(base + w.c);
    d.dbias = dbias;
    d.parts = w.parts;
    if (db || dbias) {
        d.pmax = (uint32_t*)(base + w.pmax);
        d.psum = (float*)(base + w.psum);
    }
    if (by_type(type, [&](auto t) { return run_rows<decltype(t)>(d, s); }) != hipSuccess) return NITI_ERR_HIP;
    if (db || dbias) {
        hipLaunchKernelGGL(dz_cols_kernel, dim3((unsigned)((N + 63) / 64)), dim3(1024), 0, s, d);
        if (hipGetLastError() != hipSuccess) return NITI_ERR_HIP;
    }
    if (db) {
        int8_t* at = (int8_t*)(base + w.at);
        const int64_t tm = (M + 63) / 64, tn = (N + 63) / 64;
        if (by_type(type, [&](auto t) {
                hipLaunchKernelGGL((dz_cols_codes_kernel<decltype(t)>), dim3((unsigned)(tm * tn)), dim3(256), 0, s, d, (int)tn);
                return hipGetLastError();
            }) != hipSuccess)
            return NITI_ERR_HIP;
        hipLaunchKernelGGL(dz_scale_kernel, dim3((unsigned)((N + 255) / 256)), dim3(256), 0, s, d.c, N);
        if (hipGetLastError() != hipSuccess) return NITI_ERR_HIP;
        if (transpose(a, lda, at, M, w.Mp, K, s) != hipSuccess) return NITI_ERR_HIP;
        const LinArgs A{d.q, at, d.c, nullptr, nullptr, nullptr, nullptr, db, w.Mp, w.Mp, 0, 0, lddb, N, K, w.Mp, 1, 0, 0, NITI_ACT_NONE};
        if (linear_run(A, type, nullptr, 0, s) != hipSuccess) return NITI_ERR_HIP;
    }
    if (da) {
        int8_t* bt = (int8_t*)(base + w.bt);
        if (transpose(b, ldb, bt, N, w.Np, K, s) != hipSuccess) return NITI_ERR_HIP;
        const LinArgs A{d.p, bt, d.r, nullptr, nullptr, nullptr, nullptr, da, w.Np, w.Np, 0, 0, ldda, M, K, w.Np, 1, 0, 0, NITI_ACT_NONE};
        if (linear_run(A, type, nullptr, 0, s) != hipSuccess) return NITI_ERR_HIP;
    }
    return NITI_OK;
}

}  // extern "C"
