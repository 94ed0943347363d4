// Backward pass of the product of int8 rows, by two int8 products.
//
// With dz = dy act'(z):  dbias = sum_m dz,
//   da[m][k] = r[m] sum_n p[m][n] b[n][k],  codes p and scales r of the rows of dz s_b,
//   db[n][k] = c[n] sum_m q[m][n] a[m][k],  codes q and scales c of the columns of dz s_a.
// Folding b's scale into the rows (it varies along their sum) and a's into the
// columns leaves both sums with integers only.
//
// A gated product out = act(gate) up has dz in two halves, dy up act'(gate) and dy act(gate),
// and goes the same way with both in one tile: dy and the halves of z are read once a pass.
//
// Up to five launches.  (1) Tiles of 16 x 256 of dz leave the maxima of their rows and
// the maxima and sums of their columns; (2) those are joined, in a fixed order:
// r, c and dbias; (3) dz is formed again, in tiles of 128 x 128, for the codes of
// rows and columns at once, the columns' transposed through LDS, and the same
// launch transposes a and b: the products take rows along their sum; (4), (5) the
// products, by the forward kernels.  Where both products are small they share a
// launch, and where the tiles of step 1 are few step 3 joins them itself: three
// launches.  dy and z are read twice, the second time
// mostly from the last-level cache; holding dz for step 3 would round it or cost
// four bytes an element each way.
//
// Measured, 2048 x 4096 x 4096 bf16 with SiLU: 13.7, 5.0, 24.8 (96 MB, 3.9 TB/s), 40.9 and
// 37.9 us (1.7 and 1.8 POPS), 109 to 117 together: the products' tiles make one and two rounds of the
// CUs, steps 1 and 3 are bound by memory with the activation's slope on top.  Gated, 2048 x 4096 (F) x 4096: 19 to 21, 5, 39, 74
// and 70 us, 205 to 210 together (step 1 by the vector units: an activation, its slope and two products an element; step 3 stores 76 MB of
// codes and transposes, and 17 of registers that two workgroups a CU do not hold; one workgroup a CU with all of them took 56); fp16
// 207; 32 bits 261, of which the codes 62 to 70.  Spilled are 16 registers in bf16, 21 in fp16 and 82 in 32 bits, where one workgroup a CU was not timed.
#include <type_traits>

#include "linear.h"

namespace niti {

namespace {

constexpr int SR = 16, SC = 256; // tile of step 1
constexpr int CT = 128, CTH = 512;   // tile of step 3 and its threads
constexpr int CP = CT + 4;       // its LDS pitch: lanes that write one row group hit distinct banks, two by two
constexpr int64_t kPad = 16;     // sums are padded to whole 16-byte pieces

inline int64_t up(int64_t v, int64_t m) { return (v + m - 1) / m * m; }

struct DzArgs {
    const void* dy;
    const void* z;
    const float* s_a;
    const float* s_b;
    int64_t lddy, ldz;
    int64_t M, N, Mp, Np;       // N: columns of dz
    int64_t W;                  // columns of dy: N, or N / 2 of a gated product
    int64_t tiles_m, tiles_n;   // of step 1
    int32_t a_step, b_step;
    int32_t act, sr;
    int32_t join;     // step 3 joins the tiles of step 1
    uint64_t seed;
    uint32_t call;
    int8_t* p;        // [M][Np] codes of the rows, or NULL
    int8_t* q;        // [N][Mp] codes of the columns, transposed, or NULL
    float* r;         // [2][M] scales, and the factors that form codes
    float* c;         // [2][N]
    float* dbias;     // [N] or NULL
    uint32_t* rmax;   // [tiles_n][M] magnitude bits of the row maxima
    uint32_t* cmax;   // [tiles_m][N]
    float* csum;      // [tiles_m][N]
};

// dz of 8 columns from c on of rows m, m + step, ...; zeros past the edges.  All
// loads go out before the first is used (see load_piece).  KIND: the number of
// columns of dy is a multiple of 8 (2), is at least 8 (1), or neither (0).
// G: a gated product's two halves, dy up act'(gate) and dy act(gate), from three loads.
template <typename T, int KIND, int ROWS, bool G>
struct DzRows {
    static constexpr int H = G ? 2 : 1;
    Piece<T> y[KIND ? ROWS : 1], z[KIND ? ROWS : 1], u[KIND && G ? ROWS : 1];
    __device__ __forceinline__ void load(const DzArgs& a, int64_t m, int64_t step, int c) {
        if constexpr (KIND > 0) {
#pragma unroll
            for (int i = 0; i < ROWS; i++) {
                const int64_t r = min(m + i * step, a.M - 1);
                y[i] = load_piece<T, KIND == 2>((const T*)a.dy + r * a.lddy, c, (int)a.W);
                z[i] = load_piece<T, KIND == 2>((const T*)a.z + r * a.ldz, c, (int)a.W);
                if constexpr (G) u[i] = load_piece<T, KIND == 2>((const T*)a.z + r * a.ldz + a.W, c, (int)a.W);
            }
        }
    }
    // What was formed of the loads is formed anew from here on, in place of being kept.
    __device__ __forceinline__ void forget_values() {
        if constexpr (KIND > 0) {
#pragma unroll
            for (int i = 0; i < ROWS; i++)
#pragma unroll
                for (int w = 0; w < (int)(sizeof(y[i].w) / 4); w++) asm volatile("" : "+v"(y[i].w[w]), "+v"(z[i].w[w]));
        }
    }
    // half HALF's values, the only one's or (-1) both
    template <int HALF>
    __device__ __forceinline__ void get(const DzArgs& a, int i, int64_t m, int c, float (&d)[H][CH]) {
        const int W = (int)a.W;
        float s[CH], v[CH];
        if constexpr (KIND > 0) {
            piece_values<T, KIND == 2>(y[i], c, W, d[0]);
            piece_values<T, KIND == 2>(z[i], c, W, s);
            if constexpr (G && HALF != 1) piece_values<T, KIND == 2>(u[i], c, W, v);
        } else {
            const int64_t r = min(m, a.M - 1);
            load_some((const T*)a.dy + r * a.lddy + c, W - c, d[0]);
            if (G || a.act != NITI_ACT_NONE) load_some((const T*)a.z + r * a.ldz + c, W - c, s);
            if constexpr (G && HALF != 1) load_some((const T*)a.z + r * a.ldz + a.W + c, W - c, v);
        }
        if constexpr (G && HALF != 0) {
#pragma unroll
            for (int e = 0; e < CH; e++) d[1][e] = s[e];
            act_values(a.act, d[1]);
#pragma unroll
            for (int e = 0; e < CH; e++) d[1][e] *= d[0][e];
        }
        if constexpr (G && HALF != 1) {
#pragma unroll
            for (int e = 0; e < CH; e++) d[0][e] *= v[e];
        }
        if (HALF != 1 && a.act != NITI_ACT_NONE) {
            act_slopes(a.act, s);
#pragma unroll
            for (int e = 0; e < CH; e++) d[0][e] *= s[e];
        }
#pragma unroll
        for (int h = 0; h < H; h++)
#pragma unroll
            for (int e = 0; e < CH; e++) d[h][e] = m < a.M ? d[h][e] : 0.f;
    }
};

// A vector's values of 8 columns from c on (stride 0: one value for all); zeros past the edge.
template <int KIND>
__device__ __forceinline__ void load_cols(const float* p, int step, int c, int N, float (&v)[CH]) {
    if (!step) {
        const float one = p[0];
#pragma unroll
        for (int e = 0; e < CH; e++) v[e] = c + e < N ? one : 0.f;
    } else if constexpr (KIND > 0) {
        piece_values<float, KIND == 2>(load_piece<float, KIND == 2>(p, c, N), c, N, v);
    } else {
        load_some(p + c, N - c, v);
    }
}

// Step 1.  A thread takes 8 columns of 2 rows; 32 lanes a row, 8 threads a column group.
template <typename T, int KIND, bool G>
__global__ __launch_bounds__(256) void dz_stats_kernel(DzArgs a) {
    constexpr int H = G ? 2 : 1;
    __shared__ float ssum[H][8][SC + 8];
    __shared__ uint32_t smax[H][8][SC + 8];
    const int64_t tm = blockIdx.x / (uint32_t)a.tiles_n, tn = blockIdx.x % (uint32_t)a.tiles_n;
    const int col = (threadIdx.x & 31) * CH, grp = threadIdx.x >> 5;
    const int c = (int)(tn * SC + col);
    DzRows<T, KIND, SR / 8, G> rows;
    rows.load(a, tm * SR + grp, 8, c);
    float sb[H][CH], sum[H][CH], sa[SR / 8];
    uint32_t mx[H][CH];
#pragma unroll
    for (int i = 0; i < SR / 8; i++) sa[i] = a.s_a[a.a_step ? min(tm * SR + i * 8 + grp, a.M - 1) : 0];
#pragma unroll
    for (int h = 0; h < H; h++) {
        load_cols<KIND>(a.s_b + (a.b_step ? h * a.W : 0), a.b_step, c, (int)a.W, sb[h]);
#pragma unroll
        for (int e = 0; e < CH; e++) sum[h][e] = 0.f, mx[h][e] = 0;
    }
#pragma unroll
    for (int i = 0; i < SR / 8; i++) {
        const int64_t m = tm * SR + i * 8 + grp;
        float d[H][CH];
        rows.template get<G ? -1 : 0>(a, i, m, c, d);
        uint32_t top = 0;
#pragma unroll
        for (int h = 0; h < H; h++)
#pragma unroll
            for (int e = 0; e < CH; e++) {
                sum[h][e] += d[h][e];
                mx[h][e] = max(mx[h][e], mag_bits(d[h][e] * sa[i]));
                top = max(top, mag_bits(d[h][e] * sb[h][e]));   // (zeros past the edges)
            }
#pragma unroll
        for (int o = 16; o >= 1; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o, 32));
        if ((threadIdx.x & 31) == 0 && m < a.M) a.rmax[tn * a.M + m] = top;
    }
#pragma unroll
    for (int h = 0; h < H; h++)
#pragma unroll
        for (int e = 0; e < CH; e++) ssum[h][grp][col + e] = sum[h][e], smax[h][grp][col + e] = mx[h][e];
    __syncthreads();
    const int64_t cc = tn * SC + threadIdx.x;
    if (cc < a.W) {
#pragma unroll
        for (int h = 0; h < H; h++) {
            float s = ssum[h][0][threadIdx.x];
            uint32_t m = smax[h][0][threadIdx.x];
            for (int g = 1; g < 8; g++) {
                s += ssum[h][g][threadIdx.x];
                m = max(m, smax[h][g][threadIdx.x]);
            }
            a.csum[tm * a.N + h * a.W + cc] = s;
            a.cmax[tm * a.N + h * a.W + cc] = m;
        }
    }
}

// Row m's and column c's scales from the tiles' values, in the order of the tiles.
__device__ __forceinline__ RowScale join_row(const DzArgs& a, int64_t m) {
    uint32_t mx = 0;
#pragma unroll 8
    for (int64_t t = 0; t < a.tiles_n; t++) mx = max(mx, a.rmax[t * a.M + m]);
    return row_scale(mx);
}

// Step 2.  Columns: 64 a workgroup, the tiles' values shared by 16 groups and joined in order.  Rows: 1024 a workgroup.
__global__ __launch_bounds__(1024) void dz_join_kernel(DzArgs a, int col_blocks) {
    __shared__ float ssum[16][64];
    __shared__ uint32_t smax[16][64];
    if ((int)blockIdx.x >= col_blocks) {
        const int64_t m = (int64_t)((int)blockIdx.x - col_blocks) * 1024 + threadIdx.x;
        if (m >= a.M) return;
        const RowScale rs = join_row(a, m);
        a.r[m] = rs.scale;
        a.r[a.M + m] = rs.inv;
        return;
    }
    const int col = threadIdx.x & 63, grp = threadIdx.x >> 6;
    const int64_t c = (int64_t)blockIdx.x * 64 + col;
    float s = 0.f;
    uint32_t mx = 0;
    if (c < a.N)
        for (int64_t i = grp; i < a.tiles_m; i += 128) {   // eight tiles' values in flight
            float x[8];
            uint32_t y[8];
#pragma unroll
            for (int j = 0; j < 8; j++) {
                const int64_t t = min(i + 16 * j, a.tiles_m - 1);
                x[j] = a.csum[t * a.N + c];
                y[j] = a.cmax[t * a.N + c];
            }
#pragma unroll
            for (int j = 0; j < 8; j++) {
                s += i + 16 * j < a.tiles_m ? x[j] : 0.f;
                mx = max(mx, y[j]);
            }
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
        const RowScale rs = row_scale(mx);
        a.c[c] = rs.scale;
        a.c[a.N + c] = rs.inv;
    }
}

// A CT x CT tile of bytes in LDS, transposed, to rows from n0 on (`rows` of them) of stride ld, columns m0 .. cols - 1 (whole pieces).
__device__ __forceinline__ void store_turned(const int8_t (*tile)[CP], int8_t* out, int64_t ld, int64_t n0, int64_t rows, int64_t m0,
                                             int64_t cols) {
#pragma unroll
    for (int i = 0; i < CT * CT / 16 / CTH; i++) {
        const int idx = i * CTH + threadIdx.x, row = idx / (CT / 16), pc = idx % (CT / 16) * 16;
        if (n0 + row >= rows || m0 + pc >= cols) continue;
        uint32_t w[4];
        __builtin_memcpy(w, &tile[row][pc], 16);
        *(uint4*)(out + (n0 + row) * ld + m0 + pc) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// 4 x 4 bytes: w[i] holds row i's four columns and then column i's four rows.
__device__ __forceinline__ void turn4(uint32_t (&w)[4]) {
    const uint32_t a = __builtin_amdgcn_perm(w[1], w[0], 0x05010400), b = __builtin_amdgcn_perm(w[1], w[0], 0x07030602);
    const uint32_t c = __builtin_amdgcn_perm(w[3], w[2], 0x05010400), d = __builtin_amdgcn_perm(w[3], w[2], 0x07030602);
    w[0] = __builtin_amdgcn_perm(c, a, 0x05040100);
    w[1] = __builtin_amdgcn_perm(c, a, 0x07060302);
    w[2] = __builtin_amdgcn_perm(d, b, 0x05040100);
    w[3] = __builtin_amdgcn_perm(d, b, 0x07060302);
}

// x [R][K] to be turned into t [K][Rp], zeros from column R to Rp (a multiple of 16).
struct Turn {
    const int8_t* x;
    int8_t* t;
    int64_t ldx, R, Rp, K;
    int32_t blocks, tiles_k;
};

__device__ __forceinline__ void turn_tile(const Turn& a, int block, int8_t (*tile)[CP]) {
    const int64_t r0 = (int64_t)((uint32_t)block / (uint32_t)a.tiles_k) * CT, k0 = (int64_t)((uint32_t)block % (uint32_t)a.tiles_k) * CT;
    const int pc = (threadIdx.x & 15) * 8, row = (threadIdx.x >> 4) * 4;   // four rows of 8 bytes a thread
    uint64_t v[4];
    const int64_t k = k0 + pc;
    if (a.K >= 8) {
        // (no load in a branch: past the edges the last row's or a row's last piece, set right afterwards)
#pragma unroll
        for (int i = 0; i < 4; i++) __builtin_memcpy(&v[i], a.x + min(r0 + row + i, a.R - 1) * a.ldx + min(k, a.K - 8), 8);
        if (k0 + CT > a.K || r0 + CT > a.R) {
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const int down = r0 + row + i < a.R ? (int)min((int64_t)8, max((int64_t)0, k + 8 - a.K)) : 8;
                v[i] = down < 8 ? v[i] >> (8 * down) : 0;
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; i++) {
            v[i] = 0;
            if (r0 + row + i < a.R)
                for (int e = 0; e < a.K - k; e++) v[i] |= (uint64_t)(uint8_t)a.x[(r0 + row + i) * a.ldx + k + e] << (8 * e);
        }
    }
#pragma unroll
    for (int g = 0; g < 2; g++) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; i++) w[i] = (uint32_t)(v[i] >> (32 * g));
        turn4(w);
#pragma unroll
        for (int i = 0; i < 4; i++) *(uint32_t*)&tile[pc + 4 * g + i][row] = w[i];
    }
    __syncthreads();
    store_turned(tile, a.t, a.Rp, k0, a.K, r0, a.Rp);
}

// Step 3: a CT x CT tile of codes, or one of a's or b's transposed copies.
template <typename T, int KIND, bool G>
__global__ __launch_bounds__(CTH, G ? 4 : 1) void dz_codes_kernel(DzArgs a, Turn ta, Turn tb, int codes, int tiles_c) {
    constexpr int H = G ? 2 : 1;
    __shared__ __attribute__((aligned(16))) int8_t tile[H][CT][CP];
    __shared__ __attribute__((aligned(16))) float rinv[CT], cinv[H * CT], scale[H * CT];
    int block = blockIdx.x;
    if (block >= codes) {   // the codes' tiles, which take longest, are first
        block -= codes;
        if (block < ta.blocks) turn_tile(ta, block, tile[0]);
        else turn_tile(tb, block - ta.blocks, tile[0]);
        return;
    }
    const int64_t m0 = (int64_t)((uint32_t)block / (uint32_t)tiles_c) * CT, n0 = (int64_t)((uint32_t)block % (uint32_t)tiles_c) * CT;
    const int col = (threadIdx.x & 15) * CH, row0 = (threadIdx.x >> 4) * 4;   // 8 columns of 4 rows a thread
    const int c = (int)(n0 + col);
    float sa[4];
    DzRows<T, KIND, 4, G> rows;
    rows.load(a, m0 + row0, 1, c);
#pragma unroll
    for (int i = 0; i < 4; i++) sa[i] = a.s_a[a.a_step ? min(m0 + row0 + i, a.M - 1) : 0];
    {   // the tile's factors: 128 threads a row each, 128 a column (of each half)
        const int i = threadIdx.x & (CT - 1), half = G ? (int)threadIdx.x / CT - 1 : 0;
        const int64_t m = min(m0 + i, a.M - 1), n = half * a.W + min(n0 + i, a.W - 1);
        if (threadIdx.x < CT) {
            float inv;
            if (a.join) {
                const RowScale rs = join_row(a, m);
                if (n0 == 0 && m0 + i < a.M) a.r[m] = rs.scale;
                inv = rs.inv;
            } else {
                inv = a.r[a.M + m];
            }
            rinv[i] = inv;
        } else if (threadIdx.x < (1 + H) * CT) {
            float inv;
            if (a.join) {
                float s = 0.f;
                uint32_t mx = 0;
                // up to 32 tiles, in step 2's order: the 16 groups' sums one after the other
                const int groups = (int)min((int64_t)16, a.tiles_m);
#pragma unroll 8
                for (int g = 0; g < groups; g++) {
                    const int64_t two = min((int64_t)g + 16, a.tiles_m - 1);
                    const float x = a.csum[g * a.N + n], y = a.csum[two * a.N + n];
                    s += g + 16 < a.tiles_m ? x + y : x;
                    mx = max(mx, max(a.cmax[g * a.N + n], a.cmax[two * a.N + n]));
                }
                const RowScale rs = row_scale(mx);
                if (m0 == 0 && n0 + i < a.W) {
                    a.c[n] = rs.scale;
                    if (a.dbias) a.dbias[n] = s;
                }
                inv = rs.inv;
            } else {
                inv = a.c[a.N + n];
            }
            cinv[half * CT + i] = n0 + i < a.W ? inv : 0.f;
            scale[half * CT + i] = a.s_b[a.b_step ? n : 0];
        }
    }
    __syncthreads();
    // (a gated product's halves one after the other: both at once take more registers than two workgroups a CU leave)
    auto half_codes = [&](auto half) {
        constexpr int h = decltype(half)::value;
        float sb[CH], ci[CH];
        uint32_t cmask[2] = {0, 0}, qc[4][2];   // codes of the columns: four rows of eight bytes
#pragma unroll
        for (int e = 0; e < CH; e++) {
            sb[e] = scale[h * CT + col + e];
            ci[e] = cinv[h * CT + col + e];
            cmask[e >> 2] |= (code_mask(ci[e]) & 0xFFu) << (8 * (e & 3));
        }
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const int64_t m = m0 + row0 + i;
            const bool in = m < a.M;   // rows past M are zeros, which pad the sums over m
            float both[H][CH], pc[CH], cc[CH];
            rows.template get<h>(a, i, m, c, both);
            const float(&d)[CH] = both[h];
            const float ri = rinv[row0 + i];
            if (a.sr) {
                DrawStream r(a.seed, a.call, (uint64_t)(m * a.N + h * a.W + c));
#pragma unroll
                for (int e = 0; e < CH; e++) {
                    const uint64_t u = r.next();
                    pc[e] = code_sr(d[e] * sb[e], ri, draw_hi(u));
                    cc[e] = code_sr(d[e] * sa[i], ci[e], draw_lo(u));
                }
            } else {
#pragma unroll
                for (int e = 0; e < CH; e++) {
                    pc[e] = code_rtn(d[e] * sb[e], ri);
                    cc[e] = code_rtn(d[e] * sa[i], ci[e]);
                }
            }
            // (past the edges dz is 0, and so are the codes: a draw is below 1)
            if (a.p && in) {
                const uint32_t mask = code_mask(ri);
                const uint32_t w[2] = {pack4(pc[0], pc[1], pc[2], pc[3]) & mask, pack4(pc[4], pc[5], pc[6], pc[7]) & mask};
                // a gate's row of codes ends where its partner's begins, that one's (or the only one) where the padding does
                const int end = G && h == 0 ? (int)a.W : (int)(a.Np - h * a.W);
                int8_t* dst = a.p + m * a.Np + h * a.W + c;
                if (!G || c + CH <= end) {
                    if (c < end) __builtin_memcpy(dst, w, CH);
                } else {
#pragma unroll
                    for (int e = 0; e < CH; e++)
                        if (c + e < end) dst[e] = (int8_t)(w[e >> 2] >> (8 * (e & 3)));
                }
            }
            qc[i][0] = pack4(cc[0], cc[1], cc[2], cc[3]) & cmask[0];
            qc[i][1] = pack4(cc[4], cc[5], cc[6], cc[7]) & cmask[1];
        }
#pragma unroll
        for (int g = 0; g < 2; g++) {
            uint32_t w[4] = {qc[0][g], qc[1][g], qc[2][g], qc[3][g]};
            turn4(w);
#pragma unroll
            for (int i = 0; i < 4; i++) *(uint32_t*)&tile[h][col + 4 * g + i][row0] = w[i];
        }
    };
    half_codes(std::integral_constant<int, 0>());
    if constexpr (G) {
        rows.forget_values();
        half_codes(std::integral_constant<int, 1>());
    }
    if (!a.q) return;
    __syncthreads();
#pragma unroll
    for (int h = 0; h < H; h++) store_turned(tile[h], a.q, a.Mp, h * a.W + n0, (h + 1) * a.W, m0, a.Mp);
}

// Calls f with the column count's KIND.
template <typename F>
hipError_t by_kind(int64_t W, F f) {
    if (W % CH == 0) return f(std::integral_constant<int, 2>());
    if (W > CH) return f(std::integral_constant<int, 1>());
    return f(std::integral_constant<int, 0>());
}

template <typename T, bool G>
hipError_t run_stats(const DzArgs& a, hipStream_t stream) {
    return by_kind(a.W, [&](auto k) {
        hipLaunchKernelGGL((dz_stats_kernel<T, decltype(k)::value, G>), dim3((unsigned)(a.tiles_m * a.tiles_n)), dim3(256), 0, stream, a);
        return hipGetLastError();
    });
}

template <typename T, bool G>
hipError_t run_codes(const DzArgs& a, const Turn& ta, const Turn& tb, int64_t tiles, int tiles_c, hipStream_t stream) {
    return by_kind(a.W, [&](auto k) {
        hipLaunchKernelGGL((dz_codes_kernel<T, decltype(k)::value, G>), dim3((unsigned)(ta.blocks + tb.blocks + tiles)), dim3(CTH), 0,
                           stream, a, ta, tb, (int)tiles, tiles_c);
        return hipGetLastError();
    });
}

struct BwdSpace {
    int64_t Mp, Np, tiles_m, tiles_n;
    int64_t p, q, at, bt, r, c, rmax, cmax, csum, sums, sums_bytes, total;
};

// W: columns of dy, N or half of that.
BwdSpace space(int64_t M, int64_t N, int64_t W, int64_t K) {
    BwdSpace s;
    s.Mp = up(M, kPad);
    s.Np = up(N, kPad);
    s.tiles_m = (M + SR - 1) / SR;
    s.tiles_n = (W + SC - 1) / SC;
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
    s.r = take(M * 8);
    s.c = take(N * 8);
    s.rmax = take(s.tiles_n * M * 4);
    s.cmax = take(s.tiles_m * N * 4);
    s.csum = take(s.tiles_m * N * 4);
    // the products' own workspace
    const size_t wa = linear_fwd_workspace(M, K, s.Np), wb = linear_fwd_workspace(N, K, s.Mp);
    s.sums_bytes = (int64_t)(wa > wb ? wa : wb);
    s.sums = take(s.sums_bytes);
    s.total = at;
    return s;
}

}  // namespace

size_t linear_bwd_workspace(int64_t M, int64_t N, int64_t K) {
    return M > 0 && N > 0 && K >= 0 && M < kMaxSum && N < kMaxSum && K < kMaxLd ? (size_t)space(M, N, N, K).total : 0;
}
size_t gated_bwd_workspace(int64_t M, int64_t F, int64_t K) {
    return M > 0 && F > 0 && K >= 0 && M < kMaxSum && F < kMaxSum / 2 && K < kMaxLd ? (size_t)space(M, 2 * F, F, K).total : 0;
}

namespace {

// G: N counts the columns of dz, gates and their partners.
template <bool G>
niti_status linear_backward(const void* dy, int64_t lddy, const void* z, int64_t ldz, int act, const int8_t* a,
                            int64_t lda, const float* s_a, int64_t s_a_n, const int8_t* b, int64_t ldb,
                            const float* s_b, int64_t s_b_n, void* da, int64_t ldda, void* db, int64_t lddb,
                            float* dbias, int64_t M, int64_t N, int64_t K, niti_round_mode mode, uint64_t seed,
                            uint32_t call, int type, void* ws, size_t ws_bytes, void* stream) {
    if (M < 0 || N < 0 || K < 0) return NITI_ERR_SHAPE;
    if (!valid_type(type) || act < NITI_ACT_NONE || act > NITI_ACT_SILU) return NITI_ERR_ARG;
    if (mode != NITI_ROUND_RTN && mode != NITI_ROUND_SR) return NITI_ERR_ARG;
    if (M >= kMaxSum || N >= kMaxSum || K >= kMaxLd) return NITI_ERR_UNSUPPORTED;
    const int64_t W = G ? N / 2 : N;   // columns of dy
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
    const bool has_z = G || act != NITI_ACT_NONE;
    if (!dy || !s_a || !s_b || (has_z && !z) || (db && !a) || (da && !b)) return NITI_ERR_NULL;
    if ((s_a_n != 1 && s_a_n != M) || (s_b_n != 1 && s_b_n != N)) return NITI_ERR_SHAPE;
    if (bad_ld(M > 1 ? lddy : W, W, false) || (has_z && bad_ld(M > 1 ? ldz : N, N, false)) ||
        (db && bad_ld(M > 1 ? lda : K, K, false)) || (da && bad_ld(N > 1 ? ldb : K, K, false)) ||
        (da && bad_ld(M > 1 ? ldda : K, K, true)) || (db && bad_ld(N > 1 ? lddb : K, K, true)))
        return NITI_ERR_SHAPE;
    const BwdSpace w = space(M, N, W, K);
    if (!ws || ws_bytes < (size_t)w.total) return NITI_ERR_WORKSPACE;
    if ((uintptr_t)ws & 15) return NITI_ERR_ARG;
    if (!da && !db && !dbias) return NITI_OK;
    char* base = (char*)ws;
    DzArgs d{};
    // without an activation dy stands for z, so that the kernels' loads need no branch
    d.dy = dy, d.z = has_z ? z : dy, d.s_a = s_a, d.s_b = s_b;
    d.lddy = lddy, d.ldz = has_z ? ldz : lddy;
    d.M = M, d.N = N, d.W = W, d.Mp = w.Mp, d.Np = w.Np;
    d.a_step = s_a_n == 1 ? 0 : 1, d.b_step = s_b_n == 1 ? 0 : 1;
    d.act = act, d.sr = mode == NITI_ROUND_SR, d.seed = seed, d.call = call;
    d.tiles_m = w.tiles_m, d.tiles_n = w.tiles_n;
    d.p = da ? (int8_t*)(base + w.p) : nullptr;
    d.q = db ? (int8_t*)(base + w.q) : nullptr;
    d.r = (float*)(base + w.r);
    d.c = (float*)(base + w.c);
    d.dbias = dbias;
    d.rmax = (uint32_t*)(base + w.rmax);
    d.cmax = (uint32_t*)(base + w.cmax);
    d.csum = (float*)(base + w.csum);
    if (by_type(type, [&](auto t) { return run_stats<decltype(t), G>(d, s); }) != hipSuccess) return NITI_ERR_HIP;
    // Tiles of step 3 read those of step 1 that they lie in, each again: up to 32 by 40 of them (512 x 10240) that takes
    // less than a launch (250 x 4096 x 512 26.3 -> 24.5 us, 200 x 9000 x 1024 45.2 -> 42.9, 400 x 1024 x 512 18.2 -> 16.5,
    // 512 x 10240 x 512 44.6 -> 42.7).
    d.join = (da || db) && w.tiles_m <= 32 && w.tiles_n <= 40;
    if (!d.join) {
        const int64_t cols = (N + 63) / 64;
        hipLaunchKernelGGL(dz_join_kernel, dim3((unsigned)(cols + (M + 1023) / 1024)), dim3(1024), 0, s, d, (int)cols);
        if (hipGetLastError() != hipSuccess) return NITI_ERR_HIP;
    }
    if (!da && !db) return NITI_OK;
    // (a gated product's last columns are followed by the padding of the rows of codes)
    const int64_t tr = (M + CT - 1) / CT, tn = (N + CT - 1) / CT, tc = G ? (w.Np - W + CT - 1) / CT : tn, tk = (K + CT - 1) / CT;
    Turn ta{a, (int8_t*)(base + w.at), lda, M, w.Mp, K, db ? (int32_t)(tr * tk) : 0, (int32_t)tk};
    Turn tb{b, (int8_t*)(base + w.bt), ldb, N, w.Np, K, da ? (int32_t)(tn * tk) : 0, (int32_t)tk};
    if (by_type(type, [&](auto t) { return run_codes<decltype(t), G>(d, ta, tb, tr * tc, (int)tc, s); }) != hipSuccess)
        return NITI_ERR_HIP;
    const LinArgs B{d.q, ta.t, d.c, nullptr, nullptr, nullptr, nullptr, db, w.Mp, w.Mp, 0, 0, lddb, N, K, w.Mp, 1, 0, 0, NITI_ACT_NONE, 0, 0, 0};
    const LinArgs A{d.p, tb.t, d.r, nullptr, nullptr, nullptr, nullptr, da, w.Np, w.Np, 0, 0, ldda, M, K, w.Np, 1, 0, 0, NITI_ACT_NONE, 0, 0, 0};
    void* sums = base + w.sums;
    const hipError_t e = da && db ? linear_run_pair(B, A, type, sums, (size_t)w.sums_bytes, s)
                                  : linear_run(da ? A : B, type, sums, (size_t)w.sums_bytes, s);
    if (e != hipSuccess) return NITI_ERR_HIP;
    return NITI_OK;
}

}  // namespace

}  // namespace niti

using namespace niti;

extern "C" {

niti_status niti_linear_bwd(const void* dy, int64_t lddy, const void* z, int64_t ldz, int act, const int8_t* a,
                            int64_t lda, const float* s_a, int64_t s_a_n, const int8_t* b, int64_t ldb,
                            const float* s_b, int64_t s_b_n, void* da, int64_t ldda, void* db, int64_t lddb,
                            float* dbias, int64_t M, int64_t N, int64_t K, niti_round_mode mode, uint64_t seed,
                            uint32_t call, int type, void* ws, size_t ws_bytes, void* stream) {
    return linear_backward<false>(dy, lddy, z, ldz, act, a, lda, s_a, s_a_n, b, ldb, s_b, s_b_n, da, ldda, db, lddb, dbias, M, N, K,
                                  mode, seed, call, type, ws, ws_bytes, stream);
}

niti_status niti_gated_bwd(const void* dy, int64_t lddy, const void* z, int64_t ldz, int act, const int8_t* a, int64_t lda,
                           const float* s_a, int64_t s_a_n, const int8_t* b, int64_t ldb, const float* s_b, int64_t s_b_n, void* da,
                           int64_t ldda, void* db, int64_t lddb, float* dbias, int64_t M, int64_t F, int64_t K, niti_round_mode mode,
                           uint64_t seed, uint32_t call, int type, void* ws, size_t ws_bytes, void* stream) {
    if (F >= kMaxSum / 2) return NITI_ERR_UNSUPPORTED;
    return linear_backward<true>(dy, lddy, z, ldz, act, a, lda, s_a, s_a_n, b, ldb, s_b, s_b_n, da, ldda, db, lddb, dbias, M, 2 * F, K,
                                 mode, seed, call, type, ws, ws_bytes, stream);
}

}  // extern "C"
