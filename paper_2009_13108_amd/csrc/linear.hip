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
#include "linear_tiles.h"

namespace niti {

namespace {

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
// What a product takes in each kernel is modelled by the forms of linear_tiles.h.
// Small tiles give every CU work and split the sum, large ones load less for each
// product; 128 x 128 tiles have a ring of four stages, one a CU, which a
// CU with one tile needs to cover a load's latency (800 x 2880 x 3712, 161 tiles: 25.9 ->
// 19.4 us), or of two, two tiles a CU (2048 x 4096 x 4096: 44 us, 48 with four).  Fitted to
// 500 random products of 1..8192 x 32..9216 x 32..9216 timed with each kernel;
// what the model picks takes 1.4% longer than the fastest of these seven in the
// mean, on 250 others 1.8%; 64 x 64 tiles alone 33% and 36%.
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

struct Choice {
    enum { kS11, kS12, kS22, k64, k128, k128d, k256 } kernel;
    int parts;       // of the sum
    int64_t klen;    // products of a part, whole steps
    float time;
    bool pack;       // the operands are copied to whole aligned pieces first
};

constexpr int64_t kPartLen = 512;   // least products of a part
inline int64_t part_ld(int64_t N) { return (N + 7) / 8 * 8; }

// rows: what the operands' rows are made of, aligned; room: bytes of workspace.
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
