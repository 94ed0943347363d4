// Gated product of int8 rows: both projections of a feed-forward block, the
// activation and the product in one kernel.
//
//   z[m][n] = s_a[m] s_b[n] sum_k a[m][k] b[n][k] + bias[n],  n < 2 F,   out[m][n] = act(z[m][n]) z[m][F + n]
//
// The kernels are those of the plain product with weight rows paired (see linear_tiles.h): the sums are
// exact in int32, a is read once for both projections, and z reaches memory only where it is asked for.
//
// Measured, bf16 with SiLU (F x K): 1 x 9216 x 4096 14.3 us, 5.3 TB/s of weights; 4096 x 8192 x 4096 with z 280 to 293 us, 1.9
// POPS, bound by power and by the 200 MB that it stores (without z 244, 2.25 POPS); 1000 x 1500 x 1111 in 32 bits 14.7, of which 3 to 5 go to
// copying the rows to whole pieces.
#include "linear_tiles.h"

namespace niti {

namespace {

// What a call takes in each kernel (see the forms), N counting the weight rows; store: what z adds to a round.  Found for the least
// time lost on half of 500 random calls of 1..8192 x 32..9216 x 32..9216 with whole pieces: on the other half what they pick takes
// 0.8% longer than the fastest kernel in the mean, with z 1.9% (with the plain product's constants 1.4% and 2.9%).  Rows at odd addresses
// go by the plain product's, 2.2% from the fastest on 200 calls.  Parts of a sum side by side, as that has them, gained on none of 400 calls
// more than 12%, in the mean nothing.
struct PairCost {
    Cost cost;
    float store;
};
constexpr PairCost kPair12{{16, 32, kSpread, 2.39f, 1.22f, 0.99f, 3.07f}, 0.14f};
constexpr PairCost kPair22{{32, 32, kSpread, 2.46f, 0.74f, 1.16f, 3.04f}, 1.09f};
constexpr PairCost kPairBytes12{{16, 32, kSpread, 2.01f, 0.59f, 1.23f, 2.45f}, 0.f};
constexpr PairCost kPairBytes22{{32, 32, kSpread, 2.02f, 0.86f, 1.39f, 3.48f}, 0.f};
constexpr PairCost kPair64{{64, 128, kTwo, 1.15f, 3.70f, 1.35f, 2.86f}, 0.83f};
constexpr PairCost kPairAny64{{64, 64, kSpread, 2.84f, 1.02f, 3.38f, 4.07f}, 0.f};
constexpr PairCost kPair128{{128, 128, kTwo, 2.84f, 2.72f, 4.16f, 2.62f}, 0.17f};
constexpr PairCost kPairDeep128{{128, 128, kRounds, 1.38f, 3.45f, 4.24f, 0.13f}, 1.91f};
constexpr PairCost kPair256{{256, 256, kRounds, 4.69f, 11.87f, 5.12f, 0.30f}, 1.33f};

struct Choice {
    enum { kS12, kS22, k64, k128, k128d, k256 } kernel;
    float time;
    bool pack;   // the operands are copied to whole aligned pieces first
};

// keep: z is stored as well.
Choice choose(int64_t M, int64_t F, int64_t K, Rows rows, size_t room, bool keep) {
    // columns of whole tiles: a half's last tile is not filled by the other half
    const bool whole = rows == kOfPieces, words = rows != kOfBytes;
    auto at = [&](const PairCost& p) {
        Cost c = p.cost;
        c.round += keep ? p.store : 0.f;
        return cost(c, M, (F + c.bn / 2 - 1) / (c.bn / 2) * c.bn, K);
    };
    Choice c{Choice::kS12, at(words ? kPair12 : kPairBytes12), false};
    auto take = [&](decltype(c.kernel) kernel, float time) {
        if (time < c.time) c = Choice{kernel, time, false};
    };
    take(Choice::kS22, at(words ? kPair22 : kPairBytes22));
    take(Choice::k64, at(whole ? kPair64 : kPairAny64));
    if (whole) {
        take(Choice::k128, at(kPair128));
        // (where tiles outnumber the CUs, two a CU come out a little better than the model has them)
        take(Choice::k128d, at(kPairDeep128) * (M * F > 128 * 128 * 128 ? 1.08f : 1.f));
        take(Choice::k256, at(kPair256));
    }
    const size_t copies = whole ? 0 : pack_bytes(M, 2 * F, K);
    if (copies > 0 && copies <= room) {
        Choice p = choose(M, F, up16(K), kOfPieces, 0, keep);
        p.time += 2.3f + (float)((double)copies * 2. / 3e6);   // (3 TB/s)
        p.pack = true;
        if (p.time < c.time) c = p;
    }
    return c;
}

template <typename T>
hipError_t run_gated(LinArgs A, void* ws, size_t ws_bytes, hipStream_t stream) {
    const bool whole = ring_takes(A);
    // the backward pass reads z much later: more than the L2s hold goes past them (4096 x 8192 x 4096 315 -> 284 us)
    A.z_stream = A.z && A.M * A.N * 2 * (int64_t)sizeof(T) > ((int64_t)32 << 20);
    const Choice c = choose(A.M, A.N, A.K, whole ? kOfPieces : (word_rows(A) ? kOfWords : kOfBytes), ((uintptr_t)ws & 15) == 0 ? ws_bytes : 0, A.z != nullptr);
    if (c.pack) {
        const int64_t Kp = up16(A.K);
        const uint32_t ppr = (uint32_t)(Kp / 16), pieces = (uint32_t)(A.M + 2 * A.N) * ppr;
        hipLaunchKernelGGL(linear_pack_kernel, dim3((pieces + 255) / 256), dim3(256), 0, stream, A, ppr, pieces, (int8_t*)ws);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        LinArgs P = A;
        P.a = (const int8_t*)ws, P.b = P.a + A.M * Kp;
        P.lda = P.ldb = P.K = Kp;
        return run_gated<T>(P, nullptr, 0, stream);
    }
    switch (c.kernel) {
        case Choice::kS12: return run_small<T, 1, 2, true>(A, stream);
        case Choice::kS22: return run_small<T, 2, 2, true>(A, stream);
        case Choice::k64: return whole ? run_ring<T, 64, 128, 3, 2, 2, 128, true>(A, stream) : run_any<T, true>(A, stream);
        case Choice::k128: return run_ring<T, 128, 128, 2, 4, 2, 128, true>(A, stream);
        case Choice::k128d: return run_ring<T, 128, 128, 4, 4, 2, 128, true>(A, stream);
        default: return run_ring<T, 256, 256, 4, 2, 4, 64, true>(A, stream);
    }
}

}  // namespace

// For copies of the operands, if that is how this product would go with room for them.
size_t gated_fwd_workspace(int64_t M, int64_t F, int64_t K) {
    if (M < 1 || F < 1 || K < 1 || M >= kMaxDim || F >= kMaxLd / 2 || K >= kMaxSum) return 0;
    for (Rows rows : {kOfBytes, kOfWords})
        for (bool keep : {false, true})
            if (choose(M, F, K, rows, SIZE_MAX, keep).pack) return pack_bytes(M, 2 * F, K);
    return 0;
}

}  // namespace niti

using namespace niti;

extern "C" {

niti_status niti_gated_fwd(const int8_t* a, int64_t lda, const float* s_a, int64_t s_a_n, const int8_t* b, int64_t ldb, const float* s_b,
                           int64_t s_b_n, const void* bias, int bias_type, int act, void* z, int64_t ldz, void* out, int64_t ldout,
                           int64_t M, int64_t F, int64_t K, int type, void* ws, size_t ws_bytes, void* stream) {
    if (M < 0 || F < 0 || K < 0) return NITI_ERR_SHAPE;
    if (!valid_type(type) || (bias && !valid_type(bias_type)) || act < NITI_ACT_NONE || act > NITI_ACT_SILU) return NITI_ERR_ARG;
    if (M >= kMaxDim || F >= kMaxLd / 2 || K >= kMaxSum) return NITI_ERR_UNSUPPORTED;
    if (M == 0 || F == 0) return NITI_OK;
    if (!s_a || !s_b || !out || (K > 0 && (!a || !b))) return NITI_ERR_NULL;
    if ((s_a_n != 1 && s_a_n != M) || (s_b_n != 1 && s_b_n != 2 * F)) return NITI_ERR_SHAPE;
    if (bad_ld(M > 1 ? lda : K, K, false) || bad_ld(ldb, K, false) || (z && bad_ld(M > 1 ? ldz : 2 * F, 2 * F, true)) ||
        bad_ld(M > 1 ? ldout : F, F, true))
        return NITI_ERR_SHAPE;
    if (ws_bytes > 0 && !ws) return NITI_ERR_WORKSPACE;
    LinArgs A{a, b, s_a, s_b, bias, nullptr, z, out, M > 1 ? lda : K, ldb, 0, ldz, ldout, M, F, K, s_a_n == 1 ? 0 : 1, s_b_n == 1 ? 0 : 1,
              bias_type, act, 0, 0, 0};
    // Very many rows go in slabs, so that a launch stays below 2^32 threads.
    const int64_t size = (int64_t)type_size(type), tn = (F + 31) / 32;
    int64_t slab = ((int64_t)1 << 22) / tn * 64;
    if (slab < 64) slab = 64;
    for (int64_t left = M; left > 0; left -= slab) {
        A.M = left < slab ? left : slab;
        const hipError_t e = by_type(type, [&](auto t) { return run_gated<decltype(t)>(A, ws, ws_bytes, (hipStream_t)stream); });
        if (e != hipSuccess) return NITI_ERR_HIP;
        A.a += slab * A.lda;
        if (A.a_step) A.s_a += slab;
        if (A.z) A.z = (char*)A.z + slab * A.ldz * size;
        A.out = (char*)A.out + slab * A.ldout * size;
    }
    return NITI_OK;
}

}  // extern "C"
