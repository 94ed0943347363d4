// Internal interface of the product of int8 rows (linear.hip), which its
// backward pass (linear_bwd.hip) calls too.
#pragma once

#include "scaled.h"

namespace niti {

struct LinArgs {
    const int8_t* a;     // [M][K]
    const int8_t* b;     // [N][K]
    const float* s_a;    // scale of row m at s_a[m * a_step]; NULL: 1
    const float* s_b;
    const void* bias;    // [N] or NULL
    const void* res;     // [M][N] or NULL
    void* z;             // [M][N] or NULL
    void* out;           // [M][N]
    int64_t lda, ldb, ldres, ldz, ldout;
    int64_t M, N, K;
    int32_t a_step, b_step;   // 1, or 0 for one scale
    int32_t bias_type, act;
    // Set by linear_run:
    int32_t res_dma;          // the residual's rows are whole aligned pieces within 32-bit offsets
    int32_t klen;             // products of one part of a split sum (blockIdx.y), or 0
    int64_t part;             // elements of a part's sums, from out on
};

hipError_t linear_run(const LinArgs& a, int type, void* ws, size_t ws_bytes, hipStream_t stream);
// Both, in one launch where that pays.
hipError_t linear_run_pair(const LinArgs& a, const LinArgs& b, int type, void* ws, size_t ws_bytes, hipStream_t stream);
size_t linear_fwd_workspace(int64_t M, int64_t N, int64_t K);
size_t linear_bwd_workspace(int64_t M, int64_t N, int64_t K);
size_t rmsnorm_bwd_workspace(int64_t M, int64_t D);

}  // namespace niti
