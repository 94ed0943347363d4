// Internal interface of the product of int8 rows (linear.hip), which its
// backward pass (linear_bwd.hip) calls too, and the workspaces of the row-wise operators.
#pragma once

#include "scaled.h"

#include <atomic>

namespace niti {

struct LinArgs {
    const int8_t* a;     // [M][K]
    const int8_t* b;     // [N][K]; of a gated product [2 N][K], and s_b, bias and z's columns likewise
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
    int32_t z_stream;         // z goes past the caches (set by the gated product)
};

hipError_t linear_run(const LinArgs& a, int type, void* ws, size_t ws_bytes, hipStream_t stream);
// Both, in one launch where that pays.
hipError_t linear_run_pair(const LinArgs& a, const LinArgs& b, int type, void* ws, size_t ws_bytes, hipStream_t stream);
size_t linear_fwd_workspace(int64_t M, int64_t N, int64_t K);
size_t linear_bwd_workspace(int64_t M, int64_t N, int64_t K);
size_t rmsnorm_bwd_workspace(int64_t M, int64_t D);
size_t gated_fwd_workspace(int64_t M, int64_t F, int64_t K);
size_t gated_bwd_workspace(int64_t M, int64_t F, int64_t K);
size_t embedding_bwd_workspace(int64_t M, int64_t V, int64_t D);
size_t logprobs_workspace(int64_t M, int64_t V, int64_t top);
size_t distill_workspace(int64_t M, int64_t V);

// Arrays of a workspace begin at multiples of 256 bytes.
inline size_t up256(size_t v) { return (v + 255) / 256 * 256; }

// Once for each kernel and device, from any thread: it may have more than 64 KiB of LDS.
template <auto kernel, int LDS>
inline hipError_t allow_lds() {
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

}  // namespace niti
