// AdamW over many tensors at once.
//
//   m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2,
//   p = p (1 - lr wd) - lr / (1 - b1^t) * m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// Every element is read and written once, so memory bounds it: 28 bytes an
// element with p, g, m, v in 32 bits, 14 with 8-bit states and g in 16 (62 M such
// elements: 164 us, 5.3 TB/s, and 70 us for reading their states as bf16, 5.3 TB/s;
// 61 thousand with 32-bit states 4.2 us, which is a launch).  The
// tensors of a call share launches: the table of their addresses travels in
// the kernel's arguments (no copy to the device, nothing to keep alive), a
// workgroup finds the tensor of its chunk by comparing its index with all
// starts at once, one per lane.
//
// 8-bit states.  256 consecutive elements share a scale.  A thread holds 8
// consecutive elements, half a wave a block, so that a block's maximum is a
// reduction over 32 lanes and its codes are written by the threads that hold
// the values.  The codes are those of sqrt|m| and v^(1/4): relative steps stay
// below 2 / c and 4 / c down to small values, where a linear code would lose
// them.  Code 0 for a v above 0 would make the next step divide by the new
// gradient alone; such a v keeps code 1.
#include "scaled.h"

namespace niti {

namespace {

constexpr int kTensors = 48;       // of a launch: their table has to fit the kernel's arguments
constexpr int kBlock = 256;        // elements of a scale
constexpr int PT = 8;              // elements of a thread
constexpr int kThreads = 256;
constexpr int kChunk = PT * kThreads;
constexpr int64_t kMaxChunks = (int64_t)1 << 22;   // of a launch

struct Entry {
    void* p;
    const void* g;
    void* m;
    void* v;
    float* ms;
    float* vs;
    int64_t n;
    int64_t block0;   // blocks before this tensor in the call
};

struct Step {
    float b1, c1, b2, c2;   // decay rates and 1 - rate
    float keep;             // 1 - lr * weight_decay
    float lr;               // lr / (1 - b1^t)
    float root;             // 1 / sqrt(1 - b2^t)
    float eps;
    const float* gscale;
    uint64_t seed;
    uint32_t call;
    int sr;
    int exact;              // eps is too small for the hardware's roots and reciprocals as they are
};

struct Table {
    Entry e[kTensors];
    int32_t start[kTensors];   // first chunk of each tensor; past the last one, 2^31 - 1
    Step s;
};
static_assert(sizeof(Table) <= 4096 - 64, "kernel arguments");

// Index of the tensor that chunk c belongs to: starts are ascending.
__device__ __forceinline__ int find_tensor(const int32_t* start, int c) {
    const int lane = threadIdx.x & 63;
    const bool before = lane < kTensors && start[lane < kTensors ? lane : 0] <= c;
    return __builtin_amdgcn_readfirstlane(__popcll(__ballot(before)) - 1);
}

// Maximum over the 32 lanes of a half wave.
__device__ __forceinline__ uint32_t half_max(uint32_t v) {
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o, kWave));
    return v;
}

// Scale and factor of a block's codes from its largest magnitude.
struct BlockScale {
    float scale;   // top * unit; 0 below 2^-100, NaN for a block that is not finite
    float inv;     // 1 / top, or 0
};
__device__ __forceinline__ BlockScale block_scale(uint32_t top_bits, float unit) {
    const float top = __uint_as_float(top_bits);
    BlockScale b;
    if (top_bits >= kInfBits) return BlockScale{__uint_as_float(0x7FC00000u), 0.f};
    if (top < kTopMin) return BlockScale{0.f, 0.f};
    b.scale = top * unit;
    b.inv = 1.f / top;
    return b;
}

// Square roots and reciprocals are the hardware's, good to one unit in the last
// place; the IEEE sequences around them took as long as the memory traffic.  They
// take a value below the normal range for zero: a root of at most 2^-63, which is
// below half a unit of an eps of 2^-36 / sqrt(1 - b2^t) or more.  With a smaller eps (Step::exact)
// small values are scaled up first by powers of two, which loses nothing: gradients below 1e-17
// have such v, and with eps = 0 nothing else is in the divisor.  For every eps that took
// 6 us more of the 163 of a step with 8-bit states.  (The codes' roots need no such care: what is
// that much smaller than its block's largest has code 0, or 1, either way.)
__device__ __forceinline__ float root_ratio(float m, float v, float root, float eps) {
    return m * __builtin_amdgcn_rcpf(__builtin_amdgcn_sqrtf(v) * root + eps);
}
__device__ __forceinline__ float root_ratio_exact(float m, float v, float root, float eps) {
    const bool low = v < 0x1p-100f;
    const float d = __builtin_amdgcn_sqrtf(low ? v * 0x1p60f : v) * (low ? 0x1p-30f : 1.f) * root + eps;
    const bool tiny = d < 0x1p-60f;
    const float r = __builtin_amdgcn_rcpf(tiny ? d * 0x1p64f : d);
    return m * r * (tiny ? 0x1p64f : 1.f);
}
constexpr float kUnitM = 1.f / 16129.f;                       // 1 / 127^2
constexpr float kUnitV = 1.f / (255.f * 255.f * 255.f * 255.f);   // 1 / 255^4

// A thread's elements i .. i + PT - 1 of a tensor.  FULL: all of the chunk's are
// there, and no load is in a branch, where it would be waited for.
template <typename TP, typename TG, int BITS, bool FULL>
__device__ __forceinline__ void adamw_elements(const Entry& E, const Step& S, int64_t i) {
    const int64_t left = E.n - i;
    const int n = FULL || left >= PT ? PT : (left > 0 ? (int)left : 0);
    const float gs = S.gscale ? *S.gscale : 1.f;
    float p[PT], g[PT], m[PT], v[PT];
    load_some((const TP*)E.p + i, n, p);
    load_some((const TG*)E.g + i, n, g);
    if constexpr (BITS == 32) {
        load_some((const float*)E.m + i, n, m);
        load_some((const float*)E.v + i, n, v);
    } else {
        int8_t cm[PT] = {};
        uint8_t cv[PT] = {};
        float ms = 0.f, vs = 0.f;
        if (FULL || n == PT) {
            __builtin_memcpy(cm, (const int8_t*)E.m + i, PT);
            __builtin_memcpy(cv, (const uint8_t*)E.v + i, PT);
        } else {
#pragma unroll
            for (int e = 0; e < PT; e++)
                if (e < n) cm[e] = ((const int8_t*)E.m)[i + e], cv[e] = ((const uint8_t*)E.v)[i + e];
        }
        if (FULL || n > 0) ms = E.ms[i / kBlock], vs = E.vs[i / kBlock];
#pragma unroll
        for (int e = 0; e < PT; e++) {
            const float c = (float)cm[e], d = (float)cv[e];
            m[e] = c * fabsf(c) * ms;
            v[e] = (d * d) * (d * d) * vs;
        }
    }
#pragma unroll
    for (int e = 0; e < PT; e++) {
        const float x = g[e] * gs;
        m[e] = S.b1 * m[e] + S.c1 * x;
        v[e] = S.b2 * v[e] + S.c2 * (x * x);
    }
    if (S.exact) {
#pragma unroll
        for (int e = 0; e < PT; e++) p[e] = p[e] * S.keep - S.lr * root_ratio_exact(m[e], v[e], S.root, S.eps);
    } else {
#pragma unroll
        for (int e = 0; e < PT; e++) p[e] = p[e] * S.keep - S.lr * root_ratio(m[e], v[e], S.root, S.eps);
    }
    store_some((TP*)E.p + i, n, p);
    if constexpr (BITS == 32) {
        store_some((float*)E.m + i, n, m);
        store_some((float*)E.v + i, n, v);
    } else {
        uint32_t tm = 0, tv = 0;
#pragma unroll
        for (int e = 0; e < PT; e++)
            if (e < n) tm = max(tm, mag_bits(m[e])), tv = max(tv, mag_bits(v[e]));
        const BlockScale bm = block_scale(half_max(tm), kUnitM), bv = block_scale(half_max(tv), kUnitV);
        int8_t cm[PT];
        uint8_t cv[PT];
        DrawStream draws(S.seed, S.call, ((uint64_t)E.block0 * kBlock + (uint64_t)i) >> 1);   // one for each two elements
#pragma unroll
        for (int e = 0; e < PT; e += 2) {
            uint64_t r = 0;
            if (S.sr) r = draws.next();
#pragma unroll
            for (int o = 0; o < 2; o++) {
                float rm = 127.f * __builtin_amdgcn_sqrtf(fabsf(m[e + o]) * bm.inv);
                float rv = 255.f * __builtin_amdgcn_sqrtf(__builtin_amdgcn_sqrtf(v[e + o] * bv.inv));
                if (S.sr) {
                    const uint32_t w = (uint32_t)(r >> (32 * o));
                    rm = floorf(rm + (float)(w & 0xFFFFu) * 0x1p-16f);
                    rv = floorf(rv + (float)(w >> 16) * 0x1p-16f);
                } else {
                    rm = rintf(rm);
                    rv = rintf(rv);
                }
                rm = bm.inv > 0.f ? fminf(rm, 127.f) : 0.f;
                rv = bv.inv > 0.f && v[e + o] > 0.f ? fminf(fmaxf(rv, 1.f), 255.f) : 0.f;
                cm[e + o] = (int8_t)(int)copysignf(rm, m[e + o]);
                cv[e + o] = (uint8_t)(int)rv;
            }
        }
        if (FULL || n == PT) {
            __builtin_memcpy((int8_t*)E.m + i, cm, PT);
            __builtin_memcpy((uint8_t*)E.v + i, cv, PT);
        } else {
#pragma unroll
            for (int e = 0; e < PT; e++)
                if (e < n) ((int8_t*)E.m)[i + e] = cm[e], ((uint8_t*)E.v)[i + e] = cv[e];
        }
        if ((threadIdx.x & 31) == 0 && (FULL || n > 0)) E.ms[i / kBlock] = bm.scale, E.vs[i / kBlock] = bv.scale;
    }
}

template <typename TP, typename TG, int BITS>
__global__ __launch_bounds__(kThreads) void adamw_kernel(Table tab) {
    const int k = find_tensor(tab.start, blockIdx.x);
    const Entry& E = tab.e[k];
    const int64_t first = (int64_t)((int)blockIdx.x - tab.start[k]) * kChunk;
    if (first + kChunk <= E.n)
        adamw_elements<TP, TG, BITS, true>(E, tab.s, first + threadIdx.x * PT);
    else
        adamw_elements<TP, TG, BITS, false>(E, tab.s, first + threadIdx.x * PT);
}

// Values of 8-bit states: p and g are the outputs for m and v here.
template <typename T, bool FULL>
__device__ __forceinline__ void read_elements(const Entry& E, int64_t i) {
    if (!FULL && i >= E.n) return;
    const int n = FULL ? PT : (int)min((int64_t)PT, E.n - i);
    const float ms = E.ms[i / kBlock], vs = E.vs[i / kBlock];
    int8_t cm[PT] = {};
    uint8_t cv[PT] = {};
    if (FULL || n == PT) {
        __builtin_memcpy(cm, (const int8_t*)E.m + i, PT);
        __builtin_memcpy(cv, (const uint8_t*)E.v + i, PT);
    } else {
#pragma unroll
        for (int e = 0; e < PT; e++)
            if (e < n) cm[e] = ((const int8_t*)E.m)[i + e], cv[e] = ((const uint8_t*)E.v)[i + e];
    }
    float m[PT], v[PT];
#pragma unroll
    for (int e = 0; e < PT; e++) {
        const float c = (float)cm[e], d = (float)cv[e];
        m[e] = c * fabsf(c) * ms;
        v[e] = (d * d) * (d * d) * vs;
    }
    if (E.p) store_some((T*)E.p + i, n, m);
    if (E.g) store_some((T*)const_cast<void*>(E.g) + i, n, v);
}

template <typename T>
__global__ __launch_bounds__(kThreads) void adamw_read_kernel(Table tab) {
    const int k = find_tensor(tab.start, blockIdx.x);
    const Entry& E = tab.e[k];
    const int64_t first = (int64_t)((int)blockIdx.x - tab.start[k]) * kChunk;
    if (first + kChunk <= E.n)
        read_elements<T, true>(E, first + threadIdx.x * PT);
    else
        read_elements<T, false>(E, first + threadIdx.x * PT);
}

// Fills tables with the tensors' pieces and calls launch(table, chunks) for each.
template <typename F>
hipError_t for_tables(const niti_adamw_tensor* t, int64_t count, int bits, int p_size, int g_size, bool read,
                      const Step& step, F launch) {
    Table tab;
    tab.s = step;
    int used = 0;
    int64_t chunks = 0, block0 = 0;
    auto flush = [&]() -> hipError_t {
        if (!used) return hipSuccess;
        for (int i = used; i < kTensors; i++) tab.e[i] = tab.e[0], tab.start[i] = 0x7FFFFFFF;
        const hipError_t e = launch(tab, (unsigned)chunks);
        used = 0;
        chunks = 0;
        return e;
    };
    const int s_size = bits == 8 ? 1 : 4;
    for (int64_t i = 0; i < count; i++) {
        for (int64_t at = 0; at < t[i].n;) {
            if (used == kTensors || chunks >= kMaxChunks) {
                const hipError_t e = flush();
                if (e != hipSuccess) return e;
            }
            const int64_t room = (kMaxChunks - chunks) * kChunk;
            const int64_t n = t[i].n - at < room ? t[i].n - at : room;
            auto off = [&](const void* p, int64_t bytes) { return p ? (void*)((char*)p + bytes) : nullptr; };
            Entry& e = tab.e[used];
            e.p = off(read ? t[i].m_read : t[i].p, at * p_size);
            e.g = off(read ? t[i].v_read : t[i].g, at * g_size);
            e.m = off(t[i].m, at * s_size);
            e.v = off(t[i].v, at * s_size);
            e.ms = (float*)off(t[i].m_scale, at / kBlock * 4);
            e.vs = (float*)off(t[i].v_scale, at / kBlock * 4);
            e.n = n;
            e.block0 = block0 + at / kBlock;
            tab.start[used++] = (int32_t)chunks;
            chunks += (n + kChunk - 1) / kChunk;
            at += n;
        }
        block0 += (t[i].n + kBlock - 1) / kBlock;
    }
    return flush();
}

niti_status check_tensors(const niti_adamw_tensor* t, int64_t count, int bits) {
    if (count < 0) return NITI_ERR_SHAPE;
    if (count > 0 && !t) return NITI_ERR_NULL;
    for (int64_t i = 0; i < count; i++) {
        if (t[i].n < 0) return NITI_ERR_SHAPE;
        if (t[i].n == 0) continue;
        if (!t[i].m || !t[i].v || (bits == 8 && (!t[i].m_scale || !t[i].v_scale))) return NITI_ERR_NULL;
    }
    return NITI_OK;
}

// The step's number, rates and draws are kernel arguments: a graph of it would take that step again and again.
bool capturing(hipStream_t stream) {
    hipStreamCaptureStatus st = hipStreamCaptureStatusNone;
    if (hipStreamIsCapturing(stream, &st) != hipSuccess) {
        (void)hipGetLastError();   // (the launch finds out for itself)
        return false;
    }
    return st != hipStreamCaptureStatusNone;
}

template <typename TP, typename TG>
hipError_t run_step(const niti_adamw_tensor* t, int64_t count, int bits, const Step& s, hipStream_t stream) {
    return for_tables(t, count, bits, sizeof(TP), sizeof(TG), false, s, [&](const Table& tab, unsigned grid) {
        if (bits == 8)
            hipLaunchKernelGGL((adamw_kernel<TP, TG, 8>), dim3(grid), dim3(kThreads), 0, stream, tab);
        else
            hipLaunchKernelGGL((adamw_kernel<TP, TG, 32>), dim3(grid), dim3(kThreads), 0, stream, tab);
        return hipGetLastError();
    });
}

}  // namespace

}  // namespace niti

using namespace niti;

extern "C" {

niti_status niti_adamw_step(const niti_adamw_tensor* tensors, int64_t count, int p_type, int g_type, int state_bits,
                            int64_t step, double lr, double beta1, double beta2, double eps, double weight_decay,
                            const float* grad_scale, niti_round_mode mode, uint64_t seed, void* stream) {
    if (!valid_type(p_type) || !valid_type(g_type) || (state_bits != 8 && state_bits != 32) || step < 1) return NITI_ERR_ARG;
    if (mode != NITI_ROUND_RTN && mode != NITI_ROUND_SR) return NITI_ERR_ARG;
    if (!(beta1 >= 0 && beta1 < 1 && beta2 >= 0 && beta2 < 1 && eps >= 0) || !(lr == lr) || !(weight_decay == weight_decay))
        return NITI_ERR_ARG;
    const niti_status st = check_tensors(tensors, count, state_bits);
    if (st != NITI_OK) return st;
    for (int64_t i = 0; i < count; i++)
        if (tensors[i].n > 0 && (!tensors[i].p || !tensors[i].g)) return NITI_ERR_NULL;
    if (capturing((hipStream_t)stream)) return NITI_ERR_UNSUPPORTED;
    Step s{};
    s.b1 = (float)beta1;
    s.c1 = (float)(1 - beta1);
    s.b2 = (float)beta2;
    s.c2 = (float)(1 - beta2);
    s.keep = (float)(1 - lr * weight_decay);
    s.lr = (float)(lr / (1 - pow(beta1, (double)step)));
    s.root = (float)(1 / sqrt(1 - pow(beta2, (double)step)));
    s.eps = (float)eps;
    s.exact = s.eps < 0x1p-36f * s.root;
    s.gscale = grad_scale;
    s.seed = seed;
    s.call = (uint32_t)step;
    s.sr = state_bits == 8 && mode == NITI_ROUND_SR;
    const hipError_t e = by_type(p_type, [&](auto p) {
        return by_type(g_type, [&](auto g) {
            return run_step<decltype(p), decltype(g)>(tensors, count, state_bits, s, (hipStream_t)stream);
        });
    });
    return e == hipSuccess ? NITI_OK : NITI_ERR_HIP;
}

niti_status niti_adamw_read(const niti_adamw_tensor* tensors, int64_t count, int type, void* stream) {
    if (!valid_type(type)) return NITI_ERR_ARG;
    const niti_status st = check_tensors(tensors, count, 8);
    if (st != NITI_OK) return st;
    const hipError_t e = by_type(type, [&](auto o) {
        using T = decltype(o);
        return for_tables(tensors, count, 8, sizeof(T), sizeof(T), true, Step{}, [&](const Table& tab, unsigned grid) {
            hipLaunchKernelGGL((adamw_read_kernel<T>), dim3(grid), dim3(kThreads), 0, (hipStream_t)stream, tab);
            return hipGetLastError();
        });
    });
    return e == hipSuccess ? NITI_OK : NITI_ERR_HIP;
}

}  // extern "C"
