// Device helpers shared by the token mixing kernels.
#pragma once

#include <hip/hip_runtime.h>

#include "mixing.h"

namespace sgemm_emu {

typedef __bf16 bf16_t;
typedef _Float16 f16_t;

// The element types of q, k, v and o; arithmetic is in FP32, results are
// rounded once (to nearest even) when they are stored.
template <class T>
__device__ inline float to_f32(T x) {
    return static_cast<float>(x);
}
template <class T>
__device__ inline T from_f32(float x) {
    return static_cast<T>(x);
}

// N consecutive elements, moved as one access (16 bytes at most).
template <class T, int N>
struct Pack {
    typedef T type __attribute__((ext_vector_type(N)));
};
template <class T>
struct Pack<T, 1> {
    typedef T type;
};

// Rows [first, first + count) of sequence n.  Packed sequences come from the
// device, so they are clamped to the rows there are.
struct Span {
    int64_t first;
    int count;
};

__device__ inline Span span_of(const int* cu, int n, int tokens) {
    if (cu == nullptr) return {(int64_t)n * tokens, tokens};
    const int lo = min(max(cu[n], 0), tokens);
    const int hi = min(max(cu[n + 1], lo), tokens);
    return {lo, hi - lo};
}

// Element (token t of sequence n, head h) of a view; packed sequences count
// their tokens along the one batch there is.
template <class T>
__device__ inline T* row_of(const sgemm_emu_view_t& v, bool packed, int n, const Span& s, int h) {
    T* p = static_cast<T*>(v.p) + h * v.head;
    return p + (packed ? s.first * v.token : n * v.batch);
}

// Smallest log decay that counts: e^-200 and everything below is zero in
// FP32 whatever it multiplies, and running sums of it stay exact enough.
constexpr float kLeastDecay = -200.0f;

// (NaN stays.)
__device__ inline float log_decay(float g) { return g < kLeastDecay ? kLeastDecay : g; }

// Blocks of 256 threads of one launch, which stays below 2^31 threads.
constexpr int64_t kMostBlocks = 1 << 22;

// LDS is shared by the block's waves: orders this wave's accesses to it around
// the barrier, and leaves loads from memory in flight.
__device__ inline void lds_barrier() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// Calls f(T{}) with the element type of a dtype that has been checked.
template <class F>
inline hipError_t by_dtype(int dtype, F&& f) {
    switch (dtype) {
        case SGEMM_EMU_BF16: return f(bf16_t{});
        case SGEMM_EMU_F16: return f(f16_t{});
        default: return f(float{});
    }
}

}  // namespace sgemm_emu
