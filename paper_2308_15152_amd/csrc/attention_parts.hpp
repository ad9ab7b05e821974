// Attention whose keys are cut into parts that are computed at the same time: each leaves a
// row's normalized result and log-sum in the workspace, and a second kernel joins them:
//   o = sum_p 2^(log_p - z) part_p / sum_p 2^(log_p - z),  z the largest log.
#pragma once

#include "attention_rows.hpp"
#include "attention_tile.hpp"

namespace sgemm_emu {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;
// The reference of a row that has seen nothing: below all scores, but 2^(kLeast - kLeast) is one.
constexpr float kLeast = -3e38f;

// Elements from one row of a part to the next.
template <int D>
constexpr int kPartStride = D <= 64 ? 64 : 128;
inline int part_stride(int size) { return size <= 64 ? 64 : 128; }

struct Parts {
    float* o;     // [part][row][kPartStride], or null: there is one part, which is the result
    float* logs;  // [part][row], base 2; -infinity: nothing was seen, and o is not written
    int64_t rows;  // tokens in all x query heads
};

inline int64_t parts_bytes(int64_t parts, int64_t rows, int size) {
    return (parts * rows * (part_stride(size) + 1) * 4 + 255) / 256 * 256;
}
inline Parts parts_in(void* workspace, int64_t parts, int64_t rows, int size) {
    if (parts == 1) return {nullptr, nullptr, rows};
    float* o = static_cast<float*>(workspace);
    return {o, o + parts * rows * part_stride(size), rows};
}

// Where a pass leaves a row.
// (T: the results' type)
template <class T, bool kVec>
struct RowOut {
    T* o;
    float* lse;   // natural, or null
    float* part;  // its row, or null
    float* log;
    int size;
    bool skip = false;

    // l, z: the row's sum and its reference; `here`: the lane that stores what belongs to the row.
    __device__ inline void sums(float l, float z, bool here) {
        const float log = l == 0.0f ? -__builtin_inff() : z + __builtin_amdgcn_logf(l);
        if (part != nullptr) {
            if (here) *this->log = log;
            skip = l == 0.0f;
        } else if (here && lse != nullptr) {
            *lse = log * kLn2;
        }
    }
    __device__ inline void four(int d, float x, float y, float z, float w) const {
        if (part == nullptr)
            store_four<T, kVec>(o, d, size, x, y, z, w);
        else if (d < size && !skip)
            *reinterpret_cast<Pack<float, 4>::type*>(part + d) = Pack<float, 4>::type{x, y, z, w};
    }
};

template <class T, int D, bool kVec>
__device__ inline RowOut<T, kVec> row_out(const Parts& p, int part, int64_t row, T* o, float* lse,
                                          int size) {
    return {o, lse, p.o ? p.o + (part * p.rows + row) * kPartStride<D> : nullptr,
            p.logs + part * p.rows + row, size};
}

constexpr int kJoinThreads = 256;

struct JoinArgs {
    Parts parts;
    sgemm_emu_view_t o, lse;  // lse.p may be null
    int count, tokens, q_heads, size;
    const int* slots;  // a sequence whose slot is outside [0, n_slots) has zeros; or null
    int n_slots;
};

// A row's elements are 16 or 32 lanes of four, in `groups` (a power of two up to 8) that take
// every groups-th part and are joined in LDS: few rows of many parts would otherwise wait for
// one load after another (256 rows of 32 parts: 20 us with one group, 5 with eight).
template <class T, int D, bool kVec>
__global__ __launch_bounds__(kJoinThreads) void attention_join_kernel(JoinArgs a, int groups,
                                                                      int first_block) {
    typedef Pack<float, 4>::type Four;
    constexpr int kEach = kPartStride<D> / 4;
    __shared__ Four xs[kJoinThreads];
    __shared__ float ls[kJoinThreads], zs[kJoinThreads];
    const int thread = threadIdx.x, rows = kJoinThreads / kEach / groups;
    const int in_row = thread % kEach, group = thread / kEach % groups;
    const int64_t row = (int64_t)(first_block + (int)blockIdx.x) * rows + thread / kEach / groups;
    const int d = in_row * 4;
    const bool here = row < a.parts.rows && d < a.size;
    const int64_t token = here ? row / a.q_heads : 0;
    const int h = (int)(row - token * a.q_heads), n = (int)(token / a.tokens);
    float z = kLeast, l = 0.0f;
    Four x{};
    const int slot = a.slots == nullptr ? 0 : a.slots[n];
    if (here && (a.slots == nullptr || (slot >= 0 && slot < a.n_slots))) {
#pragma unroll 4
        for (int p = group; p < a.count; p += groups) {
            const float log = a.parts.logs[p * a.parts.rows + row];
            Four y = *reinterpret_cast<const Four*>(
                a.parts.o + (p * a.parts.rows + row) * kPartStride<D> + d);
            if (log == -__builtin_inff()) y = Four{};  // (not written)
            const float to = fmaxf(z, log);
            const float f = __builtin_amdgcn_exp2f(z - to), g = __builtin_amdgcn_exp2f(log - to);
            l = l * f + g;
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = x[j] * f + y[j] * g;
            z = to;
        }
    }
    if (groups > 1) {
        xs[thread] = x, ls[thread] = l, zs[thread] = z;
        __syncthreads();
        if (group > 0) return;
        const float mine = z;
        for (int g = 1; g < groups; ++g) z = fmaxf(z, zs[thread + g * kEach]);
        const float f = __builtin_amdgcn_exp2f(mine - z);
        l *= f;
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] *= f;
        for (int g = 1; g < groups; ++g) {
            const float by = __builtin_amdgcn_exp2f(zs[thread + g * kEach] - z);
            const Four y = xs[thread + g * kEach];
            l += by * ls[thread + g * kEach];
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] += by * y[j];
        }
    }
    if (!here) return;
    const float f = l == 0.0f ? 0.0f : 1.0f / l;
    const int64_t t = token - (int64_t)n * a.tokens;
    T* o = static_cast<T*>(a.o.p) + n * a.o.batch + t * a.o.token + h * a.o.head;
    store_four<T, kVec>(o, d, a.size, x[0] * f, x[1] * f, x[2] * f, x[3] * f);
    if (d == 0 && a.lse.p != nullptr)
        static_cast<float*>(a.lse.p)[n * a.lse.batch + t * a.lse.token + h * a.lse.head] =
            l == 0.0f ? -__builtin_inff() : (z + __builtin_amdgcn_logf(l)) * kLn2;
}

template <class T, int D, bool kVec>
hipError_t launch_join(const JoinArgs& a, hipStream_t stream) {
    int groups = 1;
    while (groups < 8 && groups * 2 <= a.count) groups *= 2;
    const int rows = kJoinThreads / (kPartStride<D> / 4) / groups;
    return launch_blocks(attention_join_kernel<T, D, kVec>, (a.parts.rows + rows - 1) / rows,
                         kJoinThreads, stream, a, groups);
}

}  // namespace sgemm_emu
