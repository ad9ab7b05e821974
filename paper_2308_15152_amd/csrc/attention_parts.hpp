// Attention whose keys are cut into parts that are computed at the same time: each leaves a
// row's normalized result and log-sum in the workspace, and a second kernel joins them:
//   o = sum_p 2^(log_p - z) part_p / sum_p 2^(log_p - z),  z the largest log.
#pragma once

#include "attention_rows.hpp"
#include "attention_tile.hpp"

namespace sgemm_emu {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

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

template <class T, int D, bool kVec>
__global__ __launch_bounds__(kJoinThreads) void attention_join_kernel(JoinArgs a, int first_block) {
    constexpr int kEach = kPartStride<D> / 4;
    const int64_t row = (int64_t)(first_block + (int)blockIdx.x) * (kJoinThreads / kEach) +
                        threadIdx.x / kEach;
    const int d = (int)threadIdx.x % kEach * 4;
    if (row >= a.parts.rows || d >= a.size) return;
    const int64_t token = row / a.q_heads;
    const int h = (int)(row - token * a.q_heads), n = (int)(token / a.tokens);
    float z = -1e30f, l = 0.0f;
    for (int p = 0; p < a.count; ++p) z = fmaxf(z, a.parts.logs[p * a.parts.rows + row]);
    Pack<float, 4>::type x{};
    const int slot = a.slots == nullptr ? 0 : a.slots[n];
    if (a.slots == nullptr || (slot >= 0 && slot < a.n_slots)) {
        for (int p = 0; p < a.count; ++p) {
            const float log = a.parts.logs[p * a.parts.rows + row];
            if (log == -__builtin_inff()) continue;
            const float f = __builtin_amdgcn_exp2f(log - z);
            l += f;
            const auto y = *reinterpret_cast<const Pack<float, 4>::type*>(
                a.parts.o + (p * a.parts.rows + row) * kPartStride<D> + d);
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] += f * y[j];
        }
    }
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
    constexpr int kRows = kJoinThreads / (kPartStride<D> / 4);
    return launch_blocks(attention_join_kernel<T, D, kVec>, (a.parts.rows + kRows - 1) / kRows,
                         kJoinThreads, stream, a);
}

}  // namespace sgemm_emu
