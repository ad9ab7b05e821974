// Which rows the blocks of the attention kernels take, and their dispatch.
#pragma once

#include "attention.h"
#include "mixing.hpp"

namespace sgemm_emu {

// Part `tile` (of `rows` rows) of sequence n.
struct Place {
    int n, tile;
    bool found;
};

// The index-th part of packed sequences of which each is cut into parts of `per` rows,
// a token being `group` rows.  Every wave scans the bounds for itself, 64 sequences at a
// time; the result is the same in all lanes.
__device__ inline Place find_part(const int* cu, int batch, int tokens, int group, int per,
                                  int index) {
    const int lane = threadIdx.x & 63;
    for (int base = 0; base < batch; base += 64) {
        int parts = 0;
        if (base + lane < batch) {
            const Span s = span_of(cu, base + lane, tokens);
            parts = (int)(((int64_t)s.count * group + per - 1) / per);
        }
        int upto = parts;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int x = __shfl_up(upto, d);
            if (lane >= d) upto += x;
        }
        const uint64_t after = __ballot(upto > index);
        if (after != 0) {
            const int at = __builtin_ctzll(after);
            const int before = __shfl(upto, at) - __shfl(parts, at);
            return {__builtin_amdgcn_readfirstlane(base + at),
                    __builtin_amdgcn_readfirstlane(index - before), true};
        }
        index -= __shfl(upto, 63);
    }
    return {0, 0, false};
}

// Parts of `per` rows that sequences of `tokens` tokens have at most in all.
inline int64_t most_parts(int batch, int64_t rows, int per, bool packed) {
    if (!packed) return (rows + per - 1) / per * batch;
    return rows / per + batch;
}

// Whether every row of a view starts at a multiple of 16 bytes.
inline bool rows_aligned16(const sgemm_emu_view_t& v, int elem) {
    const int64_t n = 16 / elem;
    return (uintptr_t)v.p % 16 == 0 && v.batch % n == 0 && v.token % n == 0 && v.head % n == 0;
}

// Launches `blocks` blocks (below 2^31) of a kernel that takes the number of its first block
// last.
template <class Kernel, class... Args>
inline hipError_t launch_blocks(Kernel kernel, int64_t blocks, int threads, hipStream_t stream,
                                const Args&... args) {
    constexpr int64_t kMost = 1 << 21;  // below 2^31 threads
    for (int64_t first = 0; first < blocks; first += kMost) {
        const unsigned n = (unsigned)(blocks - first < kMost ? blocks - first : kMost);
        hipLaunchKernelGGL(kernel, dim3(n), dim3(threads), 0, stream, args..., (int)first);
        if (hipError_t e = hipGetLastError()) return e;
    }
    return hipSuccess;
}

template <int N>
struct Number {
    static constexpr int value = N;
};

// Calls f(T{}, Number<padded size>, Number<rows move as vectors>), T one of the types or F32 in
// the place of FP32.
template <class F32, class F>
inline hipError_t by_form(int dtype, int size, bool vec, F&& f) {
    const auto with = [&](auto t) {
        const auto and_with = [&](auto d) {
            return vec ? f(t, d, Number<1>{}) : f(t, d, Number<0>{});
        };
        return size <= 64 ? and_with(Number<64>{})
                          : size <= 96 ? and_with(Number<96>{}) : and_with(Number<128>{});
    };
    switch (dtype) {
        case SGEMM_EMU_BF16: return with(bf16_t{});
        case SGEMM_EMU_F16: return with(f16_t{});
        default: return with(F32{});
    }
}

}  // namespace sgemm_emu
