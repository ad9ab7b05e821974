// Tiles of the attention kernels: 32 x 32 matrix products whose operands come
// from registers or from rows staged in LDS, read along the rows or across them.
//
// One fragment is 16 bytes a lane.  The products sum over blocks of kBlock =
// 2 * 16 / sizeof(T) elements, of which the lane's half of the wave has one
// half, in an order that only has to be the same for both operands:
//   along rows:  elements kBlock/2 * half + 0, 1, ... of the block,
//   across rows: rows 4 half + 0..3 and, for 16-bit types, 8 + 4 half + 0..3.
// The second order is that of an accumulator's registers (register i of a lane is
// row 8 (i / 4) + 4 half + i % 4 of column lane % 32), so that a product's
// result, rounded to the type, is the next product's operand in place.
#pragma once

#include <hip/hip_runtime.h>

#include "mixing.hpp"

namespace sgemm_emu {

typedef float f32x16 __attribute__((ext_vector_type(16)));

template <class T>
constexpr int kPer = 16 / (int)sizeof(T);  // elements of 16 bytes
template <class T>
constexpr int kBlock = 2 * kPer<T>;  // elements that one fragment pair sums over
template <class T>
using Frag = typename Pack<T, kPer<T>>::type;

__device__ inline f32x16 mma(Frag<bf16_t> a, Frag<bf16_t> b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ inline f32x16 mma(Frag<f16_t> a, Frag<f16_t> b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}
__device__ inline f32x16 mma(Frag<float> a, Frag<float> b, f32x16 c) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], b[i], c, 0, 0, 0);
    return c;
}

// Row of register i of an accumulator in this lane.
__device__ inline int acc_row(int i, int half) { return 8 * (i / 4) + 4 * half + i % 4; }

// Block kb of an accumulator's rows as an operand that is summed over them.
template <class T>
__device__ inline Frag<T> operand(const f32x16& x, int kb) {
    Frag<T> f;
#pragma unroll
    for (int j = 0; j < kPer<T>; ++j) f[j] = from_f32<T>(x[kPer<T> * kb + j]);
    return f;
}

// Combines the two lanes that share an accumulator's column (lane and lane ^ 32).
__device__ inline float max_halves(float x) {
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                    false);
    return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}
__device__ inline float sum_halves(float x) {
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                    false);
    return __uint_as_float(p[0]) + __uint_as_float(p[1]);
}

// Rows of D elements in LDS.  The 16-byte chunks of a row are permuted by
// swizzle(row): eight rows read at one chunk, and four rows read at two
// neighbouring ones, are on different banks.
template <class T, int D>
struct Tile {
    static constexpr int kRowBytes = D * (int)sizeof(T);
    static constexpr int kChunks = kRowBytes / 16;

    static __device__ inline int swizzle(int row) { return ((row & 3) << 1) | ((row >> 2) & 1); }
    static __device__ inline int at(int row, int chunk) {
        return row * kRowBytes + ((chunk ^ swizzle(row)) << 4);
    }

    // Block kb of the elements of rows row0 + lane % 32 (row0 a multiple of 8).
    static __device__ inline Frag<T> along(const char* tile, int row0, int kb, int lane) {
        const int half = lane >> 5, row = lane & 31;
        // (chunk bits above the swizzle's three stay an immediate offset)
        const int chunk = 2 * kb + half;
        const int low = ((chunk & 7) ^ swizzle(row)) << 4;
        return *reinterpret_cast<const Frag<T>*>(tile + row * kRowBytes + low + row0 * kRowBytes +
                                                 ((chunk >> 3) << 7));
    }

    // Element d0 + lane % 32 of the rows of block kb (d0 a multiple of 32).
    static __device__ inline Frag<T> across(const char* tile, int kb, int d0, int lane) {
        const int half = lane >> 5;
        if constexpr (sizeof(T) == 2) {
            // a transposing read: 16 lanes bring 4 rows of 16 elements, 8 bytes each, and
            // every lane gets the 4 values of its column
            typedef short Short4 __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) Short4 LdsShort4;
            const int i = lane & 15, row = 4 * half + (i >> 2);
            const int chunk = d0 / 8 + 2 * ((lane >> 4) & 1) + ((i >> 1) & 1);
            const char* p = tile + row * kRowBytes + (((chunk & 7) ^ swizzle(row)) << 4) +
                            8 * (i & 1) + ((chunk >> 3) << 7) + kb * 16 * kRowBytes;
            union {
                Short4 part[2];
                Frag<T> all;
            } u;
            u.part[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsShort4*)p);
            u.part[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsShort4*)(p + 8 * kRowBytes));
            return u.all;
        } else {
            const int d = d0 + (lane & 31), chunk = d / 4;
            Frag<T> f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int row = 4 * half + j;
                f[j] = *reinterpret_cast<const float*>(
                    tile + kb * 8 * kRowBytes + row * kRowBytes +
                    (((chunk & 7) ^ swizzle(row)) << 4) + ((chunk >> 3) << 7) + 4 * (d & 3));
            }
            return f;
        }
    }
};

// `size` elements of a row, from chunk c on, zero behind them.  kVec: rows are
// 16-byte aligned and size a multiple of kPer.
template <class T, bool kVec>
__device__ inline Frag<T> load_chunk(const T* row, int c, int size, bool inside) {
    Frag<T> f;
#pragma unroll
    for (int j = 0; j < kPer<T>; ++j) f[j] = from_f32<T>(0.0f);
    if constexpr (kVec) {
        if (inside && c * kPer<T> < size) f = *reinterpret_cast<const Frag<T>*>(row + c * kPer<T>);
    } else {
#pragma unroll
        for (int j = 0; j < kPer<T>; ++j)
            if (inside && c * kPer<T> + j < size) f[j] = row[c * kPer<T> + j];
    }
    return f;
}

// kRows rows of a head on their way to LDS through registers of kThreads threads:
// loaded a tile ahead, written when the tile's place is free.
template <class T, int D, int kRows, int kThreads, bool kVec>
struct Staged {
    static constexpr int kChunks = Tile<T, D>::kChunks;
    static constexpr int kEach = kRows * kChunks / kThreads;
    static_assert(kEach * kThreads == kRows * kChunks && kThreads % kChunks == 0, "");
    Frag<T> f[kEach];

    // Rows first to first + kRows - 1 of p; zeros from row `end` on.
    __device__ inline void load(const T* p, int64_t token, int first, int end, int size, int thread) {
        const int c = thread % kChunks, r0 = thread / kChunks;
        const T* base = p + (int64_t)first * token;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int r = r0 + i * (kThreads / kChunks);
            f[i] = load_chunk<T, kVec>(base + (int)(r * (int)token), c, size, first + r < end);
        }
    }
    __device__ inline void store(char* tile, int thread) const {
        const int c = thread % kChunks, r0 = thread / kChunks;
#pragma unroll
        for (int i = 0; i < kEach; ++i)
            *reinterpret_cast<Frag<T>*>(tile + Tile<T, D>::at(r0 + i * (kThreads / kChunks), c)) = f[i];
    }
    // Puts zeros in the place of values that are not finite; whether there were any.
    __device__ inline bool clear_not_finite() {
        bool any = false;
#pragma unroll
        for (int i = 0; i < kEach; ++i)
#pragma unroll
            for (int j = 0; j < kPer<T>; ++j) {
                const float x = to_f32(f[i][j]);
                const bool bad = !(__builtin_fabsf(x) < __builtin_inff());
                any |= bad;
                if (bad) f[i][j] = from_f32<T>(0.0f);
            }
        return any;
    }
};

// Four neighbouring elements of an output row; kVec: rows are aligned to four
// elements and size a multiple of four.
template <class T, bool kVec>
__device__ inline void store_four(T* row, int d, int size, float a, float b, float c, float e) {
    if constexpr (kVec) {
        if (d < size) {
            typename Pack<T, 4>::type v;
            v[0] = from_f32<T>(a), v[1] = from_f32<T>(b), v[2] = from_f32<T>(c),
            v[3] = from_f32<T>(e);
            *reinterpret_cast<typename Pack<T, 4>::type*>(row + d) = v;
        }
    } else {
        const float x[4] = {a, b, c, e};
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (d + j < size) row[d + j] = from_f32<T>(x[j]);
    }
}

}  // namespace sgemm_emu
