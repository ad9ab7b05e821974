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

// FP32 as two FP16 parts, hi = fp16(x s) and lo = fp16(x s - hi), s a power of two for each row
// that brings its largest element to [2^14, 2^15): 22 bits of an element down to 2^-18 of
// that.  A product takes three on the matrix instructions, lo lo being below FP32's rounding;
// in tiles the parts are planes, one behind the other.
struct split_t {};

template <class T>
struct FormOf {
    typedef T Elem;  // of tiles and operands
    typedef T Out;   // of the caller's tensors
    static constexpr int kPlanes = 1;
};
template <>
struct FormOf<split_t> {
    typedef f16_t Elem;
    typedef float Out;
    static constexpr int kPlanes = 2;
};
template <class T>
using Elem = typename FormOf<T>::Elem;
template <class T>
using Out = typename FormOf<T>::Out;
template <class T>
constexpr int kPlanes = FormOf<T>::kPlanes;

// Elements of a row's place in a tile, and of a plane's row in memory.
template <int D>
constexpr int kWidth = D <= 64 ? 64 : 128;

template <class T>
struct Operand {
    Frag<Elem<T>> p[kPlanes<T>];
};

template <class T>
__device__ inline f32x16 mma(const Operand<T>& a, const Operand<T>& b, f32x16 c) {
    if constexpr (kPlanes<T> == 2) {
        c = mma(a.p[1], b.p[0], c);
        c = mma(a.p[0], b.p[1], c);
    }
    return mma(a.p[0], b.p[0], c);
}

// Row of register i of an accumulator in this lane.
__device__ inline int acc_row(int i, int half) { return 8 * (i / 4) + 4 * half + i % 4; }

// Block kb of an accumulator's rows as an operand that is summed over them.
template <class T>
__device__ inline Operand<T> operand(const f32x16& x, int kb) {
    typedef Elem<T> E;
    Operand<T> f;
#pragma unroll
    for (int j = 0; j < kPer<E>; ++j) {
        const float y = x[kPer<E> * kb + j];
        f.p[0][j] = from_f32<E>(y);
        if constexpr (kPlanes<T> == 2) f.p[1][j] = from_f32<E>(y - to_f32(f.p[0][j]));
    }
    return f;
}

// 1 / x of a power of two x, 2^-126 to 2^126.
__device__ inline float inverse_of_power(float x) {
    return __uint_as_float(0x7f000000u - __float_as_uint(x));
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

// The largest magnitude of an accumulator's column (NaN does not count).
__device__ inline float largest(const f32x16& x) {
    float most = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) most = fmaxf(most, __builtin_fabsf(x[i]));
    return max_halves(most);
}

__device__ inline f32x16 times(const f32x16& x, float f) {
    f32x16 y;
#pragma unroll
    for (int i = 0; i < 16; ++i) y[i] = x[i] * f;
    return y;
}

// A column's power of two, for weights that become FP16 operands.
struct Fit {
    static constexpr int kMostBits = 127 + 126;  // so that its inverse is normal, too
    float f = 0x1p126f;

    // So that |x| f stays below 2^15 for the column's x, of magnitudes up to `most`; what is
    // summed so far is rescaled where f changes.
    template <int N>
    __device__ inline void fit(float most, f32x16 (&sum)[N]) {
        const bool over = most * f > 0x1p15f;
        if (__any(over)) {
            // 2^10 <= most f < 2^11
            const int e = (int)(__float_as_uint(most) >> 23);
            const float to =
                over ? __uint_as_float((unsigned)max(min(264 - e, kMostBits), 1) << 23) : f;
            const float by = to / f;
#pragma unroll
            for (int d = 0; d < N; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) sum[d][i] *= by;
            f = to;
        }
    }

    // The x so far have been made smaller by 2^-fall (fall >= 0): f may rise by as much.
    // Returns log2 of what it rose by.
    __device__ inline float rise(float fall) {
        const int room = kMostBits - (int)(__float_as_uint(f) >> 23);
        const int by = min((int)fminf(fall, 300.0f), room);
        f = __uint_as_float(__float_as_uint(f) + ((unsigned)by << 23));
        return (float)by;
    }
};

// Address of LDS as the instructions take it.
__device__ inline uint32_t lds_address(const void* p) {
    return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)p;
}

// Rows of up to D elements in LDS, 64 or 128 apart.  The 16-byte chunks of a row are
// permuted by swizzle(row), so that what the 64 banks serve at a time is on all of them: 16
// rows at one chunk, or 4 rows at four neighbouring ones.
template <class T, int D>
struct Tile {
    static constexpr int kRowBytes = kWidth<D> * (int)sizeof(T);
    static constexpr int kChunks = kRowBytes / 16;
    static constexpr int kMask = kChunks == 8 ? 7 : 15;  // chunk bits that are permuted
    static constexpr int kPlain = kChunks == 8 ? 3 : 4;  // how many

    static __device__ inline int swizzle(int row) {
        if (kChunks == 8) return (row >> 1 & 1) << 2 | (row >> 2 & 3);
        return (row & 3) << 2 | (row >> 2 & 3);
    }
    static __device__ inline int at(int row, int chunk) {
        return row * kRowBytes + ((chunk ^ swizzle(row)) << 4);
    }

    // What a lane's reads have in common: along(base(tile, from_along(lane)), ...).  The
    // chunk's bits are added without carry, so that the permutation goes through.
    static __device__ inline int from_along(int lane) { return at(lane & 31, lane >> 5); }
    static __device__ inline int from_across(int lane) {
        const int half = lane >> 5, i = lane & 15;
        if (sizeof(T) == 2)
            return at(4 * half + (i >> 2), 2 * (lane >> 4 & 1) + (i >> 1 & 1)) + 8 * (i & 1);
        return at(4 * half, (lane & 31) >> 2) + 4 * (lane & 3);
    }
    static __device__ inline uint32_t base(const char* tile, int from) {
        return lds_address(tile) + from;
    }
    // A chunk further on in a row (where it adds to bits that are zero so far).
    static __device__ inline uint32_t chunk_on(uint32_t at, int chunk) {
        return (at ^ ((chunk & kMask) << 4)) + (chunk >> kPlain << (kPlain + 4));
    }

    // Block kb of the elements of rows row0 + lane % 32 (row0 a multiple of 32).
    static __device__ inline Frag<T> along(uint32_t base, int row0, int kb) {
        typedef __attribute__((address_space(3))) const Frag<T> Lds;
        return *(Lds*)(uintptr_t)(chunk_on(base, 2 * kb) + row0 * kRowBytes);
    }

    // Two transposing reads of a 16-bit type: 16 lanes bring 4 rows of 16 elements, 8 bytes
    // each, and every lane gets the 4 values of its column.
    static __device__ inline Frag<T> across_at(uint32_t first, uint32_t second) {
        typedef short Short4 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) Short4 Lds;
        union {
            Short4 part[2];
            Frag<T> all;
        } u;
        u.part[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds*)(uintptr_t)first);
        u.part[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds*)(uintptr_t)second);
        return u.all;
    }

    // Element d0 + lane % 32 of the rows of block kb (d0 a multiple of 32).
    static __device__ inline Frag<T> across(uint32_t base, int kb, int d0) {
        if constexpr (sizeof(T) == 2) {
            const uint32_t p = chunk_on(base, d0 / 8) + kb * 16 * kRowBytes;
            return across_at(p, (p ^ swizzle(8) << 4) + 8 * kRowBytes);
        } else {
            typedef __attribute__((address_space(3))) const float Lds;
            const uint32_t p = chunk_on(base, d0 / 4) + (kb >> 1) * 16 * kRowBytes;
            Frag<T> f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int row = (kb & 1) * 8 + j;
                f[j] = *(Lds*)(uintptr_t)((p ^ swizzle(row) << 4) + row * kRowBytes);
            }
            return f;
        }
    }
};

// A lane's addresses for reads of tiles that lie `offset` bytes behind a place in LDS, an
// immediate of the instructions where it is constant.
template <class E, int D>
struct Reader {
    using One = Tile<E, D>;
    uint32_t a[D / kBlock<E>], c[D / 32][2];
    __device__ inline Reader(const char* lds, int lane) {
        const uint32_t x = One::base(lds, One::from_along(lane));
        const uint32_t y = One::base(lds, One::from_across(lane));
#pragma unroll
        for (int kb = 0; kb < D / kBlock<E>; ++kb) a[kb] = One::chunk_on(x, 2 * kb);
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt) {
            c[dt][0] = One::chunk_on(y, 4 * dt);
            c[dt][1] = (c[dt][0] ^ One::swizzle(8) << 4) + 8 * One::kRowBytes;
        }
    }
    // Blocks as Tile's, of rows from the offset on.
    __device__ inline Frag<E> along(int offset, int kb) const {
        typedef __attribute__((address_space(3))) const Frag<E> Lds;
        return *(Lds*)(uintptr_t)(a[kb] + offset);
    }
    __device__ inline Frag<E> across(int offset, int kb, int dt) const {
        return One::across_at(c[dt][0] + offset + kb * 16 * One::kRowBytes,
                              c[dt][1] + offset + kb * 16 * One::kRowBytes);
    }
};
// (FP32 forms them when it reads: eight for each 32 elements across are too many)
template <int D>
struct Reader<float, D> {
    using One = Tile<float, D>;
    uint32_t x, y;
    __device__ inline Reader(const char* lds, int lane)
        : x(One::base(lds, One::from_along(lane))), y(One::base(lds, One::from_across(lane))) {}
    __device__ inline Frag<float> along(int offset, int kb) const {
        return One::along(x + offset, 0, kb);
    }
    __device__ inline Frag<float> across(int offset, int kb, int dt) const {
        return One::across(y + offset, kb, 32 * dt);
    }
};

// The planes of a tile of kRows rows.
template <class T, int D, int kRows>
struct Planes {
    using One = Tile<Elem<T>, D>;
    static constexpr int kPlaneBytes = kRows * One::kRowBytes, kBytes = kPlanes<T> * kPlaneBytes;

    static __device__ inline Operand<T> along(uint32_t base, int row0, int kb) {
        Operand<T> f;
#pragma unroll
        for (int i = 0; i < kPlanes<T>; ++i) f.p[i] = One::along(base + i * kPlaneBytes, row0, kb);
        return f;
    }
    static __device__ inline Operand<T> across(uint32_t base, int kb, int d0) {
        Operand<T> f;
#pragma unroll
        for (int i = 0; i < kPlanes<T>; ++i) f.p[i] = One::across(base + i * kPlaneBytes, kb, d0);
        return f;
    }
    // From a tile `offset` bytes behind the reader's place.
    typedef Reader<Elem<T>, D> Read;
    static __device__ inline Operand<T> along(const Read& r, int offset, int kb) {
        Operand<T> f;
#pragma unroll
        for (int i = 0; i < kPlanes<T>; ++i) f.p[i] = r.along(offset + i * kPlaneBytes, kb);
        return f;
    }
    static __device__ inline Operand<T> across(const Read& r, int offset, int kb, int dt) {
        Operand<T> f;
#pragma unroll
        for (int i = 0; i < kPlanes<T>; ++i) f.p[i] = r.across(offset + i * kPlaneBytes, kb, dt);
        return f;
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

// Chunk c of a row's planes, which are kWidth apart (and whole: zero behind the size).
template <class T, int D, bool kVec>
__device__ inline Operand<T> load_operand(const Elem<T>* row, int c, int size, bool inside) {
    Operand<T> f;
    if constexpr (kPlanes<T> == 1) {
        f.p[0] = load_chunk<T, kVec>(row, c, size, inside);
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            f.p[i] = load_chunk<Elem<T>, true>(row + i * kWidth<D>, c, kWidth<D>, inside);
    }
    return f;
}

// kRows rows of a head on their way from memory to a tile, moved by kThreads threads.
//   rows(f): f(r) is the distance in bytes of row r from the first address
//   start(tile, first, there): the loads of those rows, by their number, that there(i, r) says
//     are there; `first` is the same for all lanes, i the thread's chunk, r its row
//   finish(tile): the rows are there, for this thread's part; a barrier makes it all of them
// kVec: straight from memory to LDS, 16 bytes a lane (4 x 4096 tokens forward 573 us, through
// registers 640); rows that are not there, and what a
// tile holds behind `size` elements, are left as they were.  Else through registers, an
// element at a time, with zeros in their place.
template <class T, int D, int kRows, int kThreads, bool kVec>
struct Flow {
    using To = Tile<T, D>;
    static constexpr int kChunks = To::kChunks;
    static constexpr int kEach = kRows * kChunks / kThreads;
    static constexpr int kRowsApart = kThreads / kChunks;
    static_assert(kEach * kThreads == kRows * kChunks && kRowsApart * kChunks == kThreads, "");
    Frag<T> f[kVec ? 1 : kEach];
    uint32_t off[kEach];

    // Row of the thread's first chunk; number of a chunk in its row.
    static __device__ inline int row(int thread) { return thread / kChunks; }
    static __device__ inline int chunk(int thread, int i) {
        return (thread % kChunks) ^ To::swizzle(row(thread) + i * kRowsApart);
    }

    template <class Distance>
    __device__ inline void rows(Distance distance, int thread) {
#pragma unroll
        for (int i = 0; i < kEach; ++i)
            off[i] = distance(row(thread) + i * kRowsApart) + (kVec ? 16 * chunk(thread, i) : 0);
    }

    template <class There>
    __device__ inline void start(char* tile, const T* first, int size, int thread, There there) {
        const uint32_t at = __builtin_amdgcn_readfirstlane(lds_address(tile) + thread / 64 * 1024);
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int c = chunk(thread, i);
            const bool in = there(i, row(thread) + i * kRowsApart);
            if constexpr (kVec) {
                // (the instruction adds 16 times the lane's number to m0; the builtin would
                // make every later LDS read wait for it, whatever it reads)
                if (in && c * kPer<T> < size)
                    asm volatile(
                        "s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off[i]),
                        "s"(first), "s"(at + i * kThreads * 16)
                        : "m0", "memory");
            } else {
                f[i] = load_chunk<T, false>(
                    reinterpret_cast<const T*>(reinterpret_cast<const char*>(first) + off[i]), c, size,
                    in);
            }
        }
    }
    __device__ inline void finish(char* tile, int thread) {
        if constexpr (kVec) {
            // (and this wave is through with what it read before from the places written next)
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        } else {
#pragma unroll
            for (int i = 0; i < kEach; ++i)
                *reinterpret_cast<Frag<T>*>(tile + (thread + i * kThreads) * 16) = f[i];
        }
    }
    // Puts zeros in the place of values that are not finite in the thread's part of a tile;
    // whether there were any in rows that are there.
    template <class There>
    static __device__ inline bool clear_not_finite(char* tile, int thread, There there) {
        bool any = false;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            Frag<T>* at = reinterpret_cast<Frag<T>*>(tile + (thread + i * kThreads) * 16);
            Frag<T> x = *at;
            bool here = false;
#pragma unroll
            for (int j = 0; j < kPer<T>; ++j) {
                const bool bad = !(__builtin_fabsf(to_f32(x[j])) < __builtin_inff());
                here |= bad;
                if (bad) x[j] = from_f32<T>(0.0f);
            }
            if (here) *at = x;
            any |= here && there(i, row(thread) + i * kRowsApart);
        }
        return any;
    }
};

// Zeros in `bytes` of LDS (a multiple of 16).
__device__ inline void clear_lds(char* p, int bytes, int thread, int threads) {
    for (int at = thread * 16; at < bytes; at += threads * 16)
        *reinterpret_cast<Pack<float, 4>::type*>(p + at) = Pack<float, 4>::type{};
}

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
