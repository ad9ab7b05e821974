// Device pieces of the chunk kernels of the gated delta rule.
//
// Products are emulated FP32 on v_mfma_f32_16x16x32_f16: an operand is hi +
// lo, hi = fp16(x 2^e), lo = fp16(x 2^e - hi), with one power of two per row
// of A or column of B that brings the largest magnitude into [2^14, 2^15).  lo
// needs no scale of its own there (hi and lo share the accumulator), values
// down to 2^-15 of the largest keep 22 bits and smaller ones an absolute 2^-39
// of it, and inputs of any FP32 magnitude are represented.  The powers are
// taken out of the FP32 result, whose rows and columns are A's rows and B's
// columns.  bfloat16 and float16 inputs are exact with hi alone.
//
// Where the result of one product is the B operand of the next, it stays in
// registers: lane l of the accumulator holds rows 4 (l / 16) + 0..3 of column
// l % 16, and two stacked tiles give that lane the 8 contraction entries of a
// 32-step if the A operand lists its columns in the same order:
//   slot i of lane group g  <->  column 16 (i / 4) + 4 g + i % 4 of the step.
// All A fragments here are in that order.
#pragma once

#include "delta.h"
#include "mfmae/frag.hpp"
#include "mixing.hpp"

namespace sgemm_emu {

using mfmae::half8_t;
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 half4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kC = kDeltaChunk;

// hi (and lo) of one operand fragment.
template <int N>
struct Frag {
    half8_t part[N];
};

__device__ inline f32x4 mfma(half8_t a, half8_t b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// c += a b; lo.lo is left out (2^-22 of the product) unless kAll.
template <bool kAll = false, int NA, int NB>
__device__ inline f32x4 multiply(const Frag<NA>& a, const Frag<NB>& b, f32x4 c) {
    if (kAll && NA == 2 && NB == 2) c = mfma(a.part[NA - 1], b.part[NB - 1], c);
    if (NA == 2) c = mfma(a.part[NA - 1], b.part[0], c);
    if (NB == 2) c = mfma(a.part[0], b.part[NB - 1], c);
    return mfma(a.part[0], b.part[0], c);
}

// A power of two and its inverse.
struct Scale {
    float up, down;
};

// The one that brings m >= 0 into [2^14, 2^15), within 2^-112 <= m; infinity and
// NaN keep a finite one.
__device__ inline Scale scale_of(float m) {
    const int e = max((int)(__builtin_bit_cast(uint32_t, m) >> 23), 15);
    return {__builtin_bit_cast(float, (uint32_t)(268 - e) << 23),
            __builtin_bit_cast(float, (uint32_t)(e - 14) << 23)};
}

// Largest of the four lanes l % 16 + 16 g.  (The elements go through scalars:
// a bit cast of a vector's element reads element 0 whichever is named.)
__device__ inline float max_groups(float m) {
    uint32_t u = __builtin_bit_cast(uint32_t, m);
    const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    const uint32_t a0 = a[0], a1 = a[1];
    m = fmaxf(__builtin_bit_cast(float, a0), __builtin_bit_cast(float, a1));
    u = __builtin_bit_cast(uint32_t, m);
    const auto b = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    const uint32_t b0 = b[0], b1 = b[1];
    return fmaxf(__builtin_bit_cast(float, b0), __builtin_bit_cast(float, b1));
}

// N parts of eight values times a power of two.
template <int N>
__device__ inline Frag<N> split(const float (&x)[8], float up) {
    Frag<N> f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        f.part[0][i] = (_Float16)(x[i] * up);
        if (N == 2)
            f.part[N - 1][i] = (_Float16)__builtin_fmaf(x[i], up, -(float)f.part[0][i]);
    }
    return f;
}

// The B fragment of two stacked accumulator tiles.
template <int N>
__device__ inline Frag<N> split(f32x4 a, f32x4 b, float up) {
    const float x[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    return split<N>(x, up);
}

template <int N>
__device__ inline float largest(const f32x4 (&x)[N]) {
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) m = fmaxf(m, fabsf(x[i][r]));
    return m;
}

// Number of a triangular matrix's fragment: lower ones fill steps 0 .. i / 2 of
// tile i, upper ones steps i / 2 .. 1.
__device__ constexpr int lower_at(int tile, int step) { return tile < 2 ? tile : 2 * tile - 2 + step; }
__device__ constexpr int upper_at(int tile, int step) { return tile < 2 ? 2 * tile + step : tile + 2; }

// Chunk c of a call: its sequence, the chunk's number in it, first row and
// rows of the chunk; count <= 0 if there is no such chunk.
struct Place {
    int n;
    Span span;
    int first, count;
};

__device__ inline int chunk_base(const int* cu, int n, int tokens) {
    return min(max(cu[n], 0), tokens) / kC + n;
}

__device__ inline Place place_of(const int* cu, int c, int batch, int tokens) {
    Place p;
    int j;
    if (cu == nullptr) {
        const int each = (tokens + kC - 1) / kC;
        p.n = c / each;
        j = c - p.n * each;
    } else {  // the last sequence whose chunks start at c or before, 64 at a time
        int lo = 0, len = batch;
        while (len > 1) {
            const int step = (len + 63) / 64;
            const int i = lo + (int)(threadIdx.x & 63) * step;
            const bool at = i < lo + len && chunk_base(cu, i, tokens) <= c;
            const int k = max(__popcll(__ballot(at)) - 1, 0);
            len = min(step, len - k * step);
            lo += k * step;
        }
        p.n = lo;
        j = c - chunk_base(cu, lo, tokens);
    }
    p.span = span_of(cu, p.n, tokens);
    p.first = j * kC;
    p.count = j < 0 ? 0 : min(kC, p.span.count - p.first);
    return p;
}

// Eight consecutive elements of a row, from element e on; zero at `size` and
// after, and everywhere if !in.
template <class T>
struct Eight {
    T x[8];
};

template <class T>
__device__ inline Eight<T> load_eight(const T* row, int e, int size, bool in, bool wide) {
    Eight<T> v;
    if (wide) {  // size is a multiple of 8, the row 16-byte aligned
        u32x4 w[sizeof(T) / 2] = {};
        if (in && e < size)
#pragma unroll
            for (int i = 0; i < (int)sizeof(T) / 2; ++i)
                w[i] = reinterpret_cast<const u32x4*>(row + e)[i];
        __builtin_memcpy(&v, w, sizeof(v));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v.x[i] = in && e + i < size ? row[e + i] : from_f32<T>(0.0f);
    }
    return v;
}

// The 8 k-values of a lane as MFMA operand, in the type of the input or, for
// FP32, split.
template <class T>
struct Operand;
template <>
struct Operand<bf16_t> {
    typedef __bf16 vec __attribute__((ext_vector_type(8)));
    vec v;
    __device__ void set(const Eight<bf16_t>& x, float) { __builtin_memcpy(&v, &x, 16); }
};
template <>
struct Operand<f16_t> {
    half8_t v;
    __device__ void set(const Eight<f16_t>& x, float) { __builtin_memcpy(&v, &x, 16); }
};
template <>
struct Operand<float> {
    Frag<2> v;
    __device__ void set(const Eight<float>& x, float up) { v = split<2>(x.x, up); }
};
__device__ inline f32x4 product(const Operand<bf16_t>& a, const Operand<bf16_t>& b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v, b.v, c, 0, 0, 0);
}
__device__ inline f32x4 product(const Operand<f16_t>& a, const Operand<f16_t>& b, f32x4 c) {
    return mfma(a.v, b.v, c);
}
__device__ inline f32x4 product(const Operand<float>& a, const Operand<float>& b, f32x4 c) {
    return multiply(a.v, b.v, c);
}

// Parts of an input element as operand.
template <class T>
constexpr int kPartsOf = sizeof(T) == 4 ? 2 : 1;

// Rows of K or Q as fragments.  A thread takes 4 tokens x 8 elements: as rows
// (A operand of products with S) two 8-byte pieces a token, as columns (A
// operand of products that contract over tokens) 8 pieces of 4 tokens.  Lanes
// of a fragment are permuted by its number, which spreads the pieces that
// a wave writes at once over the banks.
template <class T, int kK>
struct Unit {
    Eight<T> x[4];

    __device__ void load(const T* rows, int64_t stride, int unit, int count, int size, bool wide) {
        const int e = 8 * (unit % (kK / 8)), t = 4 * (unit / (kK / 8));
#pragma unroll
        for (int i = 0; i < 4; ++i)
            x[i] = load_eight(rows + (t + i) * stride, e, size, t + i < count, wide);
    }

    // scale: of the four tokens
    template <bool kRowsToo, bool kColumns>
    __device__ void store(char* rows, char* columns, int unit, f32x4 scale) const {
        constexpr int kParts = kPartsOf<T>, kSteps = kK / 32;
        const int eight = unit % (kK / 8), four = unit / (kK / 8);
        half4_t part[kParts][4][2];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float v = to_f32(x[i].x[e]);
                const _Float16 hi = (_Float16)(v * scale[i]);
                part[0][i][e / 4][e % 4] = hi;
                if (kParts == 2)
                    part[kParts - 1][i][e / 4][e % 4] =
                        (_Float16)__builtin_fmaf(v, scale[i], -(float)hi);
            }
        if (kRowsToo) {
            const int step = eight / 4, half = (eight % 4) / 2, g = 2 * (eight % 2);
#pragma unroll
            for (int p = 0; p < kParts; ++p) {
                char* to = rows + ((p * 4 + four / 4) * kSteps + step) * 1024 + half * 8;
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        const int lane = (g + b) * 16 + 4 * (four % 4) + i;
                        *reinterpret_cast<half4_t*>(to + (lane ^ (step & 3)) * 16) = part[p][i][b];
                    }
            }
        }
        if (kColumns) {
            const int tile = eight / 2, step = four / 8, half = (four / 4) % 2, g = four % 4;
#pragma unroll
            for (int p = 0; p < kParts; ++p) {
                char* to = columns + ((p * (kK / 16) + tile) * 2 + step) * 1024 + half * 8;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int lane = g * 16 + 8 * (eight % 2) + e;
                    half4_t v;
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[i] = part[p][i][e / 4][e % 4];
                    *reinterpret_cast<half4_t*>(to + (lane ^ (tile & 7)) * 16) = v;
                }
            }
        }
    }
};

template <class T, int kK>
__device__ inline Frag<kPartsOf<T>> row_fragment(const char* rows, int tile, int step,
                                                              int lane) {
    constexpr int kParts = kPartsOf<T>;
    Frag<kParts> f;
#pragma unroll
    for (int p = 0; p < kParts; ++p)
        f.part[p] = *reinterpret_cast<const half8_t*>(
            rows + ((p * 4 + tile) * (kK / 32) + step) * 1024 + (lane ^ (step & 3)) * 16);
    return f;
}

template <class T, int kK>
__device__ inline Frag<kPartsOf<T>> column_fragment(const char* columns, int tile,
                                                                 int step, int lane) {
    constexpr int kParts = kPartsOf<T>;
    Frag<kParts> f;
#pragma unroll
    for (int p = 0; p < kParts; ++p)
        f.part[p] = *reinterpret_cast<const half8_t*>(
            columns + ((p * (kK / 16) + tile) * 2 + step) * 1024 + (lane ^ (tile & 7)) * 16);
    return f;
}

template <int N>
__device__ inline Frag<N> matrix_fragment(const char* matrix, int at, int lane) {
    Frag<N> f;
#pragma unroll
    for (int p = 0; p < N; ++p)
        f.part[p] =
            *reinterpret_cast<const half8_t*>(matrix + (p * 6 + at) * 1024 + lane * 16);
    return f;
}

}  // namespace sgemm_emu
