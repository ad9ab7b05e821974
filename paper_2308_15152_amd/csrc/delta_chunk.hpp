// Device pieces of the chunk kernels of the gated delta rule.
//
// Products are emulated FP32 on v_mfma_f32_16x16x32_f16: an operand is hi +
// lo, hi = fp16(x 2^e), lo = fp16(x 2^e - hi), with one power of two per row
// of A or column of B that brings the largest magnitude into [2^14, 2^15).  lo
// needs no scale of its own there (hi and lo share the accumulator), values
// down to 2^-15 of the largest keep 22 bits and smaller ones an absolute 2^-39
// of it, and inputs of any FP32 magnitude are represented.  The powers are
// taken out of the FP32 result, whose rows and columns are A's rows and B's
// columns.  Inputs of 16 bits have hi alone: float16 ones are exact, bfloat16 ones down to
// 2^-32 of their row's largest (below, to an absolute 2^-39 of it).
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
    for (int i = 0; i < 8; ++i) f.part[0][i] = (_Float16)(x[i] * up);
    if (N == 2) {
        // hi as it is packed (the compiler would make every one a second time)
        u32x4 hi = __builtin_bit_cast(u32x4, f.part[0]);
        asm("" : "+v"(hi));
        f.part[0] = __builtin_bit_cast(half8_t, hi);
#pragma unroll
        for (int i = 0; i < 8; ++i)
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

// A value that is not finite may reach later tokens of its chunk but no earlier
// ones, and a product with a triangular matrix would take it to all (0 NaN).
// So such a product's operand is looked at first: the rows of a column
// from the first such value on are left out and give NaN afterwards.  The
// check is the maximum that the scale needs anyway, taken so that NaN stays.
__device__ inline float max_nan(float a, float b) { return __builtin_elementwise_maximum(a, b); }

__device__ inline float column_largest(const f32x4 (&x)[4]) {
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) m = max_nan(m, fabsf(x[i][r]));
    uint32_t u = __builtin_bit_cast(uint32_t, m);
    const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    const uint32_t a0 = a[0], a1 = a[1];
    u = __builtin_bit_cast(uint32_t, max_nan(__builtin_bit_cast(float, a0), __builtin_bit_cast(float, a1)));
    const auto b = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    const uint32_t b0 = b[0], b1 = b[1];
    return max_nan(__builtin_bit_cast(float, b0), __builtin_bit_cast(float, b1));
}

__device__ inline bool finite(float x) { return fabsf(x) < __builtin_inff(); }

// x, of which the compiler keeps nothing ready: in code that hardly ever runs, row numbers
// made before a loop would take registers from all that does.
__device__ inline int fresh(int x) {
    asm volatile("" : "+v"(x));
    return x;
}

// The first row of this lane's column (kC if none) with a value that is not
// finite; it and the rows after it become zero, m the largest of those left.
__device__ inline int cut_column(f32x4 (&x)[4], float& m) {
    const int g = (threadIdx.x & 63) >> 4;
    int first = kC;
#pragma unroll
    for (int i = 3; i >= 0; --i)
#pragma unroll
        for (int r = 3; r >= 0; --r)
            if (!finite(x[i][r])) first = 16 * i + 4 * g + r;
    first = min(first, __shfl_xor(first, 16, 64));
    first = min(first, __shfl_xor(first, 32, 64));
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (16 * i + 4 * g + r >= first) x[i][r] = 0.0f;
    m = column_largest(x);
    return first;
}

// The same where values reach earlier tokens and no later ones (the way back): the rows up
// to the last such value become zero.  The first row after them (0 if there is none).
__device__ inline int cut_column_back(f32x4 (&x)[4], float& m) {
    const int g = fresh((threadIdx.x & 63) >> 4);
    int first = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (!finite(x[i][r])) first = 16 * i + 4 * g + r + 1;
    first = max(first, __shfl_xor(first, 16, 64));
    first = max(first, __shfl_xor(first, 32, 64));
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (16 * i + 4 * g + r < first) x[i][r] = 0.0f;
    m = column_largest(x);
    return first;
}

// Number of a triangular matrix's fragment: lower ones fill steps 0 .. i / 2 of
// tile i, upper ones steps i / 2 .. 1.
__device__ constexpr int lower_at(int tile, int step) { return tile < 2 ? tile : 2 * tile - 2 + step; }
__device__ constexpr int upper_at(int tile, int step) { return tile < 2 ? 2 * tile + step : tile + 2; }

__device__ inline int chunk_base(const int* cu, int n, int tokens) {
    return min(max(cu[n], 0), tokens) / kC + n;
}

// A walk over one sequence or one of its parts: chunks [first, first + count)
// of sequence n, numbered from base in the call; parts: all of the sequence's.
struct Walk {
    int n;
    Span span;
    int base, first, count, part, parts;
};

__device__ inline int part_base(const DeltaChunks& p, int n) {
    return chunk_base(p.cu_seqlens, n, p.tokens) / p.part_chunks + n;
}

// Walk `index`: a sequence, or a part; count <= 0 if there is no such part.
__device__ inline Walk walk_of(const DeltaChunks& p, int index) {
    Walk w{};
    const int each = (p.tokens + kC - 1) / kC;
    if (p.part_chunks == 0) {
        w.n = index;
        w.parts = 1;
    } else if (p.cu_seqlens == nullptr) {
        w.parts = (each + p.part_chunks - 1) / p.part_chunks;
        w.n = index / w.parts;
        w.part = index - w.n * w.parts;
    } else {  // the last sequence whose parts start at index or before
        int lo = 0, len = p.batch;
        while (len > 1) {
            const int step = (len + 63) / 64;
            const int i = lo + (int)(threadIdx.x & 63) * step;
            const bool at = i < lo + len && part_base(p, i) <= index;
            const int k = max(__popcll(__ballot(at)) - 1, 0);
            len = min(step, len - k * step);
            lo += k * step;
        }
        w.n = __builtin_amdgcn_readfirstlane(lo);
        w.part = index - part_base(p, w.n);
    }
    w.span = span_of(p.cu_seqlens, w.n, p.tokens);
    w.base = p.cu_seqlens ? chunk_base(p.cu_seqlens, w.n, p.tokens) : w.n * each;
    const int chunks = (w.span.count + kC - 1) / kC;
    w.count = chunks;
    if (p.part_chunks != 0) {
        // a sequence without tokens has one part, without chunks
        w.parts = max((chunks + p.part_chunks - 1) / p.part_chunks, 1);
        w.first = w.part * p.part_chunks;
        w.count = w.part < 0 || w.part >= w.parts ? -1 : min(p.part_chunks, chunks - w.first);
    }
    return w;
}

// Block -> (walk and value head, slice of columns).  The slices of a head read
// the same K, Q, T and P: they go to one XCD (blocks are dealt out to the 8 in
// turn), and consecutive heads to different ones, so that sequences of different
// lengths spread over all.  The grid is walk_blocks(); task >= tasks: nothing to do.
struct WalkTask {
    int task, slice;
};

__device__ inline WalkTask walk_task(int slices) {
    const int xcd = blockIdx.x & 7, i = blockIdx.x >> 3;
    return {i / slices * 8 + xcd, i % slices};
}
// Whether a walk takes 16 columns a block rather than 32: where those leave half of
// the CUs idle (the walk back of 32 heads of 128 x 128: 128 blocks 227 us, 256
// blocks 213; with more heads than that K and Q would be brought twice as often for nothing).
inline bool narrow(const DeltaChunks& a) {
    const int64_t walks = a.part_chunks > 0 ? a.parts : a.batch;
    return walks * a.v_heads * ((a.v_size + 31) / 32) <= 128;
}
inline int64_t walk_blocks(int64_t tasks, int64_t slices) { return (tasks + 7) / 8 * 8 * slices; }

// Chunk c of a call: its sequence, the chunk's number in it, first row and
// rows of the chunk; count <= 0 if there is no such chunk.
struct Place {
    int n;
    Span span;
    int first, count;
};

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

// Buffer descriptor of everything from p on: offsets below 2^31 are inside
// what the caller may read or write, and kPastEnd is not: loads there return
// zero, stores are dropped.
constexpr uint32_t kPastEnd = 0x80000000;

__device__ inline __amdgpu_buffer_rsrc_t buffer_at(const void* p) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, 0x7fffffff, 0x00020000);
}
template <int kBytes>
struct Word;
template <>
struct Word<2> {
    typedef uint16_t type;
    __device__ static type load(__amdgpu_buffer_rsrc_t r, uint32_t at) {
        return __builtin_amdgcn_raw_buffer_load_b16(r, at, 0, 0);
    }
    __device__ static void store(type v, __amdgpu_buffer_rsrc_t r, uint32_t at) {
        __builtin_amdgcn_raw_buffer_store_b16(v, r, at, 0, 0);
    }
};
template <>
struct Word<4> {
    typedef uint32_t type;
    __device__ static type load(__amdgpu_buffer_rsrc_t r, uint32_t at) {
        return __builtin_amdgcn_raw_buffer_load_b32(r, at, 0, 0);
    }
    __device__ static void store(type v, __amdgpu_buffer_rsrc_t r, uint32_t at) {
        __builtin_amdgcn_raw_buffer_store_b32(v, r, at, 0, 0);
    }
};
template <class T>
__device__ inline T load_word(__amdgpu_buffer_rsrc_t r, uint32_t at) {
    return __builtin_bit_cast(T, Word<sizeof(T)>::load(r, at));
}
template <class T>
__device__ inline void store_word(T v, __amdgpu_buffer_rsrc_t r, uint32_t at) {
    Word<sizeof(T)>::store(__builtin_bit_cast(typename Word<sizeof(T)>::type, v), r, at);
}

// Eight consecutive elements of a row.
template <class T>
struct Eight {
    T x[8];
};

// Elements e ... e + 7 of the row that starts at byte `row` of r; zero at `size`
// and after, and everywhere if !in.
template <class T>
__device__ inline Eight<T> load_eight(__amdgpu_buffer_rsrc_t r, uint32_t row, int e, int size,
                                      bool in, bool wide) {
    Eight<T> v;
    const uint32_t at = row + e * (uint32_t)sizeof(T);
    if (wide) {  // size is a multiple of 8, the row 16-byte aligned
        u32x4 w[sizeof(T) / 2];
        const uint32_t off = in && e < size ? at : kPastEnd;
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i)
            w[i] = __builtin_amdgcn_raw_buffer_load_b128(r, off + 16 * i, 0, 0);
        __builtin_memcpy(&v, w, sizeof(v));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v.x[i] = load_word<T>(r, in && e + i < size ? at + i * (uint32_t)sizeof(T) : kPastEnd);
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

// Place of lane l's 16 bytes in the fragment of step `step` of K's or Q's rows.
// The permutation spreads over the banks what a wave writes at once (pieces of
// 8 bytes, Unit below) and keeps its reads of 16 bytes a lane apart: the LDS takes
// those 16 lanes at a time, 0-3 with 12-15 and 20-27 and so on, so the lanes of
// group 1 may move by 0 or 12, and of group 3 from group 2's place by 0 or 12.
// (Counted: no conflicts in either; reads as columns use half of the banks, since a
// tile is one of the two pieces of every slot.)
__device__ inline int slot(int lane, int step) {
    return (lane ^ (step & 3) ^ ((lane >> 4 & 1) * 12) ^ ((lane >> 5) * 4)) * 16;
}

// Rows of K or Q as fragments in LDS.  A thread takes 4 tokens x 8 elements, in
// two 8-byte pieces a token.
template <class T, int kK>
struct Unit {
    static constexpr int kUnits = 16 * kK / 8;  // of a chunk
    Eight<T> x[4];

    // rows: of the chunk's first token
    __device__ void load(const T* rows, int64_t stride, int unit, int count, int size, bool wide) {
        const int e = 8 * (unit % (kK / 8)), t = 4 * (unit / (kK / 8));
        const __amdgpu_buffer_rsrc_t r = buffer_at(rows);
        const uint32_t step = (uint32_t)stride * sizeof(T);
        if (wide) {
            uint32_t at = e < size ? t * step + e * (uint32_t)sizeof(T) : kPastEnd;
#pragma unroll
            for (int i = 0; i < 4; ++i, at += step) {  // past the end stays past it
                const uint32_t off = count == kC || t + i < count ? at : kPastEnd;
                u32x4 w[sizeof(T) / 2];
#pragma unroll
                for (int n = 0; n < (int)sizeof(T) / 2; ++n)
                    w[n] = __builtin_amdgcn_raw_buffer_load_b128(r, off + 16 * n, 0, 0);
                __builtin_memcpy(&x[i], w, sizeof(w));
            }
        } else {
#pragma unroll 1
            for (int i = 0; i < 4; ++i) {
                Eight<T> y;
#pragma unroll
                for (int n = 0; n < 8; ++n)
                    y.x[n] = load_word<T>(r, t + i < count && e + n < size
                                                 ? (t + i) * step + (e + n) * (uint32_t)sizeof(T)
                                                 : kPastEnd);
#pragma unroll
                for (int n = 0; n < 4; ++n)
                    if (n == i) x[n] = y;
            }
        }
    }

    // scale: of the four tokens (float16 is taken as it is)
    __device__ void store(char* rows, int unit, f32x4 scale) const {
        constexpr int kParts = kPartsOf<T>, kSteps = kK / 32;
        const int eight = unit % (kK / 8), four = unit / (kK / 8);
        const int step = eight / 4, half = (eight % 4) / 2, g = 2 * (eight % 2);
        char* to = rows + ((four / 4) * kSteps + step) * 1024 + half * 8;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            half4_t part[kParts][2];
            if (__is_same(T, f16_t)) {
                __builtin_memcpy(part, &x[i], 16);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float v = to_f32(x[i].x[e]);
                    const _Float16 hi = (_Float16)(v * scale[i]);
                    part[0][e / 4][e % 4] = hi;
                    if (kParts == 2)
                        part[kParts - 1][e / 4][e % 4] =
                            (_Float16)__builtin_fmaf(v, scale[i], -(float)hi);
                }
            }
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const int at = slot((g + b) * 16 + 4 * (four % 4) + i, step);
#pragma unroll
                for (int p = 0; p < kParts; ++p)
                    *reinterpret_cast<half4_t*>(to + p * 4 * kSteps * 1024 + at) = part[p][b];
            }
        }
    }
};

// Token tile `tile`, step `step` of those rows as an operand that contracts
// over elements.
template <class T, int kK>
__device__ inline Frag<kPartsOf<T>> row_fragment(const char* rows, int tile, int step, int lane) {
    Frag<kPartsOf<T>> f;
#pragma unroll
    for (int p = 0; p < kPartsOf<T>; ++p)
        f.part[p] = *reinterpret_cast<const half8_t*>(
            rows + ((p * 4 + tile) * (kK / 32) + step) * 1024 + slot(lane, step));
    return f;
}

// Elements 16 tile ... + 15, tokens of step `step` as an operand that contracts
// over tokens: the same rows, read transposed.  Each group of 16 lanes names
// four tokens' pieces of four elements (lane 4 a + b: token a, piece b) and
// lane n receives element n of the four tokens.
template <class T, int kK>
__device__ inline Frag<kPartsOf<T>> column_fragment(const char* rows, int tile, int step,
                                                    int lane) {
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s16x4* lds_ptr;
    const int from = ((lane & 3) << 4) + ((lane >> 4) << 2) + ((lane >> 2) & 3);
    Frag<kPartsOf<T>> f;
#pragma unroll
    for (int p = 0; p < kPartsOf<T>; ++p) {
        s16x4 v[2];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const char* at = rows + ((p * 4 + 2 * step + half) * (kK / 32) + tile / 2) * 1024 +
                             slot(from, tile / 2) + 8 * (tile % 2);
            v[half] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(s16x4*)at);
        }
        __builtin_memcpy(&f.part[p], v, 16);
    }
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

// Gives what was written to LDS before, by flag, to the other wave of a pair.  A wave's
// LDS accesses are carried out in order, so neither side has to wait for its own.
__device__ inline void give(int* flag, int n) {
    asm volatile("" ::: "memory");
    __hip_atomic_store(flag, n, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
}
// Reads behind a flag, until they came after its n-th rise.
template <class F>
__device__ inline void take(const int* flag, int n, F&& read) {
    int given;
    do {
        given = __hip_atomic_load(flag, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
        asm volatile("" ::: "memory");
        read();
        asm volatile("" ::: "memory");
    } while (__builtin_amdgcn_readfirstlane(given) < n);
}

// Until a flag is at n.
__device__ inline void wait_given(const int* flag, int n) {
    while (__hip_atomic_load(flag, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP) < n)
        __builtin_amdgcn_s_sleep(1);
}

// A piece of a record on its way to LDS, 16 bytes a thread and turn.  (Here and below,
// threads without a part of their own load one all the same: which loads are
// under way is then the same on every path, and a wait waits for no later ones.)
template <int kBytes, int kThreads>
struct Copy {
    static constexpr int kPieces = kBytes / 16, kTurns = (kPieces + kThreads - 1) / kThreads;
    u32x4 x[kTurns];
    __device__ void load(const char* from, int thread) {
#pragma unroll
        for (int i = 0; i < kTurns; ++i)
            x[i] = reinterpret_cast<const u32x4*>(from)[(thread + i * kThreads) % kPieces];
    }
    __device__ void store(char* to, int thread) const {
#pragma unroll
        for (int i = 0; i < kTurns; ++i) {
            const int at = thread + i * kThreads;
            if (kPieces % kThreads == 0 || at < kPieces) reinterpret_cast<u32x4*>(to)[at] = x[i];
        }
    }
};

// A chunk's rows of K or Q on their way to LDS, with their scales.
template <class T, int kK, int kThreads>
struct Rows {
    using U = Unit<T, kK>;
    static constexpr int kMine = (U::kUnits + kThreads - 1) / kThreads;
    U u[kMine];
    f32x4 scale[kMine];
    __device__ void load(const T* rows, int64_t stride, int count, int size, bool wide,
                         const float* scales, int thread) {
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            const int unit = (thread + i * kThreads) % U::kUnits;
            u[i].load(rows, stride, unit, count, size, wide);
            if (!__is_same(T, f16_t))
                scale[i] = reinterpret_cast<const f32x4*>(scales)[unit / (kK / 8)];
        }
    }
    __device__ void store(char* to, int thread) const {
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            const int unit = thread + i * kThreads;
            if (U::kUnits % kThreads != 0 && unit >= U::kUnits) continue;
            u[i].store(to, unit, scale[i]);
        }
    }
};

// Place of lane l's four tokens among the 64 of a tile of a block of 16
// columns: spread over the banks for those who write them, four columns each.
__device__ inline int value_slot(int lane, int block) { return lane ^ (((lane >> 4) ^ block) & 3); }

// Columns of V or dO on their way to LDS, where they lie as the waves that own
// 16 columns hold them: 4 tokens of a column together.  A thread takes 4
// tokens x 4 columns of 16 kBlocks ones.
template <class T, int kBlocks, int kThreads>
struct Values {
    static constexpr int kUnits = 16 * 4 * kBlocks;
    static constexpr int kEach = kC * 16 * sizeof(T);  // bytes of a block of 16 columns
    static constexpr int kMine = (kUnits + kThreads - 1) / kThreads;
    T x[kMine][4][4];
    // rows: of the chunk's first token and first column; size: columns there are
    __device__ void load(const T* rows, int64_t stride, int count, int size, bool wide, int thread) {
        const __amdgpu_buffer_rsrc_t r = buffer_at(rows);
        const uint32_t step = (uint32_t)stride * sizeof(T);
#pragma unroll
        for (int m = 0; m < kMine; ++m) {
            const int unit = (thread + m * kThreads) % kUnits;
            const int t = unit / (4 * kBlocks) * 4, c = unit % (4 * kBlocks) * 4;
            uint32_t at = c < size ? t * step + c * (uint32_t)sizeof(T) : kPastEnd;
#pragma unroll
            for (int i = 0; i < 4; ++i, at += step) {
                if (wide) {
                    const uint32_t off = count == kC || t + i < count ? at : kPastEnd;
                    if (sizeof(T) == 2) {
                        const u32x2 w = __builtin_amdgcn_raw_buffer_load_b64(r, off, 0, 0);
                        __builtin_memcpy(x[m][i], &w, 8);
                    } else {
                        const u32x4 w = __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, 0);
                        __builtin_memcpy(x[m][i], &w, 4 * sizeof(T));
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        x[m][i][e] = load_word<T>(r, t + i < count && c + e < size
                                                         ? at + e * (uint32_t)sizeof(T) : kPastEnd);
                }
            }
        }
    }
    __device__ void store(char* to, int thread) const {
#pragma unroll
        for (int m = 0; m < kMine; ++m) {
            const int unit = thread + m * kThreads;
            if (kUnits % kThreads != 0 && unit >= kUnits) continue;
            const int four = unit / (4 * kBlocks), c = unit % (4 * kBlocks) * 4;
            char* at = to + c / 16 * kEach + four / 4 * 64 * 4 * sizeof(T);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                T w[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = x[m][i][e];
                __builtin_memcpy(at + value_slot(four % 4 * 16 + c % 16 + e, c / 16) * 4 * sizeof(T),
                                 w, 4 * sizeof(T));
            }
        }
    }
};

}  // namespace sgemm_emu
