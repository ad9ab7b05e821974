// Rotary positions: y = G(angles of the token's position) x on the first `rot`
// elements of every head, the pairs' Givens rotations taken from a table of
// cosines and sines (FP32 arithmetic, one rounding).
//
// Bound by memory: x is read and y written once; the table's row (8 bytes a
// pair) is read once per kHeads heads of a token and mostly comes from the
// caches.  A thread turns the same kVec pairs of up to kHeads heads, so their
// angles stay in registers, and moves 16 bytes at a time where the rows'
// alignment allows.  Measured: 4 x 4096 tokens of 40 heads of 128 in bfloat16 70 us, 4.85
// TB/s (a large copy: 5.0); 64 tokens 5.5 us.
#include "mixing.hpp"

namespace sgemm_emu {

namespace {

constexpr int kThreads = 256;

struct RotaryArgs {
    rotary_emu_t a;
    int units;      // pieces of a head: turned ones, then copied ones
    int turned;     // pieces that are turned
    int parts;      // groups of heads
    int per;        // heads in a group
    int rows;       // tokens of a block
    int64_t total;  // tokens in all
};

template <class T, int N>
using Vec = typename Pack<T, N>::type;

template <class T, int N>
__device__ inline Vec<T, N> load(const T* p) {
    return *reinterpret_cast<const Vec<T, N>*>(p);
}
template <class T, int N>
__device__ inline void store(T* p, Vec<T, N> v) {
    *reinterpret_cast<Vec<T, N>*>(p) = v;
}

// A piece is N pairs: in interleaved order 2N consecutive elements, in half
// order N elements and their N partners; or 2N elements that are copied.
template <class T, int N, bool kInterleaved, int kHeads>
__global__ __launch_bounds__(kThreads) void rotary_kernel(RotaryArgs p, int64_t first_block) {
    const rotary_emu_t& a = p.a;
    const int items = p.units * p.parts;
    const int half = a.rot / 2;
    for (int w = threadIdx.x; w < p.rows * items; w += kThreads) {
        const int row = w / items, item = w - row * items;
        const int part = item / p.units, unit = item - part * p.units;
        const int64_t token = (first_block + blockIdx.x) * p.rows + row;
        if (token >= p.total) return;
        const int b = (int)(token / a.tokens), t = (int)(token - (int64_t)b * a.tokens);
        const bool turn = unit < p.turned;
        float c[N], s[N];
        if (turn) {
            int64_t at = t + a.offset;
            if (a.positions != nullptr) {
                const int64_t i = b * a.position_batch + t * a.position_token;
                at = a.position_bytes == 8 ? static_cast<const int64_t*>(a.positions)[i]
                                           : (int64_t)static_cast<const int32_t*>(a.positions)[i];
            }
            const bool inside = at >= 0 && at < a.table_rows;
            const int64_t from = (inside ? at : 0) * half + unit * N;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                c[i] = inside ? a.cos_table[from + i] : __builtin_nanf("");
                s[i] = inside ? a.sin_table[from + i] : __builtin_nanf("");
                if (a.inverse) s[i] = -s[i];
            }
        }
        const int first = part * p.per, last = min(first + p.per, a.heads[0] + a.heads[1]);
        const auto row_at = [&](const sgemm_emu_view_t(&views)[2], int h)
            __attribute__((always_inline)) {
            const int which = h < a.heads[0] ? 0 : 1;
            const sgemm_emu_view_t& v = views[which];
            return static_cast<T*>(v.p) + b * v.batch + t * v.token +
                   (which ? h - a.heads[0] : h) * v.head;
        };
        if (turn || a.rot + (unit - p.turned + 1) * 2 * N <= a.size) {
            // two vectors of each head: all loads first, so that they are in flight together
            const int c0 = a.rot + (unit - p.turned) * 2 * N;
            const int ea = !turn ? c0 : kInterleaved ? unit * 2 * N : unit * N;
            const int eb = !turn || kInterleaved ? ea + N : ea + half;
            T in[kHeads][2 * N];
#pragma unroll
            for (int j = 0; j < kHeads; ++j)
                if (first + j < last) {
                    const T* x = row_at(a.x, first + j);
                    *reinterpret_cast<Vec<T, N>*>(in[j]) = load<T, N>(x + ea);
                    *reinterpret_cast<Vec<T, N>*>(in[j] + N) = load<T, N>(x + eb);
                }
#pragma unroll
            for (int j = 0; j < kHeads; ++j) {
                if (first + j >= last) continue;
                T* y = row_at(a.y, first + j);
                if (!turn && y == row_at(a.x, first + j)) continue;
                T out[2 * N];
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const int ia = kInterleaved ? 2 * i : i, ib = kInterleaved ? 2 * i + 1 : N + i;
                    const float xa = to_f32(in[j][ia]), xb = to_f32(in[j][ib]);
                    out[ia] = turn ? from_f32<T>(__builtin_fmaf(xa, c[i], -(xb * s[i]))) : in[j][ia];
                    out[ib] = turn ? from_f32<T>(__builtin_fmaf(xa, s[i], xb * c[i])) : in[j][ib];
                }
                store<T, N>(y + ea, *reinterpret_cast<Vec<T, N>*>(out));
                store<T, N>(y + eb, *reinterpret_cast<Vec<T, N>*>(out + N));
            }
        } else {  // the end of a row that is copied
            for (int h = first; h < last; ++h) {
                const T* x = row_at(a.x, h);
                T* y = row_at(a.y, h);
                if (x != y)
                    for (int e = a.rot + (unit - p.turned) * 2 * N; e < a.size; ++e) y[e] = x[e];
            }
        }
    }
}

// Whether every row of a view starts at a multiple of `bytes`.
bool rows_aligned(const sgemm_emu_view_t& v, int elem, int bytes) {
    const int64_t n = bytes / elem;
    return (uintptr_t)v.p % bytes == 0 && v.batch % n == 0 && v.token % n == 0 && v.head % n == 0;
}

template <class T, int N, int kHeads>
hipError_t launch_heads(RotaryArgs p, hipStream_t stream) {
    const rotary_emu_t& a = p.a;
    const int heads = a.heads[0] + a.heads[1];
    p.per = kHeads;
    p.parts = (heads + p.per - 1) / p.per;
    const int64_t items = (int64_t)p.units * p.parts;
    p.rows = items >= kThreads ? 1 : (int)(kThreads / items);
    const int64_t blocks = (p.total + p.rows - 1) / p.rows;
    for (int64_t first = 0; first < blocks; first += kMostBlocks) {
        const dim3 grid((unsigned)(blocks - first < kMostBlocks ? blocks - first : kMostBlocks));
        if (a.interleaved)
            hipLaunchKernelGGL((rotary_kernel<T, N, true, kHeads>), grid, dim3(kThreads), 0, stream, p,
                               first);
        else
            hipLaunchKernelGGL((rotary_kernel<T, N, false, kHeads>), grid, dim3(kThreads), 0, stream, p,
                               first);
        if (hipError_t e = hipGetLastError()) return e;
    }
    return hipSuccess;
}

template <class T, int N>
hipError_t launch(RotaryArgs p, hipStream_t stream) {
    const rotary_emu_t& a = p.a;
    p.turned = a.rot / (2 * N);
    p.units = p.turned + (a.size - a.rot + 2 * N - 1) / (2 * N);
    // Heads that share a thread's angles, whose loads are in flight together:
    // four, where that still leaves every CU its eight blocks, else one
    const int64_t work = p.total * p.units * (a.heads[0] + a.heads[1]);
    return work / (4 * kThreads) >= 8 * 256 ? launch_heads<T, N, 4>(p, stream)
                                            : launch_heads<T, N, 1>(p, stream);
}

__global__ __launch_bounds__(kThreads) void rotary_table_kernel(int rows, int half, double base,
                                                                double factor, double original,
                                                                double low, double high,
                                                                double amplitude, float* c,
                                                                float* s) {
    const int64_t n = (int64_t)rows * half;
    for (int64_t w = (int64_t)blockIdx.x * kThreads + threadIdx.x; w < n;
         w += (int64_t)gridDim.x * kThreads) {
        const int64_t p = w / half;
        const int i = (int)(w - p * half);
        constexpr double kTurn = 6.283185307179586476925;
        const double f = pow(base, -(double)i / half);
        double keep = 0.0;
        if (low < high) keep = fmin(1.0, fmax(0.0, (original * f / kTurn - low) / (high - low)));
        const double angle = (double)p * f * (keep + (1.0 - keep) / factor);
        c[w] = (float)(amplitude * cos(angle));
        s[w] = (float)(amplitude * sin(angle));
    }
}

}  // namespace

hipError_t launch_rotary(const rotary_emu_t& a, hipStream_t stream) {
    RotaryArgs p{};
    p.a = a;
    p.total = (int64_t)a.batch * a.tokens;
    if (a.x[1].p == nullptr) p.a.heads[1] = 0;
    if (p.total == 0 || a.size == 0 || p.a.heads[0] + p.a.heads[1] == 0) return hipSuccess;
    return by_dtype(a.dtype, [&](auto t) {
        using T = decltype(t);
        // 16 bytes, then 8, then an element at a time as rows, halves and the part
        // that is copied allow
        const auto fits = [&](int n) {
            const int bytes = n * (int)sizeof(T);
            for (int i = 0; i < 2; ++i)
                if (p.a.heads[i] > 0 && (!rows_aligned(a.x[i], sizeof(T), bytes) ||
                                         !rows_aligned(a.y[i], sizeof(T), bytes)))
                    return false;
            return a.rot % (2 * n) == 0;
        };
        constexpr int kMost = 16 / sizeof(T);
        if (fits(kMost)) return launch<T, kMost>(p, stream);
        if (fits(kMost / 2)) return launch<T, kMost / 2>(p, stream);
        return launch<T, 1>(p, stream);
    });
}

hipError_t launch_rotary_table(int rows, int rot, double base, double factor, double original,
                               double low, double high, double amplitude, float* cos_table,
                               float* sin_table, hipStream_t stream) {
    const int64_t n = (int64_t)rows * (rot / 2);
    if (n == 0) return hipSuccess;
    const unsigned blocks = (unsigned)((n + kThreads - 1) / kThreads < 8192
                                           ? (n + kThreads - 1) / kThreads : 8192);
    hipLaunchKernelGGL(rotary_table_kernel, dim3(blocks), dim3(kThreads), 0, stream, rows, rot / 2,
                       base, factor, original, low, high, amplitude, cos_table, sin_table);
    return hipGetLastError();
}

}  // namespace sgemm_emu
