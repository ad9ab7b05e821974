// Attention of single tokens behind a shared prefix and caches of their own.
//
// The prefix is read once for the batch: its blocks take 128 rows of a key head, of any
// sequences, through a part of the prefix's keys.  The caches' blocks take the rows of one
// sequence through a part of its cache, 32 keys to a wave.  Each leaves its rows' normalized result
// and log-sum in the workspace, and a second kernel joins the parts of a row; where there
// is one part, it is the result.
#include <algorithm>

#include "attention_core.hpp"
#include "attention_rows.hpp"

namespace sgemm_emu {

namespace {

constexpr int kThreads = 256;
constexpr int kPrefixRows = 128;

// Elements from one row of a part to the next.
template <int D>
constexpr int kStride = D <= 64 ? 64 : 128;

struct StepArgs {
    attention_emu_step_t a;
    int prefix_parts, prefix_tiles, prefix_keys;  // parts, row tiles, keys of a part
    int own_parts;
    float* parts;  // [part][row][kStride], or null: one part, written to o
    float* logs;   // [part][row], base 2
    int64_t rows;  // batch x tokens x q_heads
};

template <class T, bool kVec>
struct StepRow {
    T* o;         // or, of a part,
    float* part;  // its row
    float* log;
    int size;
    __device__ inline void sums(float l, float z) const {
        if (part != nullptr) *log = l == 0.0f ? -__builtin_inff() : z + __builtin_amdgcn_logf(l);
    }
    __device__ inline void four(int d, float x, float y, float z, float w) const {
        if (part == nullptr)
            store_four<T, kVec>(o, d, size, x, y, z, w);
        else if (d < size)
            *reinterpret_cast<Pack<float, 4>::type*>(part + d) = Pack<float, 4>::type{x, y, z, w};
    }
};

template <class T, int D, bool kVec>
__global__ __launch_bounds__(kThreads, 2) void attention_step_kernel(StepArgs s, int first_block) {
    using Prefix = Attend<T, D, 4, 1, sizeof(T) == 2 || D <= 64 ? 64 : 32, kVec>;
    using Own = Attend<T, D, 1, 4, 32, kVec>;
    constexpr int kLds = Prefix::kLds > Own::kLds ? Prefix::kLds : Own::kLds;
    __shared__ __attribute__((aligned(16))) char lds[kLds];
    const attention_emu_step_t& a = s.a;
    const int group = a.q_heads / a.k_heads;
    const float c = __builtin_fabsf(a.scale) * kLog2e;
    int block = first_block + (int)blockIdx.x;
    const int prefix_blocks = s.prefix_parts * s.prefix_tiles * a.k_heads;
    // results of part p for query head h of token t of all
    const auto out_of = [&](int p, int t, int h) {
        const int64_t row = (int64_t)t * a.q_heads + h;
        T* o = static_cast<T*>(a.o.p) + t / a.tokens * a.o.batch + t % a.tokens * a.o.token +
               h * a.o.head;
        return StepRow<T, kVec>{o, s.parts ? s.parts + (p * s.rows + row) * kStride<D> : nullptr,
                                s.logs + p * s.rows + row, a.size};
    };
    const auto q_row = [&](int t, int h) {
        return static_cast<const T*>(a.q.p) + t / a.tokens * a.q.batch + t % a.tokens * a.q.token +
               h * a.q.head;
    };
    if (block < prefix_blocks) {
        const int head = block % a.k_heads, rest = block / a.k_heads;
        const int part = rest % s.prefix_parts, tile = rest / s.prefix_parts;
        const int first = part * s.prefix_keys, end = min(first + s.prefix_keys, a.prefix);
        const auto out = [&](int r) { return out_of(part, r / group, head * group + r % group); };
        Prefix::run(
            lds, a.batch * a.tokens * group, tile * kPrefixRows,
            [&](int r) { return q_row(r / group, head * group + r % group); },
            [&](int) { return a.prefix; },
            static_cast<const T*>(a.prefix_k.p) + head * a.prefix_k.head, a.prefix_k.token,
            static_cast<const T*>(a.prefix_v.p) + head * a.prefix_v.head, a.prefix_v.token, first,
            end, a.size, c, a.scale < 0.0f, out);
        return;
    }
    block -= prefix_blocks;
    const int row_tiles = (a.tokens * group + 31) / 32;
    const int head = block % a.k_heads, rest = block / a.k_heads;
    const int tile = rest % row_tiles, part = rest / row_tiles % s.own_parts;
    const int n = rest / row_tiles / s.own_parts;
    const int slot = a.slots == nullptr ? n : a.slots[n];
    const bool in = slot >= 0 && slot < a.n_slots;
    const int keys = in ? min(max(a.lengths[n], 0), a.capacity) : 0;
    const int shift = keys - a.tokens + 1;
    const int each = ((keys + s.own_parts - 1) / s.own_parts + 31) / 32 * 32;
    const int first = min(part * each, keys), end = min(first + each, keys);
    const auto out = [&](int r) {
        return out_of(s.prefix_parts + part, n * a.tokens + r / group, head * group + r % group);
    };
    const int64_t at = in ? slot : 0;
    Own::run(
        lds, a.tokens * group, tile * 32,
        [&](int r) { return q_row(n * a.tokens + r / group, head * group + r % group); },
        [&](int r) { return r / group + shift; },
        static_cast<const T*>(a.k.p) + at * a.k.batch + head * a.k.head, a.k.token,
        static_cast<const T*>(a.v.p) + at * a.v.batch + head * a.v.head, a.v.token, first, end,
        a.size, c, a.scale < 0.0f, out);
}

// o = sum_p 2^(log_p - z) part_p / sum_p 2^(log_p - z), z the largest.
template <class T, int D, bool kVec>
__global__ __launch_bounds__(kThreads) void attention_join_kernel(StepArgs s, int parts,
                                                                  int first_block) {
    const attention_emu_step_t& a = s.a;
    const int64_t w = (first_block + blockIdx.x) * kThreads + threadIdx.x;
    const int64_t row = w / (D / 4);
    const int d = (int)(w % (D / 4)) * 4;
    if (row >= s.rows || d >= a.size) return;
    const int64_t token = row / a.q_heads;
    const int h = (int)(row - token * a.q_heads), n = (int)(token / a.tokens);
    float z = -1e30f, l = 0.0f;
    for (int p = 0; p < parts; ++p) z = fmaxf(z, s.logs[p * s.rows + row]);
    Pack<float, 4>::type x{};
    const int slot = a.slots == nullptr ? n : a.slots[n];
    if (slot >= 0 && slot < a.n_slots) {
        for (int p = 0; p < parts; ++p) {
            const float log = s.logs[p * s.rows + row];
            if (log == -__builtin_inff()) continue;
            const float f = __builtin_amdgcn_exp2f(log - z);
            l += f;
            const auto y = *reinterpret_cast<const Pack<float, 4>::type*>(
                s.parts + (p * s.rows + row) * kStride<D> + d);
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] += f * y[j];
        }
    }
    const float f = l == 0.0f ? 0.0f : 1.0f / l;
    T* o = static_cast<T*>(a.o.p) + n * a.o.batch + (token - (int64_t)n * a.tokens) * a.o.token +
           h * a.o.head;
    store_four<T, kVec>(o, d, a.size, x[0] * f, x[1] * f, x[2] * f, x[3] * f);
}

int padded(int size) { return size <= 64 ? 64 : 128; }  // kStride

// How the keys are cut.
StepArgs cut(const attention_emu_step_t& a) {
    StepArgs s{};
    s.a = a;
    const int64_t group = a.q_heads / a.k_heads;
    s.rows = (int64_t)a.batch * a.tokens * a.q_heads;
    const int64_t rows = (int64_t)a.batch * a.tokens * group;
    s.prefix_tiles = (int)((rows + kPrefixRows - 1) / kPrefixRows);
    constexpr int64_t kWanted = 512;  // blocks: two for each CU
    if (a.prefix > 0) {
        const int64_t blocks = (int64_t)s.prefix_tiles * a.k_heads;
        const int64_t most = (a.prefix + 255) / 256;
        const int64_t parts = std::max<int64_t>(1, std::min(most, kWanted / blocks));
        s.prefix_keys = (int)(((a.prefix + parts - 1) / parts + 63) / 64 * 64);
        s.prefix_parts = (a.prefix + s.prefix_keys - 1) / s.prefix_keys;
    }
    const int64_t blocks = (int64_t)a.batch * a.k_heads * ((a.tokens * group + 31) / 32);
    const int64_t most = (a.capacity + 255) / 256;
    s.own_parts = (int)std::max<int64_t>(1, std::min(most, kWanted / std::max<int64_t>(1, blocks)));
    return s;
}

int64_t part_floats(const StepArgs& s) { return s.rows * padded(s.a.size); }

}  // namespace

int64_t attention_step_workspace(const attention_emu_step_t& a) {
    const StepArgs s = cut(a);
    const int64_t parts = s.prefix_parts + s.own_parts;
    if (parts == 1) return 0;
    const int64_t bytes = parts * (part_floats(s) + s.rows) * 4;
    return (bytes + 255) / 256 * 256;
}

hipError_t launch_attention_step(const attention_emu_step_t& a, hipStream_t stream) {
    StepArgs s = cut(a);
    const int parts = s.prefix_parts + s.own_parts;
    if (parts > 1) {
        s.parts = static_cast<float*>(a.workspace);
        s.logs = s.parts + parts * part_floats(s);
    }
    const int64_t group = a.q_heads / a.k_heads;
    const int64_t blocks =
        (int64_t)s.prefix_parts * s.prefix_tiles * a.k_heads +
        (int64_t)s.own_parts * a.batch * a.k_heads * ((a.tokens * group + 31) / 32);
    const int e = a.dtype == SGEMM_EMU_F32 ? 4 : 2;
    const bool prefix = a.prefix > 0;
    const bool vec = a.size * e % 16 == 0 && rows_aligned16(a.q, e) && rows_aligned16(a.k, e) &&
                     rows_aligned16(a.v, e) && rows_aligned16(a.o, e) &&
                     (!prefix || (rows_aligned16(a.prefix_k, e) && rows_aligned16(a.prefix_v, e)));
    return by_form(a.dtype, a.size, vec, [&](auto t, auto d, auto vec) {
        using T = decltype(t);
        constexpr int D = decltype(d)::value;
        constexpr bool kVec = decltype(vec)::value != 0;
        if (hipError_t e = launch_blocks(attention_step_kernel<T, D, kVec>, blocks, kThreads, stream,
                                         s))
            return e;
        if (parts == 1) return hipSuccess;
        constexpr int kRows = kThreads / (kStride<D> / 4);
        return launch_blocks(attention_join_kernel<T, D, kVec>, (s.rows + kRows - 1) / kRows, kThreads,
                             stream, s, parts);
    });
}

}  // namespace sgemm_emu
