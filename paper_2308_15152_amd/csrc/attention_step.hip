// Attention of single tokens behind a shared prefix and caches of their own.
//
// The prefix is read once for the batch: its blocks take 128 rows of a key head, of any
// sequences, through a part of the prefix's keys.  The caches' blocks take the rows of one
// sequence through a part of its cache, 32 keys to a wave.  The parts of a row are joined by a
// second kernel; where there is one, it is the result.
//
// Bound by memory where the caches are long (128 sequences with caches of 1024 alone: 279 MB in 60
// us, 4.65 TB/s), the prefix by the matrix instructions (as a prompt of the batch's rows: 54 to 60
// us), both together 108 to 114 of the 118 us with the join.  Single sequences: latency, 8 to 10 us
// and 3 of the join.
#include <algorithm>

#include "attention_core.hpp"

namespace sgemm_emu {

namespace {

constexpr int kThreads = 256;
constexpr int kPrefixRows = 128;

struct StepArgs {
    attention_emu_step_t a;
    int prefix_parts, prefix_tiles, prefix_keys;  // parts, row tiles, keys of a part
    bool prefix_few;  // rows: 32 to a tile, whose waves share out the keys
    int own_parts;
    Parts parts;
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
    const int none = 0;  // (tensors that are not split have no factors)
    int block = first_block + (int)blockIdx.x;
    const int prefix_blocks = s.prefix_parts * s.prefix_tiles * a.k_heads;
    // results of part p for query head h of token t of all
    const auto out_of = [&](int p, int t, int h) {
        const int64_t row = (int64_t)t * a.q_heads + h;
        T* o = static_cast<T*>(a.o.p) + t / a.tokens * a.o.batch + t % a.tokens * a.o.token +
               h * a.o.head;
        return row_out<T, D, kVec>(s.parts, p, row, o, nullptr, a.size);
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
        const auto row = [&](int r) { return q_row(r / group, head * group + r % group); };
        const auto all = [&](int) { return a.prefix; };
        const T* k = static_cast<const T*>(a.prefix_k.p) + head * a.prefix_k.head;
        const T* v = static_cast<const T*>(a.prefix_v.p) + head * a.prefix_v.head;
        const int rows = a.batch * a.tokens * group;
        if (s.prefix_few)
            Own::run(lds, rows, tile * 32, row, all, k, a.prefix_k.token, v, a.prefix_v.token,
                     first, end, a.size, c, a.scale < 0.0f, out, none);
        else
            Prefix::run(lds, rows, tile * kPrefixRows, row, all, k, a.prefix_k.token, v,
                        a.prefix_v.token, first, end, a.size, c, a.scale < 0.0f, out, none);
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
        a.size, c, a.scale < 0.0f, out, none);
}

// How the keys are cut.  A cache: into parts of at least 128 keys, a tile for each wave, that
// fill the CUs (one cache of 4096 keys alone: 14.3 us with parts of 512, 11.7 of 256, 10.1 of
// 128), or, up to 32, of 384 that fill them twice, where that is more (16 caches of 4096 23.4 us
// for 25.3, 40 of 1500 25.0 for 29.3; with parts of 128 for that, 33 of 300 take 11.8 us for
// 10.3, with parts of 512 20 of 2000 22.9 for 20.2; 85 parts of one of 32768 24.0 for 20.1 with
// 64).  A prefix: into parts that fill the CUs, of at least 128 keys where one block has all
// rows that there are (16 rows behind 4096 keys 12.2 -> 11.4), else of 256, for more rows are
// more to join (64 rows behind 4096 keys 13.3 us, with 128 16.3).  Up to 64 rows are taken by
// 32, whose waves share out the keys, instead of 128 (16 rows behind 4096 keys: kernel 8.3 us
// for 10.8; 256 rows the same).  The prefix's blocks, one for each CU, come first, and those of
// the caches, which are bound by memory, run beside them: 128 sequences behind 16384 keys take
// 118 us, 144 with the blocks in turn, 141 with the prefix last, 134 with two blocks of the
// prefix for each CU.
StepArgs cut(const attention_emu_step_t& a) {
    StepArgs s{};
    s.a = a;
    const int64_t group = a.q_heads / a.k_heads;
    s.parts.rows = (int64_t)a.batch * a.tokens * a.q_heads;
    const int64_t rows = (int64_t)a.batch * a.tokens * group;
    s.prefix_few = rows <= 64;
    const int64_t tile = s.prefix_few ? 32 : kPrefixRows;
    s.prefix_tiles = (int)((rows + tile - 1) / tile);
    if (a.prefix > 0) {
        const int64_t blocks = (int64_t)s.prefix_tiles * a.k_heads;
        const int64_t each = rows <= 32 ? 128 : 256, most = (a.prefix + each - 1) / each;
        const int64_t parts =
            std::max<int64_t>(1, std::min(most, 256 / std::max<int64_t>(1, blocks)));
        s.prefix_keys = (int)(((a.prefix + parts - 1) / parts + 63) / 64 * 64);
        s.prefix_parts = (a.prefix + s.prefix_keys - 1) / s.prefix_keys;
    }
    const int64_t blocks = (int64_t)a.batch * a.k_heads * ((a.tokens * group + 31) / 32);
    const auto parts = [&](int64_t keys, int64_t fill) {
        return std::min((a.capacity + keys - 1) / keys, fill / std::max<int64_t>(1, blocks));
    };
    s.own_parts = (int)std::max<int64_t>({1, parts(128, 256), std::min<int64_t>(parts(384, 512), 32)});
    return s;
}

}  // namespace

int64_t attention_step_workspace(const attention_emu_step_t& a) {
    const StepArgs s = cut(a);
    const int64_t parts = s.prefix_parts + s.own_parts;
    return parts == 1 ? 0 : parts_bytes(parts, s.parts.rows, a.size);
}

hipError_t launch_attention_step(const attention_emu_step_t& a, hipStream_t stream) {
    StepArgs s = cut(a);
    const int parts = s.prefix_parts + s.own_parts;
    s.parts = parts_in(a.workspace, parts, s.parts.rows, a.size);
    const int64_t group = a.q_heads / a.k_heads;
    const int64_t blocks =
        (int64_t)s.prefix_parts * s.prefix_tiles * a.k_heads +
        (int64_t)s.own_parts * a.batch * a.k_heads * ((a.tokens * group + 31) / 32);
    const int e = a.dtype == SGEMM_EMU_F32 ? 4 : 2;
    const bool prefix = a.prefix > 0;
    const bool vec = a.size * e % 16 == 0 && rows_aligned16(a.q, e) && rows_aligned16(a.k, e) &&
                     rows_aligned16(a.v, e) && rows_aligned16(a.o, e) &&
                     (!prefix || (rows_aligned16(a.prefix_k, e) && rows_aligned16(a.prefix_v, e)));
    return by_form<float>(a.dtype, a.size, vec, [&](auto t, auto d, auto vec) {
        using T = decltype(t);
        constexpr int D = decltype(d)::value;
        constexpr bool kVec = decltype(vec)::value != 0;
        if (hipError_t e =
                launch_blocks(attention_step_kernel<T, D, kVec>, blocks, kThreads, stream, s))
            return e;
        if (parts == 1) return hipSuccess;
        return launch_join<T, D, kVec>(
            JoinArgs{s.parts, a.o, {}, parts, a.tokens, a.q_heads, a.size, a.slots, a.n_slots},
            stream);
    });
}

}  // namespace sgemm_emu
