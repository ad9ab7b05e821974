// Attention over whole sequences: one block per 32 kRowGroups query rows of a
// key head (a token's query heads that share it are neighbouring rows, so that grouped heads read
// a key once).  Bound by the matrix instructions and what keeps them from running at once: 4 x
// 4096 causal tokens, 32 heads of 128 in bfloat16, 569 to 620 us on two machines (966 to 887 TFLOP/s
// of the 1270 of a large product; 48% of the cycles have matrix instructions in flight, 46% vector
// ones), one prompt of 32768 with 8 heads 2.08 to 2.22 ms (1056 to 990).  On that one, where it took
// 2124, without the softmax's arithmetic 1880, without loads 1814.
#include <algorithm>

#include "attention_core.hpp"
#include "attention_split.h"

namespace sgemm_emu {

namespace {

struct ForwardArgs {
    attention_emu_forward_t a;
    int count;  // parts that a block's keys are cut into
    Parts parts;
    // the operands, split if they are FP32
    sgemm_emu_view_t q, k, v;
    const float *q_factors, *k_factors, *v_factors;
};

struct ForwardFactors {
    const float* first;  // of the sequence's tokens
    int q_heads, head, group;
    const float *k, *v;
    int64_t step;
    __device__ inline float q(int r) const {
        return first[(int64_t)(r / group) * q_heads + head + r % group];
    }
};

template <class T, int D, int kRowGroups, int kKeyGroups, int kKeys, bool kVec>
__global__ __launch_bounds__(64 * kRowGroups * kKeyGroups,
                             sizeof(Elem<T>) == 4 && D > 64 ? 1 : 2) void attention_forward_kernel(
    ForwardArgs args, int first_block) {
    const attention_emu_forward_t& a = args.a;
    using Pass = Attend<T, D, kRowGroups, kKeyGroups, kKeys, kVec>;
    __shared__ __attribute__((aligned(16))) char lds[Pass::kLds];
    const int group = a.q_heads / a.k_heads;
    const bool packed = a.cu_seqlens != nullptr;
    const int part = (first_block + (int)blockIdx.x) % args.count;
    const int block = (first_block + (int)blockIdx.x) / args.count;
    int n, head, tile;
    if (packed) {
        head = block % a.k_heads;
        const Place p = find_part(a.cu_seqlens, a.batch, a.tokens, group, Pass::kRows,
                                  block / a.k_heads);
        if (!p.found) return;
        n = p.n, tile = p.tile;
    } else {
        // the last rows of all sequences first: with a causal mask they take longest
        const int pairs = a.batch * a.k_heads;
        const int tiles = (a.tokens * group + Pass::kRows - 1) / Pass::kRows;
        const int pair = block % pairs;
        n = pair / a.k_heads, head = pair % a.k_heads;
        tile = tiles - 1 - block / pairs;
    }
    const Span sq = span_of(a.cu_seqlens, n, a.tokens);
    const Span sk = span_of(a.cu_keys, n, a.keys);
    const int rows = sq.count * group;
    typedef Elem<T> E;
    const E* q = row_of<E>(args.q, packed, n, sq, head * group);
    const E* k = row_of<E>(args.k, packed, n, sk, head);
    const E* v = row_of<E>(args.v, packed, n, sk, head);
    float* lse = a.lse.p == nullptr ? nullptr : row_of<float>(a.lse, packed, n, sq, head * group);
    auto* o = row_of<Out<T>>(a.o, packed, n, sq, head * group);
    const int64_t first_token = packed ? sq.first : (int64_t)n * a.tokens;
    const int64_t first_key = (packed ? sk.first : (int64_t)n * a.keys) * a.k_heads + head;
    const ForwardFactors factors{args.q_factors + first_token * a.q_heads, a.q_heads, head * group,
                                 group, args.k_factors + first_key, args.v_factors + first_key,
                                 a.k_heads};
    const auto out = [&](int r) {
        const int token = r / group, h = r % group;
        return row_out<Out<T>, D, kVec>(args.parts, part,
                                   (first_token + token) * a.q_heads + head * group + h,
                                   o + token * a.o.token + h * a.o.head,
                                   lse ? lse + token * a.lse.token + h * a.lse.head : nullptr,
                                   a.size);
    };
    const int shift = sk.count - sq.count + 1;
    const auto limit = [&](int r) { return a.causal ? r / group + shift : sk.count; };
    // the part's share of the keys that the block's rows see
    const int seen = min(max(limit(min((tile + 1) * Pass::kRows, rows) - 1), 0), sk.count);
    const int each = (seen + args.count * kKeys - 1) / (args.count * kKeys) * kKeys;
    const int first = min(part * each, seen), end = min(first + each, seen);
    Pass::run(
        lds, rows, tile * Pass::kRows,
        [&](int r) { return q + r / group * args.q.token + r % group * args.q.head; }, limit, k,
        args.k.token, v, args.v.token, first, end, a.size, __builtin_fabsf(a.scale) * kLog2e,
        a.scale < 0.0f, out, factors);
}

// Blocks of `rows` query rows.
int64_t blocks_of(const attention_emu_forward_t& a, int rows) {
    const int64_t group = a.q_heads / a.k_heads;
    return most_parts(a.batch, a.tokens * group, rows, a.cu_seqlens != nullptr) * a.k_heads;
}

constexpr int kRowGroups = 4;

// Whether all is so little that latency counts: blocks of 32 rows whose four waves share out
// the keys then, up to two tiles each, and FP32 is multiplied as it is (128 tokens of 32 heads
// 18.2 -> 12.6 us, 256 in FP32 26.9 -> 23.1; with 512 keys 40.7 -> 49.1 in FP32 and 17.5 -> 17.9 in
// bfloat16, with 512 blocks 13.5 -> 14.0 and 31.6 -> 35.6 in FP32).
bool few(const attention_emu_forward_t& a) {
    return a.cu_seqlens == nullptr && a.keys <= 256 && blocks_of(a, 32) <= 256;
}

// Parts of the keys: where the blocks leave CUs idle, as many as fill those, of at least 256
// keys each (512: no change), if that saves a block more steps of 64 keys than the join costs
// (its launch and traffic, about ten of them): 512 tokens, the last of 8192, 144 -> 62 us, 16 of
// 8192 132 -> 18, 512 of 2048 39 -> 33, 256 of 1024 (12 steps) 23.9 -> 20.4; 1024 tokens (8 steps)
// 24.2 -> 31.4.
int parts_of(const attention_emu_forward_t& a) {
    const int64_t blocks = blocks_of(a, 32 * kRowGroups), most = (a.keys + 255) / 256;
    if (few(a) || blocks == 0 || most <= 1 || a.cu_seqlens != nullptr) return 1;
    const int64_t parts = std::max<int64_t>(1, std::min(most, 256 / blocks));
    const int64_t steps = (a.keys + 63) / 64;
    return steps - steps / parts > 10 ? (int)parts : 1;
}

// Whether two groups of waves share a block's keys: 3 x 1001 tokens of 6 heads 26 -> 22 us; where
// other blocks fill the CUs a block's chain is not what counts (24 packed sequences 67 -> 78 us,
// 512 blocks 54 -> 64).
bool paired(const attention_emu_forward_t& a, int64_t blocks) {
    return blocks <= 256 && a.keys > 128;
}

// Tokens and keys in all.
int64_t tokens_of(const attention_emu_forward_t& a) {
    return (a.cu_seqlens != nullptr ? 1 : (int64_t)a.batch) * a.tokens;
}
int64_t keys_of(const attention_emu_forward_t& a) {
    return (a.cu_seqlens != nullptr ? 1 : (int64_t)a.batch) * a.keys;
}

int64_t bytes_of_parts(const attention_emu_forward_t& a, int parts) {
    return parts == 1 ? 0 : parts_bytes(parts, tokens_of(a) * a.q_heads, a.size);
}

}  // namespace

int64_t attention_forward_workspace(const attention_emu_forward_t& a) {
    int64_t bytes = bytes_of_parts(a, parts_of(a));
    if (a.dtype == SGEMM_EMU_F32 && !few(a))
        bytes += split_bytes(tokens_of(a), a.q_heads, a.size) +
                 2 * split_bytes(keys_of(a), a.k_heads, a.size);
    return bytes;
}

hipError_t launch_attention_forward(const attention_emu_forward_t& a, hipStream_t stream) {
    const int parts = parts_of(a);
    ForwardArgs args{a, parts, parts_in(a.workspace, parts, tokens_of(a) * a.q_heads, a.size),
                     a.q, a.k, a.v, nullptr, nullptr, nullptr};
    if (a.cu_seqlens != nullptr && a.cu_keys == nullptr) args.a.cu_keys = a.cu_seqlens;
    const int e = a.dtype == SGEMM_EMU_F32 ? 4 : 2;
    bool vec = a.size * e % 16 == 0 && rows_aligned16(a.o, e);
    if (few(a)) {
        vec = vec && rows_aligned16(a.q, e) && rows_aligned16(a.k, e) && rows_aligned16(a.v, e);
        return by_form<float>(a.dtype, a.size, vec, [&](auto t, auto d, auto vec) {
            return launch_blocks(attention_forward_kernel<decltype(t), decltype(d)::value, 1, 4, 32,
                                                          decltype(vec)::value != 0>,
                                 blocks_of(a, 32), 256, stream, args);
        });
    }
    if (a.dtype == SGEMM_EMU_F32) {
        Splitter split(a.size, static_cast<char*>(a.workspace) + bytes_of_parts(a, parts));
        const int batch = a.cu_seqlens != nullptr ? 1 : a.batch;
        const SplitTensor q = split.add(a.q, batch, a.tokens, a.q_heads);
        const SplitTensor k = split.add(a.k, batch, a.keys, a.k_heads);
        const SplitTensor v = split.add(a.v, batch, a.keys, a.k_heads);
        args.q = q.planes, args.k = k.planes, args.v = v.planes;
        args.q_factors = q.factors, args.k_factors = k.factors, args.v_factors = v.factors;
        if (hipError_t e = split.launch(stream)) return e;
    } else {
        vec = vec && rows_aligned16(a.q, e) && rows_aligned16(a.k, e) && rows_aligned16(a.v, e);
    }
    return by_form<split_t>(a.dtype, a.size, vec, [&](auto t, auto d, auto vec) {
        using T = decltype(t);
        constexpr int D = decltype(d)::value;
        constexpr bool kVec = decltype(vec)::value != 0;
        constexpr int kKeys = kPlanes<T> == 1 || D <= 64 ? 64 : 32;
        const int64_t blocks = blocks_of(a, 32 * kRowGroups) * parts;
        const hipError_t e =
            paired(a, blocks)
                ? launch_blocks(attention_forward_kernel<T, D, kRowGroups, 2, kKeys, kVec>, blocks,
                                64 * 2 * kRowGroups, stream, args)
                : launch_blocks(attention_forward_kernel<T, D, kRowGroups, 1, kKeys, kVec>, blocks,
                                64 * kRowGroups, stream, args);
        if (e != hipSuccess) return e;
        if (parts == 1) return hipSuccess;
        return launch_join<Out<T>, D, kVec>(
            JoinArgs{args.parts, a.o, a.lse, parts, a.tokens, a.q_heads, a.size, nullptr, 0},
            stream);
    });
}

}  // namespace sgemm_emu
