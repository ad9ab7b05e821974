// Attention over whole sequences: one block per 32 kRowGroups query rows of a
// key head (a token's query heads that share it are neighbouring rows).
#include "attention_core.hpp"
#include "attention_rows.hpp"

namespace sgemm_emu {

namespace {

template <class T, bool kVec>
struct ForwardRow {
    T* o;
    float* lse;  // or null
    int size;
    __device__ inline void sums(float l, float z) const {
        if (lse != nullptr)
            *lse = l == 0.0f ? -__builtin_inff() : (z + __builtin_amdgcn_logf(l)) * kLn2;
    }
    __device__ inline void four(int d, float x, float y, float z, float w) const {
        store_four<T, kVec>(o, d, size, x, y, z, w);
    }
};

template <class T, int D, int kRowGroups, int kKeyGroups, int kKeys, bool kVec>
__global__ __launch_bounds__(64 * kRowGroups * kKeyGroups, 2) void attention_forward_kernel(
    attention_emu_forward_t a, int first_block) {
    using Pass = Attend<T, D, kRowGroups, kKeyGroups, kKeys, kVec>;
    __shared__ __attribute__((aligned(16))) char lds[Pass::kLds];
    const int group = a.q_heads / a.k_heads;
    const bool packed = a.cu_seqlens != nullptr;
    const int block = first_block + (int)blockIdx.x;
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
    const T* q = row_of<T>(a.q, packed, n, sq, head * group);
    const T* k = row_of<T>(a.k, packed, n, sk, head);
    const T* v = row_of<T>(a.v, packed, n, sk, head);
    float* lse = a.lse.p == nullptr ? nullptr : row_of<float>(a.lse, packed, n, sq, head * group);
    T* o = row_of<T>(a.o, packed, n, sq, head * group);
    const auto out = [&](int r) {
        const int token = r / group, h = r % group;
        return ForwardRow<T, kVec>{o + token * a.o.token + h * a.o.head,
                                   lse ? lse + token * a.lse.token + h * a.lse.head : nullptr, a.size};
    };
    const int shift = sk.count - sq.count + 1;
    Pass::run(
        lds, rows, tile * Pass::kRows,
        [&](int r) { return q + r / group * a.q.token + r % group * a.q.head; },
        [&](int r) { return a.causal ? r / group + shift : sk.count; }, k, a.k.token, v, a.v.token, 0,
        sk.count, a.size, __builtin_fabsf(a.scale) * kLog2e, a.scale < 0.0f, out);
}

template <class T, int D, int kRowGroups, int kKeyGroups, int kKeys, bool kVec>
hipError_t launch(const attention_emu_forward_t& a, hipStream_t stream) {
    const int group = a.q_heads / a.k_heads;
    const int64_t parts = most_parts(a.batch, (int64_t)a.tokens * group, 32 * kRowGroups,
                                     a.cu_seqlens != nullptr);
    return launch_blocks(attention_forward_kernel<T, D, kRowGroups, kKeyGroups, kKeys, kVec>,
                         parts * a.k_heads, 64 * kRowGroups * kKeyGroups, stream, a);
}

}  // namespace

hipError_t launch_attention_forward(const attention_emu_forward_t& args, hipStream_t stream) {
    attention_emu_forward_t a = args;
    if (a.cu_seqlens != nullptr && a.cu_keys == nullptr) a.cu_keys = a.cu_seqlens;
    const int e = a.dtype == SGEMM_EMU_F32 ? 4 : 2;
    const bool vec = a.size * e % 16 == 0 && rows_aligned16(a.q, e) && rows_aligned16(a.k, e) &&
                     rows_aligned16(a.v, e) && rows_aligned16(a.o, e);
    return by_form(a.dtype, a.size, vec, [&](auto t, auto d, auto vec) {
        using T = decltype(t);
        constexpr int D = decltype(d)::value;
        constexpr int kKeys = sizeof(T) == 2 || D <= 64 ? 64 : 32;
        return launch<T, D, 4, 1, kKeys, decltype(vec)::value != 0>(a, stream);
    });
}

}  // namespace sgemm_emu
