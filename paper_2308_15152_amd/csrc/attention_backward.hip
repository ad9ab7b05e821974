// The gradient of attention over whole sequences, in two kernels without atomics:
//   attention_dq_kernel   a block has query rows and goes over the keys they see: dq, and
//                         delta_i = do_i o_i into the workspace;
//   attention_dkv_kernel  a block has keys and goes over the query rows (of all of the
//                         key head's query heads) that see them: dk and dv.
// Both form p = 2^(c s - z) again from the scores, c = scale log2 e, z = lse log2 e, and
// dp - delta in the accumulators of do v^T, which start at -delta.  Seven products of 2 D
// operations a pair instead of the five that one pass with shared sums would take, for sums
// whose order is fixed.
//
// Weights p and ds are rounded to the inputs' type as operands.  FP16 has no room for
// either: p is taken times 2^14, and ds times a power of two for each column of the
// accumulator (a query row, or a key), which is lowered, with what is summed so far, when a
// larger value comes.
#include "attention_core.hpp"
#include "attention_rows.hpp"

namespace sgemm_emu {

namespace {

template <class T>
constexpr bool kNarrow = false;
template <>
constexpr bool kNarrow<f16_t> = true;

// A column's power of two.
struct Fit {
    float f = 0x1p100f;

    // So that |x| f stays below 2^15; the sums are rescaled where f changes.
    template <int N>
    __device__ inline void fit(const f32x16& x, f32x16 (&sum)[N]) {
        float most = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) most = fmaxf(most, __builtin_fabsf(x[i]));
        most = max_halves(most);
        const bool over = most * f > 0x1p15f;
        if (__any(over)) {
            // 2^10 <= most f < 2^11
            const int e = (int)(__float_as_uint(most) >> 23);
            const float to = over ? __uint_as_float((unsigned)max(min(264 - e, 227), 1) << 23) : f;
            const float by = to / f;
#pragma unroll
            for (int d = 0; d < N; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) sum[d][i] *= by;
            f = to;
        }
    }
};

__device__ inline f32x16 times(const f32x16& x, float f) {
    f32x16 y;
#pragma unroll
    for (int i = 0; i < 16; ++i) y[i] = x[i] * f;
    return y;
}

constexpr int kDqWaves = 4;
constexpr int kDqRows = 32 * kDqWaves;
constexpr int kDqKeys = 32;

template <class T, int D, bool kVec>
__global__ __launch_bounds__(64 * kDqWaves, 2) void attention_dq_kernel(attention_emu_backward_t a,
                                                                     int64_t first_block) {
    using KV = Tile<T, D>;
    constexpr int kThreads = 64 * kDqWaves, kBlocks = D / kBlock<T>, kParts = 32 / kBlock<T>;
    constexpr int kTileBytes = kDqKeys * D * (int)sizeof(T);
    __shared__ __attribute__((aligned(16))) char lds[4 * kTileBytes];
    const int group = a.q_heads / a.k_heads;
    const bool packed = a.cu_seqlens != nullptr;
    const int64_t block = first_block + blockIdx.x;
    int n, head, tile;
    if (packed) {
        head = (int)(block % a.k_heads);
        const Place p = find_part(a.cu_seqlens, a.batch, a.tokens, group, kDqRows,
                                  (int)(block / a.k_heads));
        if (!p.found) return;
        n = p.n, tile = p.tile;
    } else {
        const int pairs = a.batch * a.k_heads;
        const int tiles = (a.tokens * group + kDqRows - 1) / kDqRows;
        const int pair = (int)(block % pairs);
        n = pair / a.k_heads, head = pair % a.k_heads;
        tile = tiles - 1 - (int)(block / pairs);
    }
    const Span sq = span_of(a.cu_seqlens, n, a.tokens);
    const Span sk = span_of(a.cu_keys, n, a.keys);
    const int rows = sq.count * group, last_row = rows - 1;
    const T* k = row_of<T>(a.k, packed, n, sk, head);
    const T* v = row_of<T>(a.v, packed, n, sk, head);

    const int lane = threadIdx.x & 63, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row0 = tile * kDqRows, wave_row = row0 + 32 * wave;
    const int row = wave_row + (lane & 31);
    const int r = min(row, last_row), token = r / group, h = head * group + r % group;
    const bool valid = row < rows;
    Frag<T> Q[kBlocks], DO[kBlocks];
    float delta = 0.0f;
    {
        const T* q = row_of<T>(a.q, packed, n, sq, h) + token * a.q.token;
        const T* o = row_of<T>(a.o, packed, n, sq, h) + token * a.o.token;
        const T* d = row_of<T>(a.d_o, packed, n, sq, h) + token * a.d_o.token;
#pragma unroll
        for (int kb = 0; kb < kBlocks; ++kb) {
            Q[kb] = load_chunk<T, kVec>(q, 2 * kb + half, a.size, valid);
            DO[kb] = load_chunk<T, kVec>(d, 2 * kb + half, a.size, valid);
            const Frag<T> x = load_chunk<T, kVec>(o, 2 * kb + half, a.size, valid);
#pragma unroll
            for (int j = 0; j < kPer<T>; ++j)
                delta = __builtin_fmaf(to_f32(DO[kb][j]), to_f32(x[j]), delta);
        }
        delta = sum_halves(delta);
    }
    const int64_t out_row = (packed ? sq.first : (int64_t)n * a.tokens) + token;
    if (valid && half == 0) static_cast<float*>(a.workspace)[out_row * a.q_heads + h] = delta;
    // (rows that see nothing have lse -infinity)
    float z = __builtin_inff();
    if (valid) {
        const float lse = row_of<float>(a.lse, packed, n, sq, h)[token * a.lse.token];
        if (lse != -__builtin_inff()) z = lse * kLog2e;
    }
    const float c = a.scale * kLog2e;
    const int shift = sk.count - sq.count + 1;
    const auto seen = [&](int r) {
        return a.causal ? min(max(min(r, last_row) / group + shift, 0), sk.count) : sk.count;
    };
    const int lim = seen(row), lim_min = seen(wave_row), lim_max = seen(wave_row + 31);
    const int count = (seen(row0 + kDqRows - 1) + kDqKeys - 1) / kDqKeys;

    f32x16 dQ[D / 32];
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt) dQ[dt] = f32x16{};
    Fit fit;
    Staged<T, D, kDqKeys, kThreads, kVec> st_k, st_v;
    const auto load = [&](int t) {
        st_k.load(k, a.k.token, t * kDqKeys, sk.count, a.size, threadIdx.x);
        st_v.load(v, a.v.token, t * kDqKeys, sk.count, a.size, threadIdx.x);
    };
    if (count > 0) load(0);
    for (int t = 0; t < count; ++t) {
        char* kt = lds + (t & 1) * 2 * kTileBytes;
        char* vt = kt + kTileBytes;
        st_k.store(kt, threadIdx.x);
        st_v.store(vt, threadIdx.x);
        if (t + 1 < count) load(t + 1);
        lds_barrier();
        const int key0 = t * kDqKeys;
        if (key0 >= lim_max) continue;
        f32x16 S{}, dP;
#pragma unroll
        for (int i = 0; i < 16; ++i) dP[i] = -delta;
#pragma unroll
        for (int kb = 0; kb < kBlocks; ++kb) {
            S = mma(KV::along(kt, 0, kb, lane), Q[kb], S);
            dP = mma(KV::along(vt, 0, kb, lane), DO[kb], dP);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i)
            dP[i] *= __builtin_amdgcn_exp2f(__builtin_fmaf(S[i], c, -z));
        if (key0 + kDqKeys > lim_min) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (key0 + acc_row(i, half) >= lim) dP[i] = 0.0f;
        }
        if constexpr (kNarrow<T>) {
            fit.fit(dP, dQ);
            dP = times(dP, fit.f);
        }
#pragma unroll
        for (int kb = 0; kb < kParts; ++kb) {
            const Frag<T> x = operand<T>(dP, kb);
#pragma unroll
            for (int dt = 0; dt < D / 32; ++dt)
                dQ[dt] = mma(KV::across(kt, kb, 32 * dt, lane), x, dQ[dt]);
        }
    }
    if (!valid) return;
    const float f = kNarrow<T> ? a.scale / fit.f : a.scale;
    T* dq = row_of<T>(a.dq, packed, n, sq, h) + token * a.dq.token;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
            store_four<T, kVec>(dq, 32 * dt + acc_row(i, half), a.size, dQ[dt][i] * f,
                                dQ[dt][i + 1] * f, dQ[dt][i + 2] * f, dQ[dt][i + 3] * f);
}

constexpr int kDkvWaves = 4;
constexpr int kDkvKeys = 32 * kDkvWaves;
constexpr int kDkvRows = 32;

template <class T, int D, bool kVec>
__global__ __launch_bounds__(64 * kDkvWaves, 2) void attention_dkv_kernel(attention_emu_backward_t a,
                                                                       int64_t first_block) {
    using QD = Tile<T, D>;
    constexpr int kThreads = 64 * kDkvWaves, kBlocks = D / kBlock<T>, kParts = 32 / kBlock<T>;
    constexpr int kTileBytes = kDkvRows * D * (int)sizeof(T);
    constexpr int kChunks = QD::kChunks, kEach = kDkvRows * kChunks / kThreads;
    // (the weights' shift; FP16 only)
    constexpr float kShift = kNarrow<T> ? 14.0f : 0.0f, kBack = kNarrow<T> ? 0x1p-14f : 1.0f;
    struct Row {
        float z[kDkvRows], delta[kDkvRows];
        int seen[kDkvRows];
    };
    __shared__ __attribute__((aligned(16))) char lds[4 * kTileBytes];
    __shared__ __attribute__((aligned(16))) Row of_rows[2];
    const int group = a.q_heads / a.k_heads;
    const bool packed = a.cu_seqlens != nullptr;
    const int64_t block = first_block + blockIdx.x;
    int n, head, tile;
    if (packed) {
        head = (int)(block % a.k_heads);
        const Place p =
            find_part(a.cu_keys, a.batch, a.keys, 1, kDkvKeys, (int)(block / a.k_heads));
        if (!p.found) return;
        n = p.n, tile = p.tile;
    } else {
        // the first keys of all sequences first: with a causal mask they take longest
        const int pairs = a.batch * a.k_heads;
        const int pair = (int)(block % pairs);
        n = pair / a.k_heads, head = pair % a.k_heads;
        tile = (int)(block / pairs);
    }
    const Span sq = span_of(a.cu_seqlens, n, a.tokens);
    const Span sk = span_of(a.cu_keys, n, a.keys);
    const int rows = sq.count * group;
    const int lane = threadIdx.x & 63, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int block_key = tile * kDkvKeys, wave_key = block_key + 32 * wave;
    const int key = wave_key + (lane & 31);
    const bool valid = key < sk.count;
    const int key_in = min(key, sk.count - 1);
    Frag<T> K[kBlocks], V[kBlocks];
    {
        const T* k = row_of<T>(a.k, packed, n, sk, head) + key_in * a.k.token;
        const T* v = row_of<T>(a.v, packed, n, sk, head) + key_in * a.v.token;
#pragma unroll
        for (int kb = 0; kb < kBlocks; ++kb) {
            K[kb] = load_chunk<T, kVec>(k, 2 * kb + half, a.size, valid);
            V[kb] = load_chunk<T, kVec>(v, 2 * kb + half, a.size, valid);
        }
    }
    const int shift = sk.count - sq.count + 1;
    // the first row that sees the block's first key, the wave's first and last one
    const auto first_row = [&](int key) {
        return a.causal ? min(max(key - shift + 1, 0), sq.count) * group : 0;
    };
    const int t0 = first_row(block_key) / kDkvRows;
    const int count = (rows + kDkvRows - 1) / kDkvRows;
    const int wave_from = first_row(wave_key), wave_all = first_row(wave_key + 31);

    f32x16 dK[D / 32], dV[D / 32];
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt) dK[dt] = f32x16{}, dV[dt] = f32x16{};
    Fit fit;

    const int my_chunk = threadIdx.x % kChunks, my_row = threadIdx.x / kChunks;
    const T* q0 = row_of<T>(a.q, packed, n, sq, head * group);
    const T* d0 = row_of<T>(a.d_o, packed, n, sq, head * group);
    const float* lse0 = row_of<float>(a.lse, packed, n, sq, head * group);
    const float* delta0 = static_cast<const float*>(a.workspace) +
                          (packed ? sq.first : (int64_t)n * a.tokens) * a.q_heads + head * group;
    Frag<T> st_q[kEach], st_d[kEach];
    float st_z = 0.0f, st_delta = 0.0f;
    int st_seen = 0;
    const auto load = [&](int t) {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int row = t * kDkvRows + my_row + i * (kThreads / kChunks);
            const int r = min(row, rows - 1), token = r / group, h = r % group;
            st_q[i] = load_chunk<T, kVec>(q0 + token * a.q.token + h * a.q.head, my_chunk, a.size,
                                          row < rows);
            st_d[i] = load_chunk<T, kVec>(d0 + token * a.d_o.token + h * a.d_o.head, my_chunk,
                                          a.size, row < rows);
        }
        if (threadIdx.x < kDkvRows) {
            const int row = t * kDkvRows + threadIdx.x;
            const int r = min(row, rows - 1), token = r / group, h = r % group;
            const float lse = lse0[token * a.lse.token + h * a.lse.head];
            const bool sees = row < rows && lse != -__builtin_inff();
            st_z = sees ? lse * kLog2e - kShift : __builtin_inff();
            st_delta = row < rows ? delta0[(int64_t)token * a.q_heads + h] : 0.0f;
            st_seen = a.causal ? token + shift : sk.count;
        }
    };
    if (t0 < count) load(t0);
    const float c = a.scale * kLog2e;
    for (int t = t0; t < count; ++t) {
        char* qt = lds + (t & 1) * 2 * kTileBytes;
        char* dt_ = qt + kTileBytes;
        Row& rw = of_rows[t & 1];
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int at = QD::at(my_row + i * (kThreads / kChunks), my_chunk);
            *reinterpret_cast<Frag<T>*>(qt + at) = st_q[i];
            *reinterpret_cast<Frag<T>*>(dt_ + at) = st_d[i];
        }
        if (threadIdx.x < kDkvRows) {
            rw.z[threadIdx.x] = st_z;
            rw.delta[threadIdx.x] = st_delta;
            rw.seen[threadIdx.x] = st_seen;
        }
        if (t + 1 < count) load(t + 1);
        lds_barrier();
        if ((t + 1) * kDkvRows <= wave_from) continue;
        f32x16 S{}, dP;
#pragma unroll
        for (int i = 0; i < 16; ++i) dP[i] = -rw.delta[acc_row(i, half)];
#pragma unroll
        for (int kb = 0; kb < kBlocks; ++kb) {
            S = mma(QD::along(qt, 0, kb, lane), K[kb], S);
            dP = mma(QD::along(dt_, 0, kb, lane), V[kb], dP);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            S[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(S[i], c, -rw.z[acc_row(i, half)]));
            dP[i] *= S[i];
        }
        if (t * kDkvRows < wave_all) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (key >= rw.seen[acc_row(i, half)]) S[i] = 0.0f, dP[i] = 0.0f;
        }
        if constexpr (kNarrow<T>) {
            fit.fit(dP, dK);
            dP = times(dP, fit.f);
        }
#pragma unroll
        for (int kb = 0; kb < kParts; ++kb) {
            const Frag<T> p = operand<T>(S, kb), x = operand<T>(dP, kb);
#pragma unroll
            for (int dt = 0; dt < D / 32; ++dt) {
                dV[dt] = mma(QD::across(dt_, kb, 32 * dt, lane), p, dV[dt]);
                dK[dt] = mma(QD::across(qt, kb, 32 * dt, lane), x, dK[dt]);
            }
        }
    }
    if (!valid) return;
    const float fk = kNarrow<T> ? a.scale * kBack / fit.f : a.scale;
    T* dk = row_of<T>(a.dk, packed, n, sk, head) + key * a.dk.token;
    T* dv = row_of<T>(a.dv, packed, n, sk, head) + key * a.dv.token;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const int d = 32 * dt + acc_row(i, half);
            store_four<T, kVec>(dk, d, a.size, dK[dt][i] * fk, dK[dt][i + 1] * fk,
                                dK[dt][i + 2] * fk, dK[dt][i + 3] * fk);
            store_four<T, kVec>(dv, d, a.size, dV[dt][i] * kBack, dV[dt][i + 1] * kBack,
                                dV[dt][i + 2] * kBack, dV[dt][i + 3] * kBack);
        }
}

}  // namespace

int64_t attention_backward_workspace(const attention_emu_backward_t& a) {
    const int64_t rows = a.cu_seqlens != nullptr ? a.tokens : (int64_t)a.batch * a.tokens;
    return (rows * a.q_heads * 4 + 255) / 256 * 256;
}

hipError_t launch_attention_backward(const attention_emu_backward_t& args, hipStream_t stream) {
    attention_emu_backward_t a = args;
    if (a.cu_seqlens != nullptr && a.cu_keys == nullptr) a.cu_keys = a.cu_seqlens;
    const int e = a.dtype == SGEMM_EMU_F32 ? 4 : 2;
    bool vec = a.size * e % 16 == 0;
    for (const sgemm_emu_view_t* x : {&a.q, &a.k, &a.v, &a.o, &a.d_o, &a.dq, &a.dk, &a.dv})
        vec = vec && rows_aligned16(*x, e);
    const bool packed = a.cu_seqlens != nullptr;
    const int64_t group = a.q_heads / a.k_heads;
    const int64_t q_parts = most_parts(a.batch, a.tokens * group, kDqRows, packed) * a.k_heads;
    const int64_t k_parts = most_parts(a.batch, a.keys, kDkvKeys, packed) * a.k_heads;
    return by_form(a.dtype, a.size, vec, [&](auto t, auto d, auto vec) {
        using T = decltype(t);
        constexpr int D = decltype(d)::value;
        constexpr bool kVec = decltype(vec)::value != 0;
        if (a.tokens > 0)
            if (hipError_t e = launch_blocks(attention_dq_kernel<T, D, kVec>, q_parts, 64 * kDqWaves,
                                             0, stream, a))
                return e;
        return launch_blocks(attention_dkv_kernel<T, D, kVec>, k_parts, 64 * kDkvWaves, 0, stream, a);
    });
}

}  // namespace sgemm_emu
