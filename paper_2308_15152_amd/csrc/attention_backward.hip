// The gradient of attention over whole sequences, in two kernels without atomics:
//   attention_dq_kernel   a block has query rows and goes over the keys they see: dq, and
//                         delta_i = do_i o_i into the workspace;
//   attention_dkv_kernel  a block has keys and goes over the query rows (of all of the
//                         key head's query heads) that see them: dk and dv.
// Both form p = 2^(c s - z) again from the scores, c = scale log2 e, z = lse log2 e, and
// dp - delta in the accumulators of do v^T, which start at -delta.  Seven products of 2 D
// operations a pair instead of the five that one pass with shared sums would take, for sums
// whose order is fixed.  Bound by the matrix instructions and the reads of operands from LDS:
// 2 x 4096 causal tokens, 16 heads of 128 in bfloat16, 517 us (545 on another machine), of which dq
// 205 (1005 TFLOP/s) and dk and dv 306 (898).  With 16-byte chunks out of LDS permuted so that no two of a read meet on
// a bank, and addresses formed again for each tile instead of reloaded from scratch (a reload
// waits for the tile's loads, too), dk and dv took 1340 -> 620; with keys and values, whose
// registers did not suffice, partly in LDS, and two waves for each SIMD, 314.
//
// Weights p and ds are rounded to the inputs' type as operands.  FP16 has no room for
// either: p is taken times 2^14, and ds times a power of two for each column of the
// accumulator (a query row, or a key), which is lowered, with what is summed so far, when a
// larger value comes.
#include <algorithm>

#include "attention_parts.hpp"
#include "attention_split.h"

namespace sgemm_emu {

namespace {

template <class T>
constexpr bool kNarrow = __is_same(Elem<T>, f16_t);

struct BackwardArgs {
    attention_emu_backward_t a;
    float* delta;  // [token in all][query head]
    // the operands, split if they are FP32
    sgemm_emu_view_t q, k, v, d_o;
    const float *q_factors, *k_factors, *v_factors, *do_factors;
    // parts that the query rows of a block of keys are cut into, and where they leave their sums:
    // [part][dv, dk][key in all][key head][kPartStride], or null: one part
    int count;
    float* parts;
    int64_t key_rows;
};

__device__ inline Pack<float, 4>::type four_floats(const float* p) {
    return *reinterpret_cast<const Pack<float, 4>::type*>(p);
}

// For the scheduler: kinds of instructions, and f of 0 .. n - 1 as constants.
constexpr int kMatrix = 0x8, kLdsRead = 0x100;

template <int n, int i = 0, class F>
__device__ inline __attribute__((always_inline)) void schedule_steps(F f) {
    if constexpr (i < n) {
        f(Number<i>{});
        schedule_steps<n, i + 1>(f);
    }
}

// From |z| = kCoarse on a weight p = 2^(c s - z) may be off by factors, for z's last bit comes to be
// no longer small beside one: it is taken as one at most there, and NaN stays.
constexpr float kCoarse = 0x1p16f;

constexpr int kDqWaves = 4;
constexpr int kDqRows = 32 * kDqWaves;
constexpr int kDqKeys = 32;
constexpr int kFewKeys = 128;
// A row's weights are taken to be all there if they sum to one up to this, and if the sum of ds is
// no more than a step of what o's roundings explain, of itself and of the weights that made it, by
// half a step each: keys that are elsewhere may weigh next to nothing and still make up all
// of delta.  (|ds| is summed by pairs of keys, which takes half as long: 0.4% of the time.)
constexpr float kWhole = 0x1p-12f;
template <class T>
constexpr float kStep = __is_same(T, bf16_t) ? 0x1p-7f : 0x1p-10f;
// Below so many blocks (two for each CU) two groups of waves share a block's keys: the gradient with
// 384 blocks of 2048 keys takes 192 us for 203, that of 16 packed sequences, 2500 tokens in all, 112
// for 127; with 512 blocks it would take 3 us more than without.
constexpr int kDqPaired = 512;

// (FP32 operands of more than 96 elements take the registers of two waves)
// kGroups groups of waves take every kGroups-th tile of keys and are joined at the end.
template <class T, int D, bool kVec, int kGroups>
__global__ __launch_bounds__(64 * kDqWaves * kGroups,
                             kPlanes<T> == 2 && D > 96 ? kGroups : 2) void
attention_dq_kernel(BackwardArgs args, int first_block) {
    typedef Elem<T> E;
    using KV = Planes<T, D, kDqKeys>;
    constexpr bool kSplit = kPlanes<T> == 2;
    constexpr int kThreads = 64 * kDqWaves, kBlocks = D / kBlock<E>, kParts = 32 / kBlock<E>;
    constexpr int kTileBytes = KV::kBytes;
    constexpr int kJoin = (kGroups - 1) * kDqWaves * D / 8 * 1024;
    constexpr int kTiles = kGroups * 4 * kTileBytes;
    __shared__ __attribute__((aligned(16))) char lds_all[kTiles > kJoin ? kTiles : kJoin];
    // factors of keys and values
    __shared__ float of_all[kSplit ? kGroups * 4 * kDqKeys : 1];
    const attention_emu_backward_t& a = args.a;
    const int group = a.q_heads / a.k_heads;
    const bool packed = a.cu_seqlens != nullptr;
    const int block = first_block + (int)blockIdx.x;
    int n, head, tile;
    if (packed) {
        head = block % a.k_heads;
        const Place p = find_part(a.cu_seqlens, a.batch, a.tokens, group, kDqRows,
                                  block / a.k_heads);
        if (!p.found) return;
        n = p.n, tile = p.tile;
    } else {
        const int pairs = a.batch * a.k_heads;
        const int tiles = (a.tokens * group + kDqRows - 1) / kDqRows;
        const int pair = block % pairs;
        n = pair / a.k_heads, head = pair % a.k_heads;
        tile = tiles - 1 - block / pairs;
    }
    const Span sq = span_of(a.cu_seqlens, n, a.tokens);
    const Span sk = span_of(a.cu_keys, n, a.keys);
    const int rows = sq.count * group, last_row = rows - 1;
    const E* k = row_of<E>(args.k, packed, n, sk, head);
    const E* v = row_of<E>(args.v, packed, n, sk, head);

    const int lane = threadIdx.x & 63, half = lane >> 5;
    const int all_waves = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int group_of = all_waves / kDqWaves, wave = all_waves % kDqWaves;
    const int thread = (int)threadIdx.x % kThreads;  // in the group
    char* const lds = lds_all + group_of * 4 * kTileBytes;
    float* const of_tiles = of_all + (kSplit ? group_of * 4 * kDqKeys : 0);
    const int row0 = tile * kDqRows, wave_row = row0 + 32 * wave;
    const int row = wave_row + (lane & 31);
    const int r = min(row, last_row), token = r / group, h = head * group + r % group;
    const bool valid = row < rows;
    const int64_t in_all = (packed ? sq.first : (int64_t)n * a.tokens) + token;
    Operand<T> Q[kBlocks], DO[kBlocks];
    float delta = 0.0f, of_delta = 0.0f;  // and the sum of its terms' magnitudes
    {
        const E* q = row_of<E>(args.q, packed, n, sq, h) + token * args.q.token;
        const E* x = row_of<E>(args.d_o, packed, n, sq, h) + token * args.d_o.token;
        const Out<T>* o = row_of<Out<T>>(a.o, packed, n, sq, h) + token * a.o.token;
        const Out<T>* d = row_of<Out<T>>(a.d_o, packed, n, sq, h) + token * a.d_o.token;
#pragma unroll
        for (int kb = 0; kb < kBlocks; ++kb) {
            Q[kb] = load_operand<T, D, kVec>(q, 2 * kb + half, a.size, valid);
            DO[kb] = load_operand<T, D, kVec>(x, 2 * kb + half, a.size, valid);
        }
#pragma unroll
        for (int kb = 0; kb < D / kBlock<Out<T>>; ++kb) {
            const Frag<Out<T>> x = load_chunk<Out<T>, kVec>(o, 2 * kb + half, a.size, valid);
            const Frag<Out<T>> y = load_chunk<Out<T>, kVec>(d, 2 * kb + half, a.size, valid);
#pragma unroll
            for (int j = 0; j < kPer<Out<T>>; ++j) {
                const float term = to_f32(x[j]) * to_f32(y[j]);
                delta += term;
                of_delta += __builtin_fabsf(term);
            }
        }
        delta = sum_halves(delta);
        of_delta = sum_halves(of_delta);
    }
    // (rows that see nothing have lse -infinity)
    float z = __builtin_inff();
    if (valid) {
        const float lse = row_of<float>(a.lse, packed, n, sq, h)[token * a.lse.token];
        if (lse != -__builtin_inff()) z = lse * kLog2e;
    }
    const bool coarse = __builtin_fabsf(z) >= kCoarse, any_coarse = __any(coarse && valid);
    // what the row's q and do have been divided by
    float q_factor = 1.0f, do_factor = 1.0f;
    if constexpr (kSplit) {
        q_factor = args.q_factors[in_all * a.q_heads + h];
        do_factor = args.do_factors[in_all * a.q_heads + h];
    }
    // (factors multiply a product at once: one alone may take it past FP32's range)
    const float c = kSplit ? 1.0f : a.scale * kLog2e;
    const float of_scores = a.scale * kLog2e * q_factor;
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
    // (what is not loaded multiplies zeros and has to be finite)
    clear_lds(lds, 4 * kTileBytes, thread, kThreads);
    lds_barrier();
    Flow<E, D, kDqKeys, kThreads, kVec || kSplit> fk, fv;
    const int width = kSplit ? kWidth<D> : a.size;
    const uint32_t k_row = (uint32_t)args.k.token * sizeof(E);
    const uint32_t v_row = (uint32_t)args.v.token * sizeof(E);
    const int64_t first_key = (packed ? sk.first : (int64_t)n * a.keys) * a.k_heads + head;
    float st_factor = 0.0f;
    fk.rows([&](int r) { return r * k_row; }, thread);
    fv.rows([&](int r) { return r * v_row; }, thread);
    const auto load = [&](int t) {
        const int key = t * kDqKeys, most = sk.count - 1 - key;
        char* to = lds + (t / kGroups & 1) * 2 * kTileBytes;
        const auto there = [&](int, int r) { return r <= most; };
        if constexpr (kSplit) {
            const int i = thread % kDqKeys;
            if (thread < 2 * kDqKeys)
                st_factor = i > most ? 0.0f
                                     : (thread < kDqKeys ? args.k_factors : args.v_factors)
                                           [first_key + (int64_t)(key + i) * a.k_heads];
        }
#pragma unroll
        for (int i = 0; i < kPlanes<T>; ++i) {
            fk.start(to + i * KV::kPlaneBytes, k + key * args.k.token + i * kWidth<D>, width,
                     thread, there);
            fv.start(to + kTileBytes + i * KV::kPlaneBytes, v + key * args.v.token + i * kWidth<D>,
                     width, thread, there);
        }
    };
    const typename KV::Read read(lds, lane);
    float weight = 0.0f, rest = 0.0f, size_of_rest = 0.0f;  // sums of the row's p, ds and |ds|
    // one tile, in the first or the second place
    const auto step = [&](int t, auto odd, auto only_rest) __attribute__((always_inline)) {
        constexpr int k_at = decltype(odd)::value * 2 * kTileBytes, v_at = k_at + kTileBytes;
        char* kt = lds + k_at;
        char* vt = lds + v_at;
        // (the last group may have one tile less, and comes to the barrier all the same)
        const bool here = kGroups == 1 || t < count;
        float* const of_tile = of_tiles + decltype(odd)::value * 2 * kDqKeys;
        if (here) {
            fk.finish(kt, thread);
            fv.finish(vt, thread);
            if (kSplit && thread < 2 * kDqKeys) of_tile[thread] = st_factor;
        }
        lds_barrier();
        if (t + kGroups < count) load(t + kGroups);
        if (!here) return;
        const int key0 = t * kDqKeys;
        if (key0 >= lim_max) return;
        f32x16 S{}, dP;
#pragma unroll
        for (int i = 0; i < 16; ++i) dP[i] = kSplit ? 0.0f : -delta;
#pragma unroll
        for (int kb = 0; kb < kBlocks; ++kb) {
            S = mma(KV::along(read, k_at, kb), Q[kb], S);
            dP = mma(KV::along(read, v_at, kb), DO[kb], dP);
        }
        f32x16 by;  // the keys' factors
        if constexpr (kSplit) {
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const auto x = four_floats(of_tile + 8 * (i / 4) + 4 * half);
                const auto y = four_floats(of_tile + kDqKeys + 8 * (i / 4) + 4 * half);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    by[i + j] = x[j];
                    S[i + j] *= x[j] * of_scores;
                    dP[i + j] = __builtin_fmaf(dP[i + j], y[j] * do_factor, -delta);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) S[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(S[i], c, -z));
        // (for all weights, where they are formed, the one takes 1.5% of the time)
        if (key0 + kDqKeys > lim_min || any_coarse) {
            const float most = coarse ? 1.0f : __builtin_inff();
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                S[i] = __builtin_elementwise_minimum(S[i], most);
                if (key0 + acc_row(i, half) >= lim) S[i] = dP[i] = 0.0f;
            }
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) dP[i] *= S[i];
        if constexpr (kSplit) {
#pragma unroll
            for (int i = 0; i < 16; ++i) dP[i] *= by[i];
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) weight += S[i];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float two = dP[i] + dP[i + 8];
                rest += two, size_of_rest += __builtin_fabsf(two);
            }
        }
        if constexpr (decltype(only_rest)::value != 0) return;
        if constexpr (kNarrow<T>) {
            fit.fit(largest(dP), dQ);
            dP = times(dP, fit.f);
        }
#pragma unroll
        for (int kb = 0; kb < kParts; ++kb) {
            const Operand<T> x = operand<T>(dP, kb);
#pragma unroll
            for (int dt = 0; dt < D / 32; ++dt)
                dQ[dt] = mma(KV::across(read, k_at, kb, dt), x, dQ[dt]);
        }
    };
    const auto pass = [&](auto only_rest) __attribute__((always_inline)) {
        weight = rest = size_of_rest = 0.0f;
        if (group_of < count) load(group_of);
        for (int t = group_of; t < count + group_of; t += 2 * kGroups) {
            step(t, Number<0>{}, only_rest);
            if (t + kGroups < count + group_of) step(t + kGroups, Number<1>{}, only_rest);
        }
        if constexpr (!kSplit) {
            weight = sum_halves(weight);
            rest = sum_halves(rest);
            size_of_rest = sum_halves(size_of_rest);
            if constexpr (kGroups == 2) {
                __shared__ float sums[2][3][kDqRows];
                const int at = 32 * wave + (lane & 31);
                if (half == 0) {
                    sums[group_of][0][at] = weight, sums[group_of][1][at] = rest;
                    sums[group_of][2][at] = size_of_rest;
                }
                __syncthreads();
                weight = sums[0][0][at] + sums[1][0][at];
                rest = sums[0][1][at] + sums[1][1][at];
                size_of_rest = sums[0][2][at] + sums[1][2][at];
            }
            // (sum p |do v| <= sum |ds| + |delta|)
            if (__builtin_fabsf(weight - 1.0f) < kWhole &&
                __builtin_fabsf(rest) <=
                    kStep<E> * (of_delta + size_of_rest + __builtin_fabsf(delta)))
                delta += rest;
            // (the places are free for the next pass)
            __syncthreads();
        }
    };
    // Where a row's weights sum to one (o and lse may be of more keys than are given), its ds sum
    // to zero but for the error of delta, which is that of an o of 8 or 11 bits.  dk is formed
    // with delta put right by it (FP16, 1000 keys: an error of 2.9e-4 for 3.1e-4; 526 -> 530 us
    // for 4096 tokens).  In dq it matters where keys are few (bfloat16, 30 keys: 2.3e-3 for
    // 3.1e-3; 500 keys: 2.35e-3 for 2.5e-3): there it is found beforehand (32 sequences of 64
    // tokens 38.5 -> 40 us; with 512 keys it would be 251 -> 288).
    if constexpr (!kSplit) {
        if (count * kDqKeys <= kFewKeys) pass(Number<1>{});
    }
    pass(Number<0>{});
    if (valid && half == 0 && group_of == 0) args.delta[in_all * a.q_heads + h] = delta;
    const float f = kNarrow<T> ? inverse_of_power(fit.f) : 1.0f;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt) dQ[dt] = times(dQ[dt], a.scale);
    if constexpr (kGroups == 2) {
        typedef Pack<float, 4>::type Four;
        Four* const sums = reinterpret_cast<Four*>(lds_all) + wave * (D / 8 * 64) + lane;
        __syncthreads();
        if (group_of == 1) {
#pragma unroll
            for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    sums[(4 * dt + i) * 64] = Four{dQ[dt][4 * i], dQ[dt][4 * i + 1],
                                                   dQ[dt][4 * i + 2], dQ[dt][4 * i + 3]} * f;
        }
        __syncthreads();
        if (group_of == 1 || !valid) return;
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const Four x = sums[(4 * dt + i) * 64];
#pragma unroll
                for (int j = 0; j < 4; ++j) dQ[dt][4 * i + j] = dQ[dt][4 * i + j] * f + x[j];
            }
    }
    if (!valid) return;
    const float by = kGroups == 2 ? 1.0f : f;
    Out<T>* dq = row_of<Out<T>>(a.dq, packed, n, sq, h) + token * a.dq.token;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
            store_four<Out<T>, kVec>(dq, 32 * dt + acc_row(i, half), a.size, dQ[dt][i] * by,
                                dQ[dt][i + 1] * by, dQ[dt][i + 2] * by, dQ[dt][i + 3] * by);
}

// A block's waves: kKeyGroups times 32 keys, each shared by kRowGroups waves that take
// 32 query rows of a tile each and are joined at the end.  As many waves as two for each SIMD,
// where registers and LDS hold them (not with FP32 of more than 64 elements).
template <class T, int D>
struct DkvShape {
    static constexpr bool kWide = kPlanes<T> == 2 && D > 64;
    static constexpr int kKeyGroups = 2;
    static constexpr int kRowGroups = kWide ? 2 : 4;
    static constexpr int kWaves = kKeyGroups * kRowGroups, kThreads = 64 * kWaves;
    // tiles of 32 rows that a wave takes between two barriers: two where they are small (32
    // sequences of 512 tokens with heads of 64 147 -> 142 us, 16 packed ones 125 -> 122)
    static constexpr int kUnits = kPlanes<T> == 1 && D <= 64 ? 2 : 1;
    static constexpr int kKeys = 32 * kKeyGroups, kRows = 32 * kRowGroups * kUnits;
    // How much of the keys' and values' operands is in registers; the rest, which
    // does not fit, is read from LDS for every tile
    static constexpr int kBlocks = D / kBlock<Elem<T>>;
    static constexpr bool kFull = kPlanes<T> == 1 && D > 96;
    static constexpr int kKeyBlocks = kFull ? kBlocks / 2 : kBlocks;
    static constexpr int kValueBlocks = kFull ? 0 : kBlocks;
    static constexpr int kLdsBlocks = 2 * kBlocks - kKeyBlocks - kValueBlocks;
};

// The query rows of a key head in tiles: `tokens` tokens with `heads` of their `group` query
// heads each, `parts` tiles for all of those.  One head to a tile where heads are so far
// apart that distances within a token pass 32 bits.
struct RowTiles {
    int tokens, heads, parts;
    __device__ inline RowTiles(int group, int rows, bool far)
        : tokens(far ? rows : max(rows / group, 1)),
          heads(far ? 1 : min(group, rows)),
          parts((group + heads - 1) / heads) {}
};

template <class T, int D, bool kVec, class Shape = DkvShape<T, D>>
__global__ __launch_bounds__(Shape::kThreads, Shape::kWaves / 4) void attention_dkv_kernel(
    BackwardArgs args, int first_block) {
    typedef Elem<T> E;
    const attention_emu_backward_t& a = args.a;
    constexpr bool kSplit = kPlanes<T> == 2;
    constexpr int kThreads = Shape::kThreads, kRows = Shape::kRows, kRowGroups = Shape::kRowGroups;
    using QD = Planes<T, D, kRows>;
    constexpr int kBlocks = D / kBlock<E>, kParts = 32 / kBlock<E>;
    constexpr int kTileBytes = QD::kBytes, kRowBytes = QD::One::kRowBytes;
    // (the weights' shift; FP16 only)
    constexpr float kShift = kNarrow<T> ? 14.0f : 0.0f, kBack = kNarrow<T> ? 0x1p-14f : 1.0f;
    struct Row {
        float z[kRows], delta[kRows];
        int seen[kRows];
        float q[kSplit ? kRows : 4], d_o[kSplit ? kRows : 4];  // factors
    };
    constexpr int kJoin = (kRowGroups - 1) * Shape::kKeyGroups * D / 32 * 4096;
    constexpr int kLds = 4 * kTileBytes > kJoin ? 4 * kTileBytes : kJoin;
    __shared__ __attribute__((aligned(16))) char lds[kLds];
    __shared__ __attribute__((aligned(16))) Row of_rows[2];
    // [key group][block][lane]
    __shared__ Operand<T>
        operands[Shape::kLdsBlocks > 0 ? Shape::kKeyGroups * Shape::kLdsBlocks * 64 : 1];
    const int group = a.q_heads / a.k_heads;
    const bool packed = a.cu_seqlens != nullptr;
    const int part = (first_block + (int)blockIdx.x) % args.count;
    const int block = (first_block + (int)blockIdx.x) / args.count;
    int n, head, tile;
    if (packed) {
        head = block % a.k_heads;
        const Place p = find_part(a.cu_keys, a.batch, a.keys, 1, Shape::kKeys, block / a.k_heads);
        if (!p.found) return;
        n = p.n, tile = p.tile;
    } else {
        // the first keys of all sequences first: with a causal mask they take longest
        const int pairs = a.batch * a.k_heads;
        const int pair = block % pairs;
        n = pair / a.k_heads, head = pair % a.k_heads;
        tile = block / pairs;
    }
    const Span sq = span_of(a.cu_seqlens, n, a.tokens);
    const Span sk = span_of(a.cu_keys, n, a.keys);
    const int tokens = sq.count;
    const int thread = threadIdx.x, lane = thread & 63, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(thread >> 6);
    const int row_group = wave % kRowGroups, key_group = wave / kRowGroups;
    const int block_key = tile * Shape::kKeys, wave_key = block_key + 32 * key_group;
    const int key = wave_key + (lane & 31);
    const bool valid = key < sk.count;
    const int key_in = min(key, sk.count - 1);
    constexpr int kKeyBlocks = Shape::kKeyBlocks, kValueBlocks = Shape::kValueBlocks;
    Operand<T> K[kKeyBlocks], V[kValueBlocks > 0 ? kValueBlocks : 1];
    Operand<T>* const more = operands + key_group * Shape::kLdsBlocks * 64 + lane;
    {
        const E* k = row_of<E>(args.k, packed, n, sk, head) + key_in * args.k.token;
        const E* v = row_of<E>(args.v, packed, n, sk, head) + key_in * args.v.token;
#pragma unroll
        for (int kb = 0; kb < kBlocks; ++kb) {
            const Operand<T> x = load_operand<T, D, kVec>(k, 2 * kb + half, a.size, valid);
            const Operand<T> y = load_operand<T, D, kVec>(v, 2 * kb + half, a.size, valid);
            if (kb < kKeyBlocks)
                K[kb] = x;
            else if (row_group == 0)
                more[(kb - kKeyBlocks) * 64] = x;
            if (kb < kValueBlocks)
                V[kb] = y;
            else if (row_group == 0)
                more[(kBlocks - kKeyBlocks + kb - kValueBlocks) * 64] = y;
        }
    }
    const auto key_block = [&](int kb) __attribute__((always_inline)) {
        return kb < kKeyBlocks ? K[kb < kKeyBlocks ? kb : 0] : more[(kb - kKeyBlocks) * 64];
    };
    const auto value_block = [&](int kb) __attribute__((always_inline)) {
        return kb < kValueBlocks ? V[kb < kValueBlocks ? kb : 0]
                                 : more[(kBlocks - kKeyBlocks + kb - kValueBlocks) * 64];
    };
    const int shift = sk.count - tokens + 1;  // token i sees keys below i + shift
    const bool far = (int64_t)(group - 1) * max(args.q.head, args.d_o.head) > (1 << 28);
    const RowTiles tiles(group, kRows, far);
    const int all = (tokens + tiles.tokens - 1) / tiles.tokens * tiles.parts;
    const int from = a.causal ? min(max(block_key - shift + 1, 0), tokens) : 0;
    // the tiles of rows that see some of the keys, and the block's part of them
    const int t_first = from / tiles.tokens * tiles.parts;
    const int each = (all - t_first + args.count - 1) / args.count;
    const int t0 = min(t_first + part * each, all), count = min(t0 + each, all);

    // first and last token of the wave's rows in a tile
    int unit_first[Shape::kUnits], unit_last[Shape::kUnits];
#pragma unroll
    for (int unit = 0; unit < Shape::kUnits; ++unit) {
        unit_first[unit] = 32 * (row_group + unit * kRowGroups) / tiles.heads;
        unit_last[unit] = (32 * (row_group + unit * kRowGroups) + 31) / tiles.heads;
    }

    f32x16 dK[D / 32], dV[D / 32];
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt) dK[dt] = f32x16{}, dV[dt] = f32x16{};
    Fit fit, fit_v;
    // (what is not loaded multiplies zeros and has to be finite)
    clear_lds(lds, 4 * kTileBytes, thread, kThreads);
    lds_barrier();

    const E* q0 = row_of<E>(args.q, packed, n, sq, head * group);
    const E* d0 = row_of<E>(args.d_o, packed, n, sq, head * group);
    const float* lse0 = row_of<float>(a.lse, packed, n, sq, head * group);
    const int64_t row_in_all =
        (packed ? sq.first : (int64_t)n * a.tokens) * a.q_heads + head * group;
    // what the lane's key and value have been divided by
    float k_factor = 1.0f, v_factor = 1.0f;
    if constexpr (kSplit) {
        const int64_t i = ((packed ? sk.first : (int64_t)n * a.keys) + key_in) * a.k_heads + head;
        k_factor = args.k_factors[i], v_factor = args.v_factors[i];
    }
    Flow<E, D, kRows, kThreads, kVec || kSplit> fq, fd;
    const int width = kSplit ? kWidth<D> : a.size;
    // of the thread's chunks: their rows' tokens and heads in the tile, a byte each
    uint32_t chunk_tokens[(fq.kEach + 3) / 4] = {}, chunk_heads[(fq.kEach + 3) / 4] = {};
#pragma unroll
    for (int i = 0; i < fq.kEach; ++i) {
        const int r = fq.row(thread) + i * fq.kRowsApart;
        chunk_tokens[i / 4] |= min(r / tiles.heads, 255) << i % 4 * 8;
        chunk_heads[i / 4] |= r % tiles.heads << i % 4 * 8;
    }
    const auto distance = [&](const sgemm_emu_view_t& v) {
        return [&](int r) {
            return (uint32_t)(r / tiles.heads * (int)v.token + r % tiles.heads * (int)v.head) *
                   (uint32_t)sizeof(E);
        };
    };
    fq.rows(distance(args.q), thread);
    fd.rows(distance(args.d_o), thread);
    float st_lse = 0.0f, st_delta = 0.0f, st_q = 0.0f, st_do = 0.0f;
    int st_seen = 0;
    int from_along = QD::One::from_along(lane), from_across = QD::One::from_across(lane);
    const auto load = [&](int t) {
        const int token0 = t / tiles.parts * tiles.tokens, head0 = t % tiles.parts * tiles.heads;
        const int tokens_in = min(tiles.tokens, tokens - token0);
        const int heads_in = min(tiles.heads, group - head0);
        char* to = lds + (t & 1) * 2 * kTileBytes;
        const auto there = [&](int i, int) {
            return (int)(chunk_tokens[i / 4] >> i % 4 * 8 & 255) < tokens_in &&
                   (int)(chunk_heads[i / 4] >> i % 4 * 8 & 255) < heads_in;
        };
        if (thread < kRows) {
            int row = thread;
            asm volatile("" : "+v"(row));
            const int token = row / tiles.heads, h = row % tiles.heads;
            st_lse = -__builtin_inff(), st_delta = 0.0f, st_q = 0.0f, st_do = 0.0f;
            st_seen = a.causal ? token0 + token + shift : sk.count;
            if (token < tokens_in && h < heads_in) {
                const int64_t i = token0 + token;
                st_lse = lse0[i * a.lse.token + (head0 + h) * a.lse.head];
                const int64_t at = row_in_all + i * a.q_heads + head0 + h;
                st_delta = args.delta[at];
                if constexpr (kSplit) st_q = args.q_factors[at], st_do = args.do_factors[at];
            }
        }
        const E* q = q0 + token0 * args.q.token + head0 * args.q.head;
        const E* o = d0 + token0 * args.d_o.token + head0 * args.d_o.head;
#pragma unroll
        for (int i = 0; i < kPlanes<T>; ++i) {
            fq.start(to + i * QD::kPlaneBytes, q + i * kWidth<D>, width, thread, there);
            fd.start(to + kTileBytes + i * QD::kPlaneBytes, o + i * kWidth<D>, width, thread,
                     there);
        }
    };
    if (t0 < count) load(count - 1);
    const float c = kSplit ? 1.0f : a.scale * kLog2e;
    const float of_scores = a.scale * kLog2e * k_factor;
    // from the last rows, which all blocks of a head have, so that those that run beside each
    // other find them in the caches
    for (int t = count - 1; t >= t0; --t) {
        char* qt = lds + (t & 1) * 2 * kTileBytes;
        char* ot = qt + kTileBytes;
        Row& rw = of_rows[t & 1];
        fq.finish(qt, thread);
        fd.finish(ot, thread);
        if (thread < kRows) {
            // (rows that see nothing, and those that are none, have lse -infinity)
            rw.z[thread] =
                st_lse == -__builtin_inff() ? __builtin_inff() : st_lse * kLog2e - kShift;
            rw.delta[thread] = -st_delta;
            rw.seen[thread] = st_seen;
            if constexpr (kSplit) rw.q[thread] = st_q, rw.d_o[thread] = st_do;
        }
        lds_barrier();
        if (t > t0) load(t - 1);
        const int token0 = t / tiles.parts * tiles.tokens;
        // (addresses are formed for every tile: kept, they would take registers that the
        // sums need)
        asm volatile("" : "+v"(from_along), "+v"(from_across));
        const auto rows_of_unit = [&](int unit) __attribute__((always_inline)) {
            const int row0 = 32 * (row_group + unit * kRowGroups);
            // tokens of the wave's rows
            const int wave_first = token0 + unit_first[unit], wave_last = token0 + unit_last[unit];
            if (a.causal && wave_last + shift <= wave_key) return;
            const uint32_t q_along = QD::One::base(qt + row0 * kRowBytes, from_along);
            const uint32_t o_along = QD::One::base(ot + row0 * kRowBytes, from_along);
            const uint32_t q_across = QD::One::base(qt + row0 * kRowBytes, from_across);
            const uint32_t o_across = QD::One::base(ot + row0 * kRowBytes, from_across);
            const auto per_row = [&](const float* x, int i) {  // rows of registers i to i + 3
                return four_floats(x + row0 + 8 * (i / 4) + 4 * half);
        };
        f32x16 P{}, dP;
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const auto x = per_row(rw.delta, i);
#pragma unroll
            for (int j = 0; j < 4; ++j) dP[i + j] = kSplit ? 0.0f : x[j];
        }
#pragma unroll
        for (int kb = 0; kb < kBlocks; ++kb) {
            P = mma(QD::along(q_along, 0, kb), key_block(kb), P);
            dP = mma(QD::along(o_along, 0, kb), value_block(kb), dP);
        }
        if constexpr (!kSplit) {  // reads two steps ahead of the products that take them
            constexpr auto reads = [](int kb) {
                return kb >= kBlocks ? 0 : 2 + (kb >= kKeyBlocks) + (kb >= kValueBlocks);
            };
            __builtin_amdgcn_sched_group_barrier(kLdsRead, 4 + reads(0) + reads(1), 0);
            schedule_steps<kBlocks>([&](auto step) {
                __builtin_amdgcn_sched_group_barrier(kMatrix, 2, 0);
                __builtin_amdgcn_sched_group_barrier(kLdsRead, reads(decltype(step)::value + 2), 0);
            });
        } else {
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const auto x = per_row(rw.q, i), y = per_row(rw.d_o, i), z = per_row(rw.delta, i);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    P[i + j] *= x[j] * of_scores;
                    dP[i + j] = __builtin_fmaf(dP[i + j], y[j] * v_factor, z[j]);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const auto x = per_row(rw.z, i);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float log = __builtin_fmaf(P[i + j], c, -x[j]);
                // (for all: FP16 has no room for more than one, and a branch in its own right takes
                // 2 x 1024 tokens in FP32 from 304 to 384 us, by the registers it needs)
                log = __builtin_elementwise_minimum(log, kShift);
                P[i + j] = __builtin_amdgcn_exp2f(log);
            }
        }
        const bool masked = a.causal && wave_first + shift <= wave_key + 31;
        if (masked) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (key >= rw.seen[row0 + acc_row(i, half)]) P[i] = 0.0f, dP[i] = 0.0f;
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) dP[i] *= P[i];
        if constexpr (kSplit) {
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const auto x = per_row(rw.q, i), y = per_row(rw.d_o, i);
#pragma unroll
                for (int j = 0; j < 4; ++j) P[i + j] *= y[j], dP[i + j] *= x[j];
            }
            fit_v.fit(largest(P), dV);
            P = times(P, fit_v.f);
        }
#pragma unroll
        for (int kb = 0; kb < kParts; ++kb) {
            const Operand<T> x = operand<T>(P, kb);
#pragma unroll
            for (int dt = 0; dt < D / 32; ++dt)
                dV[dt] = mma(QD::across(o_across, kb, 32 * dt), x, dV[dt]);
        }
        if constexpr (kNarrow<T>) {
            fit.fit(largest(dP), dK);
            dP = times(dP, fit.f);
        }
#pragma unroll
        for (int kb = 0; kb < kParts; ++kb) {
            const Operand<T> x = operand<T>(dP, kb);
#pragma unroll
            for (int dt = 0; dt < D / 32; ++dt)
                dK[dt] = mma(QD::across(q_across, kb, 32 * dt), x, dK[dt]);
        }
        };
        rows_of_unit(0);
        if (Shape::kUnits == 2) rows_of_unit(1);
    }

    // the sums of the waves with the same keys, in the order of their rows
    const auto join = [&](f32x16(&sum)[D / 32], float f, Out<T>* to, float* to_part)
        __attribute__((always_inline)) {
        typedef Pack<float, 4>::type Four;
        lds_barrier();
        Four* const mine = reinterpret_cast<Four*>(lds) +
                           ((row_group - 1) * Shape::kKeyGroups + key_group) * (D / 8) * 64 + lane;
        if (row_group > 0) {
#pragma unroll
            for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    mine[(dt * 4 + i) * 64] = Four{sum[dt][4 * i] * f, sum[dt][4 * i + 1] * f,
                                                   sum[dt][4 * i + 2] * f, sum[dt][4 * i + 3] * f};
        }
        lds_barrier();
        if (row_group > 0 || !valid) return;
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                Four x{sum[dt][4 * i] * f, sum[dt][4 * i + 1] * f, sum[dt][4 * i + 2] * f,
                       sum[dt][4 * i + 3] * f};
#pragma unroll
                for (int g = 1; g < kRowGroups; ++g)
                    x += reinterpret_cast<const Four*>(lds)[((g - 1) * Shape::kKeyGroups + key_group) *
                                                                (D / 8) * 64 +
                                                            (dt * 4 + i) * 64 + lane];
                const int d = 32 * dt + acc_row(4 * i, half);
                if (to_part != nullptr)
                    store_four<float, true>(to_part, d, kPartStride<D>, x[0], x[1], x[2], x[3]);
                else
                    store_four<Out<T>, kVec>(to, d, a.size, x[0], x[1], x[2], x[3]);
            }
    };
    const int64_t key_row = ((packed ? sk.first : (int64_t)n * a.keys) + key_in) * a.k_heads + head;
    float* const dv_part = args.parts ? args.parts + (part * 2 * args.key_rows + key_row) *
                                                         kPartStride<D>
                                      : nullptr;
    float* const dk_part = args.parts ? dv_part + args.key_rows * kPartStride<D> : nullptr;
    join(dV, kSplit ? kBack / fit_v.f : kBack,
         row_of<Out<T>>(a.dv, packed, n, sk, head) + key_in * a.dv.token, dv_part);
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt) dK[dt] = times(dK[dt], a.scale);
    join(dK, kNarrow<T> ? kBack / fit.f : 1.0f,
         row_of<Out<T>>(a.dk, packed, n, sk, head) + key_in * a.dk.token, dk_part);
}

// dv and dk as the sums of their parts, in order.
template <class T, int D, bool kVec>
__global__ __launch_bounds__(256) void attention_sum_kernel(BackwardArgs args, int first_block) {
    typedef Pack<float, 4>::type Four;
    constexpr int kEach = kPartStride<D> / 4;
    const attention_emu_backward_t& a = args.a;
    const int64_t at =
        (int64_t)(first_block + (int)blockIdx.x) * (256 / kEach) + threadIdx.x / kEach;
    const int d = threadIdx.x % kEach * 4;
    if (at >= 2 * args.key_rows || d >= a.size) return;
    Four x{};
#pragma unroll 4
    for (int p = 0; p < args.count; ++p)
        x += *reinterpret_cast<const Four*>(args.parts + (p * 2 * args.key_rows + at) * kPartStride<D> +
                                            d);
    const sgemm_emu_view_t& to = at < args.key_rows ? a.dv : a.dk;
    const int64_t row = at < args.key_rows ? at : at - args.key_rows;
    const int64_t key = row / a.k_heads, n = key / a.keys;
    T* out = static_cast<T*>(to.p) + n * to.batch + (key - n * a.keys) * to.token +
             (row - key * a.k_heads) * to.head;
    store_four<T, kVec>(out, d, a.size, x[0], x[1], x[2], x[3]);
}

int64_t batch_of(const attention_emu_backward_t& a) {
    return a.cu_seqlens != nullptr ? 1 : a.batch;
}

int64_t delta_bytes(const attention_emu_backward_t& a) {
    return (batch_of(a) * a.tokens * a.q_heads * 4 + 255) / 256 * 256;
}

int64_t planes_bytes(const attention_emu_backward_t& a) {
    if (a.dtype != SGEMM_EMU_F32) return 0;
    return 2 * split_bytes(batch_of(a) * a.tokens, a.q_heads, a.size) +
           2 * split_bytes(batch_of(a) * a.keys, a.k_heads, a.size);
}

// Parts of the query rows of a block of keys: where the blocks are fewer than the CUs, as many as
// fill those, of at least 512 rows each (256: no change): 3 x 1001 tokens with 2 key heads in
// FP32 250 -> 177 us, 2048 with 4 heads in bfloat16 95 -> 89.
int parts_of(const attention_emu_backward_t& a) {
    const int64_t blocks = most_parts(a.batch, a.keys, 64, a.cu_seqlens != nullptr) * a.k_heads;
    if (blocks == 0 || a.cu_seqlens != nullptr) return 1;
    const int64_t most = (int64_t)a.tokens * (a.q_heads / a.k_heads) / 512;
    return (int)std::max<int64_t>(1, std::min(most, (256 + blocks / 2) / blocks));
}

int64_t sums_bytes(const attention_emu_backward_t& a, int parts) {
    if (parts == 1) return 0;
    const int64_t rows = parts * 2 * batch_of(a) * a.keys * a.k_heads;
    return (rows * part_stride(a.size) * 4 + 255) / 256 * 256;
}

}  // namespace

int64_t attention_backward_workspace(const attention_emu_backward_t& a) {
    return delta_bytes(a) + planes_bytes(a) + sums_bytes(a, parts_of(a));
}

hipError_t launch_attention_backward(const attention_emu_backward_t& a, hipStream_t stream) {
    char* const ws = static_cast<char*>(a.workspace);
    const bool packed = a.cu_seqlens != nullptr;
    BackwardArgs args{};
    args.a = a;
    if (packed && a.cu_keys == nullptr) args.a.cu_keys = a.cu_seqlens;
    args.delta = reinterpret_cast<float*>(ws);
    args.q = a.q, args.k = a.k, args.v = a.v, args.d_o = a.d_o;
    args.count = parts_of(a);
    args.key_rows = batch_of(a) * a.keys * a.k_heads;
    if (args.count > 1)
        args.parts = reinterpret_cast<float*>(ws + delta_bytes(a) + planes_bytes(a));
    const int e = a.dtype == SGEMM_EMU_F32 ? 4 : 2;
    bool vec = a.size * e % 16 == 0;
    for (const sgemm_emu_view_t* x : {&a.o, &a.d_o, &a.dq, &a.dk, &a.dv})
        vec = vec && rows_aligned16(*x, e);
    if (a.dtype == SGEMM_EMU_F32) {
        Splitter split(a.size, ws + delta_bytes(a));
        const int batch = (int)batch_of(a);
        const SplitTensor q = split.add(a.q, batch, a.tokens, a.q_heads);
        const SplitTensor k = split.add(a.k, batch, a.keys, a.k_heads);
        const SplitTensor v = split.add(a.v, batch, a.keys, a.k_heads);
        const SplitTensor d_o = split.add(a.d_o, batch, a.tokens, a.q_heads);
        args.q = q.planes, args.k = k.planes, args.v = v.planes, args.d_o = d_o.planes;
        args.q_factors = q.factors, args.k_factors = k.factors, args.v_factors = v.factors;
        args.do_factors = d_o.factors;
        if (hipError_t e = split.launch(stream)) return e;
    } else {
        for (const sgemm_emu_view_t* x : {&a.q, &a.k, &a.v}) vec = vec && rows_aligned16(*x, e);
    }
    const int64_t group = a.q_heads / a.k_heads;
    const int64_t q_blocks = most_parts(a.batch, a.tokens * group, kDqRows, packed) * a.k_heads;
    return by_form<split_t>(a.dtype, a.size, vec, [&](auto t, auto d, auto vec) {
        using T = decltype(t);
        constexpr int D = decltype(d)::value;
        constexpr bool kVec = decltype(vec)::value != 0;
        if (a.tokens > 0) {
            // (split operands of more than 96 elements leave no registers for two groups)
            constexpr int kGroups = kPlanes<T> == 1 || D <= 96 ? 2 : 1;
            const hipError_t e =
                q_blocks < kDqPaired
                    ? launch_blocks(attention_dq_kernel<T, D, kVec, kGroups>, q_blocks,
                                    64 * kDqWaves * kGroups, stream, args)
                    : launch_blocks(attention_dq_kernel<T, D, kVec, 1>, q_blocks, 64 * kDqWaves,
                                    stream, args);
            if (e != hipSuccess) return e;
        }
        using Shape = DkvShape<T, D>;
        const int64_t blocks =
            most_parts(a.batch, a.keys, Shape::kKeys, packed) * a.k_heads * args.count;
        if (hipError_t e = launch_blocks(attention_dkv_kernel<T, D, kVec>, blocks, Shape::kThreads,
                                         stream, args))
            return e;
        if (args.count == 1) return hipSuccess;
        constexpr int kRows = 256 / (kPartStride<D> / 4);
        return launch_blocks(attention_sum_kernel<Out<T>, D, kVec>,
                             (2 * args.key_rows + kRows - 1) / kRows, 256, stream, args);
    });
}

}  // namespace sgemm_emu
