// One pass of softmax attention over a range of keys, for a block's query rows.
//
// Per row, with scores s_j = q k_j (unscaled) and c = scale log2 e > 0, the pass keeps a
// score m, its reference z = c m - kBias, l = sum_j 2^(c s_j - z) and O = sum_j 2^(c s_j - z) v_j,
// all in FP32.  They only move where a row's largest score is more than 2^kSlack above m: the
// weights then stay below 2^(kSlack + kBias) and the result does not depend on m.
//
// z is rounded, and all weights of a row are off by that: below |z| = kCoarse by 2^(1/8) at most.
// From there on the last bit of z comes to be no longer small beside one, and weights would pass
// FP16's range, or be zeros for all keys.  Such a row's weights are 2^(c (s_j - m) + kBias), with
// a difference that is exact near the largest score.  That has to be where m moves: a branch of its
// own between the scores and the products takes 4 x 4096 tokens from 573 to 620 us.
//
// The products are S^T = K Q^T and O^T = V^T P^T in 32 x 32 tiles: a lane holds
// one query row, so that its reference, sum and rescaling are scalars of the lane, and
// the weights of S^T's accumulator are the second product's operand in place.  Weights
// are rounded to the inputs' type (11 or 8 bits, relative to each weight) for the matrix
// instructions; l sums them before that.
#pragma once

#include "attention_parts.hpp"

namespace sgemm_emu {

// A block's waves are kKeyGroups groups that take every kKeyGroups-th tile of kKeys keys and
// are joined at the end, of kRowGroups waves with 32 rows each.  Two waves for each SIMD hide each
// other's softmax behind matrix instructions (4 x 4096 tokens 654 us for 995 with one).  Tiles of
// 64 keys have half the barriers of 32 (24 packed prompts 67 us for 82; 4 x 4096 tokens 572 for
// 559).  The waves of a group share its tiles; where they are one (kRowGroups == 1), its keys go
// straight from memory to operands.
template <class T, int D, int kRowGroups, int kKeyGroups, int kKeys, bool kVec>
struct Attend {
    static constexpr bool kShared = kRowGroups > 1;
    static_assert(kShared || kKeys == 32, "");
    static constexpr int kThreads = 64 * kRowGroups * kKeyGroups;
    static constexpr int kRows = 32 * kRowGroups;
    typedef Elem<T> E;
    static constexpr bool kSplit = kPlanes<T> == 2;
    static_assert(kShared || !kSplit, "");
    using KV = Planes<T, D, kKeys>;
    static constexpr int kTileBytes = KV::kBytes;
    static constexpr int kPlace = (kShared ? 2 : 1) * kTileBytes;  // of a tile's keys and values
    static constexpr int kTiles = kKeyGroups * 2 * kPlace;
    static constexpr int kJoinRow = D + 4;  // floats
    // (shared: [row group][4 registers][lane] of the second group's sums, and l and z)
    static constexpr int kJoin = kShared ? (kKeyGroups - 1) * kRowGroups * (D / 8 * 1024 + 512)
                                         : kKeyGroups * 32 * (kJoinRow + 2) * 4;
    static_assert(!kShared || kKeyGroups <= 2, "");
    static constexpr int kFactors = kSplit ? 2 * kKeys : 0;  // of a tile's keys and values
    static constexpr int kLds =
        (kTiles > kJoin ? kTiles : kJoin) + 2 * kKeyGroups * kFactors * 4 + 16;
    static constexpr int kTileThreads = 64 * kRowGroups;
    // FP16 weights keep 11 bits down to 2^-14: 2^-21 of a row's largest
    static constexpr float kBias = __is_same(E, f16_t) ? 7.0f : 0.0f;
    static constexpr float kSlack = 8.0f;
    static constexpr float kCoarse = 0x1p22f;

    // rows: query rows there are; the block takes row0 to row0 + kRows - 1.
    // q_row(r): its elements; limit(r): how many keys it sees (not decreasing in r).
    // k, v: row 0 of the keys and values; the pass goes over keys first to end - 1.
    // out(r): where a row's results go; of that, sums(l, z, here) and four(d, ...).
    // factors: what the rows of split tensors have been divided by: q(r), k[], v[] (`step` apart).
    template <class QRow, class Limit, class Results, class Factors>
    static __device__ __attribute__((always_inline)) void run(
        char* lds, int rows, int row0, QRow q_row, Limit limit, const E* k, int64_t k_token,
        const E* v, int64_t v_token, int first, int end, int size, float c, bool negative,
        Results out, Factors factors) {
        constexpr int kBlocks = D / kBlock<E>;
        constexpr int kParts = 32 / kBlock<E>;  // operand blocks of 32 keys
        constexpr bool kVecTile = kVec || kSplit;
        const int width = kSplit ? kWidth<D> : size;
        const int lane = threadIdx.x & 63, half = lane >> 5;
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int group = wave / kRowGroups, row_group = wave % kRowGroups;
        const int wave_row = row0 + 32 * row_group;
        const int tile_thread = (int)threadIdx.x % kTileThreads;
        char* tiles = lds + group * 2 * kPlace;
        int* bad = reinterpret_cast<int*>(lds + kLds - 16);

        const int row = wave_row + (lane & 31), last_row = rows - 1;
        Operand<T> Q[kBlocks];
        {
            const E* p = q_row(min(row, last_row));
#pragma unroll
            for (int kb = 0; kb < kBlocks; ++kb) {
                Q[kb] = load_operand<T, D, kVec>(p, 2 * kb + half, size, row < rows);
            }
        }
        // (split scores come in units of c s: what q and k have been divided by multiplies them at
        // once, for one alone may take a product past FP32's range)
        float of_scores = 1.0f;
        if constexpr (kSplit) of_scores = c * factors.q(min(row, last_row)), c = 1.0f;
        // keys seen by the lane's row, by the wave's first and last one, by the block's
        const auto seen = [&](int r) { return min(max(limit(min(r, last_row)), first), end); };
        const int lim = seen(row), lim_min = seen(wave_row), lim_max = seen(wave_row + 31);
        const int block_min = seen(row0), block_max = seen(row0 + kRows - 1);
        const int count = (block_max - first + kKeys - 1) / kKeys;
        // from this tile on, some row of the block does not see all of the keys
        const int cleared = (block_min - first) / kKeys;

        const typename KV::Read read(tiles, lane);

        f32x16 O[D / 32];
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt) O[dt] = f32x16{};
        float l = 0.0f, m = -__builtin_inff();
        // z; -kBias of a coarse row, whose scores are taken less m
        float less = kLeast;
        bool coarse = false;
        const auto reference = [&](float m) {
            return m > -__builtin_inff() ? __builtin_fmaf(m, c, -kBias) : kLeast;
        };
        // split values: a weight times its value's factor becomes an operand, for which each row
        // has a power of two by what it weighs itself: by the largest factor of a tile's values,
        // one that a row does not see, or hardly weighs, took the bits of all others
        Fit fit;
        bool found = false;
        if (kVecTile && width < kWidth<D>) {
            clear_lds(lds, kTiles, threadIdx.x, kThreads);
            lds_barrier();
        }

        using Load = Flow<E, D, kKeys, kTileThreads, kVecTile>;
        Load fk, fv;
        Operand<T> K[kShared ? 1 : kBlocks];
        float* const of_tiles = reinterpret_cast<float*>(lds + kLds - 16) -
                                2 * (group + 1) * kFactors;
        float st_factor = 0.0f;
        constexpr int step = kKeyGroups;
        const uint32_t k_row = (uint32_t)k_token * sizeof(E), v_row = (uint32_t)v_token * sizeof(E);
        const auto place = [&](int t) {
            return tiles + (t / kKeyGroups & 1) * kPlace;
        };
        if (kShared) fk.rows([&](int r) { return r * k_row; }, tile_thread);
        fv.rows([&](int r) { return r * v_row; }, tile_thread);
        const auto load = [&](int t) {
            const int key = first + t * kKeys, most = end - 1 - key;
            // (keys behind the last one are masked, and values there cleared if need be)
            const auto there = [&](int, int r) { return r <= most; };
            if constexpr (kSplit) {
                const int i = tile_thread % kKeys;
                if (tile_thread < kFactors)
                    st_factor = i > most ? 0.0f
                                         : (tile_thread < kKeys ? factors.k
                                                                : factors.v)[(key + i) * factors.step];
            }
            if constexpr (kShared) {
#pragma unroll
                for (int i = 0; i < kPlanes<T>; ++i)
                    fk.start(place(t) + i * KV::kPlaneBytes, k + key * k_token + i * kWidth<D>, width,
                             tile_thread, there);
            } else {
                const E* p = k + (key + min(lane & 31, most)) * k_token;
#pragma unroll
                for (int kb = 0; kb < kBlocks; ++kb)
                    K[kb] = load_operand<T, D, kVec>(p, 2 * kb + half, size, true);
            }
#pragma unroll
            for (int i = 0; i < kPlanes<T>; ++i)
                fv.start(place(t) + kPlace - kTileBytes + i * KV::kPlaneBytes,
                         v + key * v_token + i * kWidth<D>, width, tile_thread, there);
        };
        if (group < count) load(group);
        // (after the loads: these wait for the first of them)
        if (threadIdx.x == 0) *bad = 0;
        lds_barrier();
        if (negative)
#pragma unroll
            for (int kb = 0; kb < kBlocks; ++kb)
#pragma unroll
                for (int i = 0; i < kPlanes<T>; ++i)
#pragma unroll
                    for (int j = 0; j < kPer<E>; ++j) Q[kb].p[i][j] = -Q[kb].p[i][j];
        // one tile, in the first or the second of the wave's places
        const auto tile = [&](int t, auto odd) __attribute__((always_inline)) {
            constexpr int at = decltype(odd)::value * kPlace, v_at = at + kPlace - kTileBytes;
            char* kt = tiles + at;
            char* vt = tiles + v_at;
            // (a group of several waves may have one tile less than the others, for whose sake
            // it comes to the barrier)
            const bool here = kKeyGroups == 1 || !kShared || t < count;
            float* const of_tile = of_tiles + decltype(odd)::value * kFactors;
            if (here) {
                if (kShared) fk.finish(kt, tile_thread);
                fv.finish(vt, tile_thread);
                // values that are not finite reach only rows that see them: where some row
                // does not, they are left out here and added at the end
                if (t >= cleared)
#pragma unroll
                    for (int i = 0; i < kPlanes<T>; ++i)
                        found |= Load::clear_not_finite(
                            vt + i * KV::kPlaneBytes, tile_thread,
                            [&](int, int r) { return first + t * kKeys + r < end; });
                if (kSplit && tile_thread < kFactors) of_tile[tile_thread] = st_factor;
            }
            f32x16 S[kKeys / 32];
            if constexpr (kShared) {
                lds_barrier();
                if (t + step < count) load(t + step);
                if (!here) return;
            } else {
                S[0] = f32x16{};
#pragma unroll
                for (int kb = 0; kb < kBlocks; ++kb) S[0] = mma(K[kb], Q[kb], S[0]);
                if (t + step < count) load(t + step);
            }
            const int key0 = first + t * kKeys;
            if (key0 >= lim_max) return;

            if constexpr (kShared) {
#pragma unroll
                for (int s = 0; s < kKeys / 32; ++s) {
                    S[s] = f32x16{};
#pragma unroll
                    for (int kb = 0; kb < kBlocks; ++kb)
                        S[s] = mma(KV::along(read, at + 32 * s * KV::One::kRowBytes, kb), Q[kb], S[s]);
                }
            }
            // factors of registers i to i + 3
            const auto four_of = [&](const float* x, int s, int i) {
                return *reinterpret_cast<const Pack<float, 4>::type*>(x + 32 * s + 8 * (i / 4) +
                                                                      4 * half);
            };
            if constexpr (kSplit) {
#pragma unroll
                for (int s = 0; s < kKeys / 32; ++s)
#pragma unroll
                    for (int i = 0; i < 16; i += 4) {
                        const auto x = four_of(of_tile, s, i);
#pragma unroll
                        for (int j = 0; j < 4; ++j) S[s][i + j] *= x[j] * of_scores;
                    }
            }
            if (key0 + kKeys > lim_min) {
#pragma unroll
                for (int s = 0; s < kKeys / 32; ++s)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (key0 + 32 * s + acc_row(i, half) >= lim) S[s][i] = -__builtin_inff();
            }
            float top = S[0][0];
#pragma unroll
            for (int s = 0; s < kKeys / 32; ++s)
#pragma unroll
                for (int i = 0; i < 16; ++i) top = fmaxf(top, S[s][i]);
            top = max_halves(top);
            if (__any(__builtin_fmaf(top, c, -kBias) > less + kSlack || coarse)) {
                const bool moves = (top - m) * c > kSlack;  // (z + kSlack may be z)
                const float z = reference(m), to = moves ? reference(top) : z;
                coarse = __builtin_fabsf(to) >= kCoarse && __builtin_fabsf(to) < -kLeast;
                const float fall = moves ? (coarse ? (top - m) * c : to - z) : 0.0f;
                m = moves ? top : m;
                less = coarse ? -kBias : to;
                const float f = __builtin_amdgcn_exp2f(-fall);
                const float of_sum = kSplit ? __builtin_amdgcn_exp2f(fit.rise(fall) - fall) : f;
#pragma unroll
                for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
                    for (int i = 0; i < 16; ++i) O[dt][i] *= of_sum;
                l *= f;
                // (s_j - m: one more product, of ones and -m)
                const float by = coarse ? -m : 0.0f;
#pragma unroll
                for (int s = 0; s < kKeys / 32; ++s)
                    S[s] = __builtin_amdgcn_mfma_f32_32x32x2f32(half == 0 ? 1.0f : 0.0f, by, S[s], 0,
                                                                0, 0);
            }
#pragma unroll
            for (int s = 0; s < kKeys / 32; ++s) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    S[s][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(S[s][i], c, -less));
                    l += S[s][i];
                }
            }
            if constexpr (kSplit) {
                float most = 0.0f;
#pragma unroll
                for (int s = 0; s < kKeys / 32; ++s) {
#pragma unroll
                    for (int i = 0; i < 16; i += 4) {
                        const auto x = four_of(of_tile + kKeys, s, i);
#pragma unroll
                        for (int j = 0; j < 4; ++j) S[s][i + j] *= x[j];
                    }
                    most = fmaxf(most, largest(S[s]));
                }
                fit.fit(most, O);
#pragma unroll
                for (int s = 0; s < kKeys / 32; ++s) S[s] = times(S[s], fit.f);
            }
#pragma unroll
            for (int s = 0; s < kKeys / 32; ++s) {
#pragma unroll
                for (int kb = 0; kb < kParts; ++kb) {
                    const Operand<T> P = operand<T>(S[s], kb);
#pragma unroll
                    for (int dt = 0; dt < D / 32; ++dt)
                        O[dt] = mma(KV::across(read, v_at, s * kParts + kb, dt), P, O[dt]);
                }
            }
        };
        // (waves that meet at barriers go on until the first group is through)
        const int last = kShared ? count + group : count;
        for (int t = group; t < last; t += 2 * step) {
            tile(t, Number<0>{});
            if (t + step < last) tile(t + step, Number<1>{});
        }
        l = sum_halves(l);
        float z = reference(m);
        float unit = kSplit ? inverse_of_power(fit.f) : 1.0f;  // of O
        if (found) *bad = 1;
        __syncthreads();
        const bool repair = *bad != 0;

        if constexpr (kShared && kKeyGroups == 2) {
            typedef Pack<float, 4>::type Four;
            Four* const sums = reinterpret_cast<Four*>(lds) + row_group * (D / 8 * 64 + 32) + lane;
            float* const of_row = reinterpret_cast<float*>(sums + D / 8 * 64 - lane) + lane;
            if (group == 1) {
#pragma unroll
                for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        sums[(4 * dt + i) * 64] =
                            Four{O[dt][4 * i], O[dt][4 * i + 1], O[dt][4 * i + 2],
                                 O[dt][4 * i + 3]} * unit;
                of_row[0] = l, of_row[64] = z;
            }
            __syncthreads();
            if (group == 1) return;
            const float other_l = of_row[0], other_z = of_row[64], top = fmaxf(z, other_z);
            const float f = __builtin_amdgcn_exp2f(z - top), g = __builtin_amdgcn_exp2f(other_z - top);
            l = l * f + other_l * g;
            z = top;
#pragma unroll
            for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const Four x = sums[(4 * dt + i) * 64];
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        O[dt][4 * i + j] = O[dt][4 * i + j] * (f * unit) + x[j] * g;
                }
            unit = 1.0f;
        }
        if constexpr (kShared) {
            if (row < rows) {
                if (repair)
                    for (int j = first + cleared * kKeys; j < lim; ++j)
#pragma unroll
                        for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
                            for (int i = 0; i < 16; ++i)
                                O[dt][i] += not_finite(v + j * v_token, 32 * dt + acc_row(i, half), size);
                const float f = l == 0.0f ? 0.0f : (kSplit ? unit : 1.0f) / l;
                auto to = out(row);
                to.sums(l, z, half == 0);
#pragma unroll
                for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
                    for (int i = 0; i < 16; i += 4)
                        to.four(32 * dt + acc_row(i, half), O[dt][i] * f, O[dt][i + 1] * f,
                                O[dt][i + 2] * f, O[dt][i + 3] * f);
            }
        } else {
            float* join = reinterpret_cast<float*>(lds);
            float* state = join + kKeyGroups * 32 * kJoinRow;
            const int n = lane & 31;
            float* mine = join + (wave * 32 + n) * kJoinRow;
#pragma unroll
            for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
                for (int i = 0; i < 16; i += 4)
                    *reinterpret_cast<Pack<float, 4>::type*>(mine + 32 * dt + acc_row(i, half)) =
                        Pack<float, 4>::type{O[dt][i], O[dt][i + 1], O[dt][i + 2], O[dt][i + 3]};
            if (half == 0) state[2 * (wave * 32 + n)] = l, state[2 * (wave * 32 + n) + 1] = z;
            __syncthreads();
            for (int w = threadIdx.x; w < 32 * (D / 4); w += kThreads) {
                const int r = w / (D / 4), d = w % (D / 4) * 4;
                if (row0 + r >= rows) break;
                float zs = kLeast, ls = 0.0f;
#pragma unroll
                for (int g = 0; g < kKeyGroups; ++g) zs = fmaxf(zs, state[2 * (g * 32 + r) + 1]);
                Pack<float, 4>::type x{};
#pragma unroll
                for (int g = 0; g < kKeyGroups; ++g) {
                    const float f = __builtin_amdgcn_exp2f(state[2 * (g * 32 + r) + 1] - zs);
                    ls += f * state[2 * (g * 32 + r)];
                    const auto y = *reinterpret_cast<const Pack<float, 4>::type*>(
                        join + (g * 32 + r) * kJoinRow + d);
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[j] += f * y[j];
                }
                const float f = ls == 0.0f ? 0.0f : 1.0f / ls;
                if (repair) {
                    const int to = seen(row0 + r);
                    for (int j = first + cleared * kKeys; j < to; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[e] += not_finite(v + j * v_token, d + e, size);
                }
                auto to = out(row0 + r);
                to.sums(ls, zs, d == 0);
                to.four(d, x[0] * f, x[1] * f, x[2] * f, x[3] * f);
            }
        }
    }

    // Element d of a row of values if it is not finite, else 0.  A positive weight of infinity
    // or NaN is the same.
    static __device__ inline float not_finite(const E* p, int d, int size) {
        const float x = d < size ? to_f32(p[d]) : 0.0f;
        return __builtin_fabsf(x) < __builtin_inff() ? 0.0f : x;
    }
};

}  // namespace sgemm_emu
