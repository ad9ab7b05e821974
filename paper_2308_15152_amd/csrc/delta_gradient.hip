// The gated delta rule's gradient, last kernel: dQ, dK, dbeta and dg of every
// chunk, from S before it, the gradient D of S after it, U, dY and dO.  With
//   E1 = dO S^T,  E2 = dY S^T,  E3 = U D^T             (64 x k_size),
//   M1 = scale e^{G_t - G_s} (dO U^T)_ts, s <= t,  M2 = e^{G_t - G_s} (dY U^T)_ts, s < t,
//   W = -(diag(e^G) E2 + M2 K),
//   C = diag(e^{G_64 - G}) E3 + M1^T Q - M2^T diag(beta) K:
//   dQ = scale diag(e^G) E1 + M1 K,     dK = diag(beta) W + C,
//   dbeta_t = dY_t.V_t + K_t.W_t,
//   dg_t = e^{G_64} <D, S> + sum_{i >= t} a_i + sum_{j < t} b_j + sum_{i >= t > j} X_ij,
//     a_i = e^{G_i} (scale Q_i.E1_i - beta_i K_i.E2_i),   b_j = e^{G_64 - G_j} K_j.E3_j,
//     X_ij = M1_ij Q_i.K_j - beta_i M2_ij K_i.K_j
// (every path of a token's decay: state to state, state to output, write to
// state, write to output or write).  The last sum is the sum over i >= t of row
// sums less column sums of X, taken in FP64: it cancels.
//
// A block takes one chunk of one key head and goes through its value heads, so
// that dQ and dK are summed in registers in a fixed order.  A wave owns 16 of
// the key's elements (columns of E, W, C, dQ, dK): S and D are read and split by
// one wave each, straight into operand registers, while dO, dY and U go through
// LDS as fragments that all waves use (also as each other's B operands for M1
// and M2).  Then M1 and M2 take their place there.  One block fits a CU, so loads and
// products of the 224 KB that a head of 128 x 128 reads overlap little: 2 x 4096 tokens of
// 16 heads in bfloat16 take 266 us, 1.7 TB/s.
#include <type_traits>

#include "delta_chunk.hpp"

namespace sgemm_emu {

namespace {

constexpr int kWaves = 8;
constexpr int kThreads = 64 * kWaves;
constexpr int kPitch = 68;

// LDS, in bytes.
template <class T, int kK>
struct Layout {
    static constexpr int kParts = kPartsOf<T>;
    static constexpr int kSteps = kK / 32, kTiles = kK / 16;
    static constexpr int kColumns = kParts * 4 * kSteps * 1024;  // K^T or Q^T
    // columns of V taken at a time, in steps of 32 (with four steps the registers do
    // not hold them, at 128 x 128: 307 us against 268 for 2 x 4096 tokens of 16 heads)
    static constexpr int kVSteps = 2;
    static constexpr int kPart = 4 * kVSteps * 1024;  // one part of dO, dY or U
    static constexpr int kAtKt = 0;
    static constexpr int kAtQt = kAtKt + kColumns;
    static constexpr int kShared = kAtQt + kColumns;
    static constexpr int kAtDo = kShared;  // dO, dY, U ...
    static constexpr int kAtDy = kAtDo + kParts * kPart;
    static constexpr int kAtU = kAtDy + 2 * kPart;
    static constexpr int kEndA = kAtU + 2 * kPart;
    static constexpr int kAtM = kShared;  // ... or M1, M2 in FP32, and as fragments
    static constexpr int kMatrix = kC * kPitch * 4;
    static constexpr int kAtFragments = kAtM + 2 * kMatrix;
    static constexpr int kEndB = kAtFragments + 4 * 2 * DeltaRecord::kMatrix;
    static constexpr int kAtSmall = kEndA > kEndB ? kEndA : kEndB;
    struct Small {
        double G[kC];  // (the arrays stay 16-byte aligned)
        float beta[kC], key_down[kC], query_down[kC];
        union {
            float down[3][kC];   // inverse row scales of dO, dY, U
            double rows[2][kC];  // row sums of X, of either term
        };
        float m_down[4][kC];     // of M1, M2, M1^T, M2^T
        float dot[kC];           // dY_t.V_t
        float rise[kC], tail[kC];  // e^G, e^{G_64 - G}
        float end[kWaves];          // <D, S> per wave
        double columns[2][4][kC];   // column sums of X, of each row tile
    };
    static constexpr int kBytes = kAtSmall + (int)sizeof(Small);
};

// Sum over the 16 lanes of a group, in every one of them.
__device__ inline float sum_row(float x) {
    const auto turned = [](float y, auto by) {
        return __builtin_bit_cast(
            float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, y), 0x120 + decltype(by)::value,
                                            0xf, 0xf, true));
    };
    x += turned(x, std::integral_constant<int, 8>{});
    x += turned(x, std::integral_constant<int, 4>{});
    x += turned(x, std::integral_constant<int, 2>{});
    return x + turned(x, std::integral_constant<int, 1>{});
}

__device__ inline double sum_row(double x) {
    const auto turned = [](double y, auto by) {
        uint64_t u = __builtin_bit_cast(uint64_t, y);
        const uint32_t lo = __builtin_amdgcn_mov_dpp((int)u, 0x120 + decltype(by)::value, 0xf, 0xf, true);
        const uint32_t hi =
            __builtin_amdgcn_mov_dpp((int)(u >> 32), 0x120 + decltype(by)::value, 0xf, 0xf, true);
        return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
    };
    x += turned(x, std::integral_constant<int, 8>{});
    x += turned(x, std::integral_constant<int, 4>{});
    x += turned(x, std::integral_constant<int, 2>{});
    return x + turned(x, std::integral_constant<int, 1>{});
}

// Rows of tile `tile` of M (or its transpose), columns times `by`, as fragments.
template <bool kTransposed>
__device__ inline void write_fragments(const float* M, const float* by, const float* by2, int tile,
                                       int lane, char* to, float* down) {
    const int row = lane & 15, g = lane >> 4;
    float x[2][8], m = 0.0f;
#pragma unroll
    for (int step = 0; step < 2; ++step)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int other = 2 * step + half;
            const bool full = kTransposed ? other >= tile : other <= tile;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int a = 16 * tile + row, b = 16 * other + 4 * g + i;
                float v = 0.0f;
                if (full) v = (kTransposed ? M[b * kPitch + a] : M[a * kPitch + b]) * by[b];
                if (full && by2) v *= by2[b];
                x[step][4 * half + i] = v;
                m = fmaxf(m, fabsf(v));
            }
        }
    const Scale s = scale_of(max_groups(m));
    if (g == 0) down[16 * tile + row] = s.down;
#pragma unroll
    for (int step = 0; step < 2; ++step) {
        if (kTransposed ? step < tile / 2 : step > tile / 2) continue;
        const int at = kTransposed ? upper_at(tile, step) : lower_at(tile, step);
        const Frag<2> f = split<2>(x[step], s.up);
#pragma unroll
        for (int p = 0; p < 2; ++p)
            *reinterpret_cast<half8_t*>(to + (p * 6 + at) * 1024 + lane * 16) = f.part[p];
    }
}

// kWide: all rows of q, k, v, d_o and of the workspace in 16-byte loads.
// kShared: key heads with more than one value head.
template <class T, int kK, bool kWide, bool kShared>
__global__ __launch_bounds__(kThreads, 1) void delta_gradient_kernel(DeltaChunks p) {
    using L = Layout<T, kK>;
    constexpr int kVSteps = L::kVSteps, kVBlock = 32 * kVSteps;
    constexpr int kOwn = 4 * L::kTiles / kWaves;  // token tiles of a wave
    extern __shared__ __attribute__((aligned(16))) char lds[];
    auto& small = *reinterpret_cast<typename L::Small*>(lds + L::kAtSmall);

    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int kh = blockIdx.x % p.k_heads, c = blockIdx.x / p.k_heads;
    const Place at = place_of(p.cu_seqlens, c, p.batch, p.tokens);
    if (at.count <= 0) return;  // the whole block
    const bool packed = p.cu_seqlens != nullptr;
    const int group = p.v_heads / p.k_heads;
    const int tile = wave % L::kTiles, own = wave / L::kTiles * kOwn;

    // K^T and Q^T, and this lane's elements of K and Q
    const T* k = row_of<const T>(p.k, packed, at.n, at.span, kh) + (int64_t)at.first * p.k.token;
    const T* q = row_of<const T>(p.q, packed, at.n, at.span, kh) + (int64_t)at.first * p.q.token;
    {
        const float* f = reinterpret_cast<const float*>(
            p.records + ((int64_t)c * p.v_heads + kh * group) * p.record_bytes);
        // half of the waves each
        const bool is_q = wave >= kWaves / 2;
        const int id = threadIdx.x & (kThreads / 2 - 1);
        Rows<T, kK, kThreads / 2> u;
        u.load(is_q ? q : k, is_q ? p.q.token : p.k.token, at.count, p.k_size, kWide,
               f + 64 * (is_q ? DeltaRecord::kQueryScale : DeltaRecord::kKeyScale), id);
        u.store(lds + (is_q ? L::kAtQt : L::kAtKt), id);
        if (threadIdx.x < kC) {  // powers of two: exact
            small.key_down[threadIdx.x] = 1.0f / f[64 * DeltaRecord::kKeyScale + threadIdx.x];
            small.query_down[threadIdx.x] = 1.0f / f[64 * DeltaRecord::kQueryScale + threadIdx.x];
        }
    }
    f32x4 dq[kOwn] = {}, dk[kOwn] = {};  // sums over the heads (kShared)
    T* dqo = row_of<T>(p.dq, packed, at.n, at.span, kh) + (int64_t)at.first * p.dq.token;
    T* dko = row_of<T>(p.dk, packed, at.n, at.span, kh) + (int64_t)at.first * p.dk.token;
    const auto put_rows = [&](int i, f32x4 x, f32x4 y) __attribute__((always_inline)) {
        // (Addresses made here: from scratch, each would wait for the store before it.)
        int lane = threadIdx.x & 63;
        __asm__ volatile("" : "+v"(lane));
        const int e = 16 * tile + (lane & 15);
        const __amdgpu_buffer_rsrc_t to_q = buffer_at(dqo), to_k = buffer_at(dko);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int t = 16 * i + 4 * (lane >> 4) + r;
            const bool in = e < p.k_size && t < at.count;
            store_word(from_f32<T>(x[r]), to_q,
                       in ? (t * (uint32_t)p.dq.token + e) * (uint32_t)sizeof(T) : kPastEnd);
            store_word(from_f32<T>(y[r]), to_k,
                       in ? (t * (uint32_t)p.dk.token + e) * (uint32_t)sizeof(T) : kPastEnd);
        }
    };
    for (int h = kh * group; h < (kh + 1) * group; ++h) {
        // Everything that depends on the lane is formed again for every head:
        // kept from one to the next, some 250 LDS addresses would be in scratch.
        int lane = threadIdx.x & 63;
        __asm__ volatile("" : "+v"(lane));
        const int row = lane & 15, g = lane >> 4;
        const int64_t task = (int64_t)c * p.v_heads + h;
        __syncthreads();  // the last head's values are used
        if (wave == 0) {
            const char* record = p.records + task * p.record_bytes;
            const double G = reinterpret_cast<const double*>(record + DeltaRecord::kAtSums)[lane];
            small.G[lane] = G;
            small.rise[lane] = expf((float)G);
            small.tail[lane] = expf((float)(__shfl(G, 63, 64) - G));
            small.beta[lane] = reinterpret_cast<const float*>(record)[64 * DeltaRecord::kBeta + lane];
            small.dot[lane] = 0.0f;
        }
        const T* v = row_of<const T>(p.v, packed, at.n, at.span, h) + (int64_t)at.first * p.v.token;
        const T* d_o = row_of<const T>(p.d_o, packed, at.n, at.span, h) + (int64_t)at.first * p.d_o.token;
        const float* u = p.updates + task * kC * p.v_size;
        const float* dy = p.dsides + task * kC * p.v_size;
        const float* S = p.states + task * ((p.k_size + 15) / 16 * 16) * p.v_size;
        const float* D = p.dstates + task * ((p.k_size + 15) / 16 * 16) * p.v_size;

        f32x4 e1[kOwn] = {}, e2[kOwn] = {}, e3[kOwn] = {}, m[4] = {};
        float sd = 0.0f;
        // A block's rows: this wave's of S and D, to be B operands (columns: key
        // elements), and 16 of dO and U (waves 0 to 3) or of dY and V (4 to 7).  With keys
        // of up to 64 they are loaded while the block before is multiplied (3 x 1001
        // tokens of 6 heads, 64 x 96, in float32: 71 us without, 67 with); with 128 there
        // are no registers for that (2 x 4096 tokens: 268 us without, 333 with).
        constexpr bool kAhead = kK == 64;
        Eight<float> sx[kVSteps], dx[kVSteps], fx[kVSteps];
        Eight<T> tx[kVSteps];
        const auto load_state = [&](const float* from, Eight<float>(&x)[kVSteps], int v0, int lane)
                                    __attribute__((always_inline)) {
            const int ke = 16 * tile + (lane & 15);
#pragma unroll
            for (int j = 0; j < kVSteps; ++j)
                x[j] = load_eight<float>(buffer_at(from), 4u * ke * p.v_size,
                                         v0 + 32 * j + 8 * (lane >> 4), p.v_size, ke < p.k_size, kWide);
        };
        const auto load_rows = [&](int v0, int lane) __attribute__((always_inline)) {
            const int t = 16 * (wave % 4) + (lane & 15);
            const uint32_t at_t = t * (uint32_t)(wave < 4 ? p.d_o.token : p.v.token) *
                                  (uint32_t)sizeof(T);
            const __amdgpu_buffer_rsrc_t rt = buffer_at(wave < 4 ? d_o : v),
                                         rf = buffer_at(wave < 4 ? u : dy);
#pragma unroll
            for (int j = 0; j < kVSteps; ++j) {
                const int e = v0 + 32 * j + 8 * (lane >> 4);
                tx[j] = load_eight<T>(rt, at_t, e, p.v_size, t < at.count, kWide);
                fx[j] = load_eight<float>(rf, 4u * t * p.v_size, e, p.v_size, true, kWide);
            }
        };
        const auto load_all = [&](int v0, int lane) __attribute__((always_inline)) {
            load_state(S, sx, v0, lane);
            load_rows(v0, lane);
            load_state(D, dx, v0, lane);
        };
        if (kAhead) load_all(0, lane);
        for (int v0 = 0; v0 < p.v_size; v0 += kVBlock) {
            __asm__ volatile("" : "+v"(lane));
            const int row = lane & 15, g = lane >> 4;
            lds_barrier();  // the last block's fragments are used
            if (!kAhead) load_all(v0, lane);
            const int t = 16 * (wave % 4) + row;
            const auto put = [&](auto parts, const auto (&x)[kVSteps], char* to, float* down)
                __attribute__((always_inline)) {
                constexpr int kN = decltype(parts)::value;
                float top = 0.0f;
#pragma unroll
                for (int j = 0; j < kVSteps; ++j)
#pragma unroll
                    for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(to_f32(x[j].x[e])));
                const Scale s = scale_of(max_groups(top));
                if (g == 0) down[t] = s.down;
#pragma unroll
                for (int j = 0; j < kVSteps; ++j) {
                    float w[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) w[e] = to_f32(x[j].x[e]);
                    const Frag<kN> f = split<kN>(w, s.up);
#pragma unroll
                    for (int n = 0; n < kN; ++n)
                        *reinterpret_cast<half8_t*>(to + n * L::kPart +
                                                    ((wave % 4) * kVSteps + j) * 1024 + lane * 16) =
                            f.part[n];
                }
            };
            if (wave < 4) {
                put(std::integral_constant<int, L::kParts>{}, tx, lds + L::kAtDo, small.down[0]);
            } else {
                float sum = 0.0f;
#pragma unroll
                for (int j = 0; j < kVSteps; ++j)
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        sum = __builtin_fmaf(fx[j].x[e], to_f32(tx[j].x[e]), sum);
                sum += __shfl_xor(sum, 16, 64);
                sum += __shfl_xor(sum, 32, 64);
                if (g == 0) small.dot[t] += sum;
            }
            put(std::integral_constant<int, 2>{}, fx, lds + (wave < 4 ? L::kAtU : L::kAtDy),
                small.down[wave < 4 ? 2 : 1]);
            float smax = 0.0f, dmax = 0.0f;
#pragma unroll
            for (int j = 0; j < kVSteps; ++j)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    smax = fmaxf(smax, fabsf(sx[j].x[e]));
                    dmax = fmaxf(dmax, fabsf(dx[j].x[e]));
                    if (own == 0) sd = __builtin_fmaf(sx[j].x[e], dx[j].x[e], sd);
                }
            const Scale ss = scale_of(max_groups(smax)), ds = scale_of(max_groups(dmax));
            Frag<2> sb[kVSteps];
#pragma unroll
            for (int j = 0; j < kVSteps; ++j) sb[j] = split<2>(sx[j].x, ss.up);
            lds_barrier();
            if (kAhead) {  // (zero, and not loaded, after the last block)
                load_state(S, sx, v0 + kVBlock, lane);
                load_rows(v0 + kVBlock, lane);
            }
            const auto fragment = [&](auto parts, int from, int i, int j)
                __attribute__((always_inline)) {
                constexpr int kN = decltype(parts)::value;
                Frag<kN> f;
#pragma unroll
                for (int n = 0; n < kN; ++n)
                    f.part[n] = *reinterpret_cast<const half8_t*>(
                        lds + from + n * L::kPart + (i * kVSteps + j) * 1024 + lane * 16);
                return f;
            };
            constexpr std::integral_constant<int, L::kParts> one{};
            constexpr std::integral_constant<int, 2> two{};
            // (the barriers to the scheduler keep few values alive at a time)
#pragma unroll
            for (int i = 0; i < kOwn; ++i) {
                f32x4 a1{}, a2{};
#pragma unroll
                for (int j = 0; j < kVSteps; ++j) {
                    a1 = multiply(fragment(one, L::kAtDo, own + i, j), sb[j], a1);
                    a2 = multiply(fragment(two, L::kAtDy, own + i, j), sb[j], a2);
                }
                const int t = 16 * (own + i) + 4 * g;
                e1[i] += a1 * *reinterpret_cast<const f32x4*>(small.down[0] + t) * ss.down;
                e2[i] += a2 * *reinterpret_cast<const f32x4*>(small.down[1] + t) * ss.down;
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int j = 0; j < kVSteps; ++j) sb[j] = split<2>(dx[j].x, ds.up);
            if (kAhead) load_state(D, dx, v0 + kVBlock, lane);
#pragma unroll
            for (int i = 0; i < kOwn; ++i) {
                f32x4 a3{};
#pragma unroll
                for (int j = 0; j < kVSteps; ++j)
                    a3 = multiply(fragment(two, L::kAtU, own + i, j), sb[j], a3);
                const int t = 16 * (own + i) + 4 * g;
                e3[i] += a3 * *reinterpret_cast<const f32x4*>(small.down[2] + t) * ds.down;
                __builtin_amdgcn_sched_barrier(0);
            }
            // rows wave % 4 of dO U^T (waves 0 to 3) and dY U^T
            const int mt = wave % 4;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (i > mt) continue;
                f32x4 a{};
#pragma unroll
                for (int j = 0; j < kVSteps; ++j) {
                    const Frag<2> b = fragment(two, L::kAtU, i, j);
                    if (wave < 4)
                        a = multiply(fragment(one, L::kAtDo, mt, j), b, a);
                    else
                        a = multiply(fragment(two, L::kAtDy, mt, j), b, a);
                }
                const float cd = small.down[2][16 * i + row];
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    m[i][r] = __builtin_fmaf(a[r], small.down[wave < 4 ? 0 : 1][16 * mt + 4 * g + r] * cd,
                                             m[i][r]);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        __syncthreads();  // dO, dY and U are used
        float* M1 = reinterpret_cast<float*>(lds + L::kAtM);
        float* M2 = M1 + kC * kPitch;
        {
            const int mt = wave % 4;
            float* M = wave < 4 ? M1 : M2;
            double rows[4] = {};
            const char* kk_rows = lds + (wave < 4 ? L::kAtQt : L::kAtKt);
            const int at_t = 4 * mt + g;
            const f32x4 beta = reinterpret_cast<const f32x4*>(small.beta)[at_t];
            f32x4 by = reinterpret_cast<const f32x4*>(wave < 4 ? small.query_down
                                                               : small.key_down)[at_t];
            if (wave >= 4) by *= -beta;
            double Gt[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) Gt[r] = small.G[16 * mt + 4 * g + r];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int s = 16 * i + row;
                double column = 0.0;
                if (i <= mt) {
                    // Q K^T or -diag(beta) K K^T
                    f32x4 kk{};
#pragma unroll
                    for (int j = 0; j < L::kSteps; ++j)
                        kk = multiply(row_fragment<T, kK>(kk_rows, mt, j, lane),
                                      row_fragment<T, kK>(lds + L::kAtKt, i, j, lane), kk);
                    kk *= by * small.key_down[s];
                    const double Gs = small.G[s];
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int t = 16 * mt + 4 * g + r;
                        const bool on = wave < 4 ? s <= t : s < t;
                        const float e = on ? expf((float)(Gt[r] - Gs)) : 0.0f;
                        const float x = on ? (wave < 4 ? p.scale * e : e) * m[i][r] : 0.0f;
                        M[t * kPitch + s] = x;
                        // a token and itself have no decay between them
                        const double y = s < t ? (double)(x * kk[r]) : 0.0;
                        rows[r] += y;
                        column += y;
                    }
                }
                column += __shfl_xor(column, 16, 64);
                column += __shfl_xor(column, 32, 64);
                if (g == 0) small.columns[wave / 4][mt][s] = column;
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                rows[r] = sum_row(rows[r]);
                if (row == 0) small.rows[wave / 4][16 * mt + 4 * g + r] = rows[r];
            }
        }
        __syncthreads();
        {
            const int mt = wave % 4;
            char* to = lds + L::kAtFragments;
            constexpr int kBytes = 2 * DeltaRecord::kMatrix;
            if (wave < 4) {
                write_fragments<false>(M1, small.key_down, nullptr, mt, lane, to, small.m_down[0]);
                write_fragments<true>(M1, small.query_down, nullptr, mt, lane, to + 2 * kBytes,
                                      small.m_down[2]);
            } else {
                write_fragments<false>(M2, small.key_down, nullptr, mt, lane, to + kBytes,
                                       small.m_down[1]);
                write_fragments<true>(M2, small.key_down, small.beta, mt, lane, to + 3 * kBytes,
                                      small.m_down[3]);
            }
        }
        __syncthreads();
        const double last = small.G[kC - 1];
        // K.W, a and b of every tile of elements, where M1 was
        auto& part = *reinterpret_cast<float(*)[3][L::kTiles][kC]>(lds + L::kAtM);
            // this lane's element of K or Q at row 16 i + 4 g + r, scaled as the fragments
            const auto element = [&](const char* rows, int i, int r)
                __attribute__((always_inline)) {
                const char* from = rows + (i * L::kSteps + tile / 2) * 1024 +
                                   slot(((row >> 2) << 4) + 4 * g + r, tile / 2) + 8 * (tile % 2) +
                                   2 * (row & 3);
                float x = (float)*reinterpret_cast<const _Float16*>(from);
                if (L::kParts == 2)
                    x += (float)*reinterpret_cast<const _Float16*>(from + 4 * L::kSteps * 1024);
                return x;
            };
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            const int ti = own + i;
            f32x4 a[4] = {};
            const char* from = lds + L::kAtFragments;
            constexpr int kBytes = 2 * DeltaRecord::kMatrix;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const auto kt = column_fragment<T, kK>(lds + L::kAtKt, tile, j, lane);
                if (j <= ti / 2) {
                    a[0] = multiply(matrix_fragment<2>(from, lower_at(ti, j), lane), kt, a[0]);
                    a[1] = multiply(matrix_fragment<2>(from + kBytes, lower_at(ti, j), lane), kt, a[1]);
                }
                if (j >= ti / 2) {
                    const auto qt = column_fragment<T, kK>(lds + L::kAtQt, tile, j, lane);
                    a[2] = multiply(matrix_fragment<2>(from + 2 * kBytes, upper_at(ti, j), lane), qt, a[2]);
                    a[3] = multiply(matrix_fragment<2>(from + 3 * kBytes, upper_at(ti, j), lane), kt, a[3]);
                }
            }
            const auto of_rows = [&](const float* x) __attribute__((always_inline)) {
                return reinterpret_cast<const f32x4*>(x)[4 * ti + g];
            };
            const f32x4 beta = of_rows(small.beta), rise = of_rows(small.rise);
            const f32x4 de = e1[i] * rise * p.scale, we = e2[i] * rise;
            const f32x4 te = e3[i] * of_rows(small.tail);
            const f32x4 w = -(we + a[1] * of_rows(small.m_down[1]));
            const f32x4 dqt = de + a[0] * of_rows(small.m_down[0]);
            const f32x4 dkt = beta * w + (te + (a[2] * of_rows(small.m_down[2]) -
                                                a[3] * of_rows(small.m_down[3])));
            const f32x4 kdown = of_rows(small.key_down), qdown = of_rows(small.query_down);
            if (kShared) {
                dq[i] += dqt;
                dk[i] += dkt;
            } else {
                put_rows(ti, dqt, dkt);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int t = 16 * ti + 4 * g + r;
                const float kd = element(lds + L::kAtKt, ti, r) * kdown[r];
                const float qd = element(lds + L::kAtQt, ti, r) * qdown[r];
                const float sums[3] = {sum_row(kd * w[r]),
                                       sum_row(__builtin_fmaf(qd, de[r], -(beta[r] * kd * we[r]))),
                                       sum_row(kd * te[r])};
                if (row == 0)
#pragma unroll
                    for (int n = 0; n < 3; ++n) part[n][tile][t] = sums[n];
            }
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int d = 1; d < 64; d *= 2) sd += __shfl_xor(sd, d, 64);
        if (lane == 0) small.end[wave] = sd;
        __syncthreads();
        if (wave == 0) {
            float db = small.dot[lane], s = 0.0f;
            double later = 0.0, before = 0.0;  // summed over i >= t and j <= t
#pragma unroll
            for (int i = 0; i < L::kTiles; ++i) {
                db += part[0][i][lane];
                later += part[1][i][lane];
                before += part[2][i][lane];
            }
#pragma unroll
            for (int i = 0; i < kWaves; ++i) s += small.end[i];
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                later += small.rows[n][lane];
#pragma unroll
                for (int i = 0; i < 4; ++i) later -= small.columns[n][i][lane];
            }
            const double b = before;
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                const double x = __shfl_down(later, d, 64), y = __shfl_up(before, d, 64);
                if (lane + d < 64) later += x;
                if (lane >= d) before += y;
            }
            if (lane < at.count) {
                const int64_t t = at.first + lane;
                if (p.dbeta.p)
                    row_of<float>(p.dbeta, packed, at.n, at.span, h)[t * p.dbeta.token] = db;
                if (p.dg.p)
                    row_of<float>(p.dg, packed, at.n, at.span, h)[t * p.dg.token] =
                        (float)(later + (before - b) + (double)(expf((float)last) * s));
            }
        }
    }
    if (kShared)
#pragma unroll
        for (int i = 0; i < kOwn; ++i) put_rows(own + i, dq[i], dk[i]);
}

template <class T, int kK, bool kWide, bool kShared>
hipError_t launch(const DeltaChunks& a, hipStream_t stream) {
    constexpr int kBytes = Layout<T, kK>::kBytes;
    static_assert(kBytes <= 160 * 1024, "LDS of a CU");
    const void* kernel = reinterpret_cast<const void*>(delta_gradient_kernel<T, kK, kWide, kShared>);
    if (hipError_t e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, kBytes))
        return e;
    hipLaunchKernelGGL((delta_gradient_kernel<T, kK, kWide, kShared>), dim3((unsigned)(a.chunks * a.k_heads)),
                       dim3(kThreads), kBytes, stream, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_delta_gradient(const DeltaChunks& a, hipStream_t stream) {
    if (a.chunks == 0) return hipSuccess;
    return by_dtype(a.dtype, [&](auto t) {
        using T = decltype(t);
        // single-element loads are a kernel of their own: in one with the wide
        // ones they would double its code, which does not fit the instruction
        // cache as it is
        const bool small = a.k_size <= 64;
        if (!a.wide || !a.wide_values)
            return small ? launch<T, 64, false, true>(a, stream)
                         : launch<T, 128, false, true>(a, stream);
        if (a.v_heads > a.k_heads)
            return small ? launch<T, 64, true, true>(a, stream)
                         : launch<T, 128, true, true>(a, stream);
        return small ? launch<T, 64, true, false>(a, stream)
                     : launch<T, 128, true, false>(a, stream);
    });
}

}  // namespace sgemm_emu
