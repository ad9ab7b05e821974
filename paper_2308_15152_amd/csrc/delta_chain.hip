// The gated delta rule, second kernel: the walk over a sequence's chunks that
// carries the state,
//   U = T diag(beta) (V - diag(e^G) K S),
//   O = scale diag(e^G) Q S + P U,   S' = e^{G_64} S + K^T diag(e^{G_64 - G}) U.
//
// Columns of S are independent: a wave owns 16 of them (all rows, in the
// accumulator layout) and carries them through the whole sequence, so the
// chunk's chain of products never leaves its registers and needs no barrier.
// The waves of a block share one head's K, Q, T and P, staged in LDS as A
// fragments; the next chunk's are loaded into registers while the current one
// is computed.
#include "delta_chunk.hpp"

namespace sgemm_emu {

namespace {

enum { kOutputs, kStates };  // what the walk writes: O, or S and U per chunk

// LDS of one chunk, in bytes.
template <class T, int kK, int kMode>
struct Layout {
    static constexpr int kParts = sizeof(T) == 4 ? 2 : 1;  // of K and Q
    // of P, and of S and U where they make O: rounding them to fp16 alone costs
    // 2^-12 relative, unseen in a bfloat16 result (2^-8) but not in others
    static constexpr int kOut = __is_same(T, bf16_t) ? 1 : 2;
    static constexpr int kSteps = kK / 32, kTiles = kK / 16;
    static constexpr int kRows = 4 * kSteps * 1024;  // one part of K or Q
    static constexpr int kAtK = 0;
    static constexpr int kAtKt = kAtK + kParts * kRows;
    static constexpr int kAtQ = kAtKt + kParts * kRows;
    static constexpr int kAtT = kAtQ + (kMode == kOutputs ? kParts * kRows : 0);
    static constexpr int kAtP = kAtT + 2 * DeltaRecord::kMatrix;
    static constexpr int kAtF = kAtP + (kMode == kOutputs ? kOut * DeltaRecord::kMatrix : 0);
    static constexpr int kBytes = kAtF + DeltaRecord::kFactorBytes;
    // two buffers where they fit: then one barrier a chunk
    static constexpr int kBuffers = 2 * kBytes <= 160 * 1024 ? 2 : 1;
};

template <class T, int kK, int kWaves, int kMode>
__global__ __launch_bounds__(64 * kWaves, 1) void delta_chain_kernel(DeltaChunks p) {
    using L = Layout<T, kK, kMode>;
    constexpr int kThreads = 64 * kWaves;
    constexpr int kUnits = 16 * kK / 8;  // 4 x 8 pieces of K or Q
    constexpr int kMine = (kUnits + kThreads - 1) / kThreads;
    constexpr int kCopy = (L::kAtF - L::kAtT) / 16;  // 16-byte pieces of T and P
    constexpr int kCopies = (kCopy + kThreads - 1) / kThreads;
    constexpr int kFactors = DeltaRecord::kFactorBytes / 16;
    constexpr int kFactorCopies = (kFactors + kThreads - 1) / kThreads;
    extern __shared__ __attribute__((aligned(16))) char lds[];

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int g = lane >> 4;
    const int slices = (p.v_size + 16 * kWaves - 1) / (16 * kWaves);
    const int slice = blockIdx.x % slices;
    const int h = (blockIdx.x / slices) % p.v_heads, n = blockIdx.x / slices / p.v_heads;
    const int kh = h / (p.v_heads / p.k_heads);
    const bool packed = p.cu_seqlens != nullptr;
    const Span span = span_of(p.cu_seqlens, n, p.tokens);
    const int chunks = (span.count + kC - 1) / kC;
    const int first_chunk = packed ? chunk_base(p.cu_seqlens, n, p.tokens)
                                   : n * ((p.tokens + kC - 1) / kC);
    const int col = (slice * kWaves + wave) * 16 + (lane & 15);
    const bool in = col < p.v_size;

    const T* k = row_of<const T>(p.k, packed, n, span, kh);
    const T* q = row_of<const T>(p.q, packed, n, span, kh);
    const T* v = row_of<const T>(p.v, packed, n, span, h) + col;
    T* o = kMode == kOutputs ? row_of<T>(p.o, packed, n, span, h) + col : nullptr;

    // state, rows 16 i + 4 g + r
    f32x4 S[L::kTiles];
    const int64_t state = ((int64_t)n * p.v_heads + h) * p.k_size * p.v_size + col;
#pragma unroll
    for (int i = 0; i < L::kTiles; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int row = 16 * i + 4 * g + r;
            S[i][r] = p.initial && in && row < p.k_size
                          ? p.initial[state + (int64_t)row * p.v_size] : 0.0f;
        }

    // what the next chunk needs, on its way
    Unit<T, kK> ku[kMine], qu[kMine];
    f32x4 kscale[kMine], qscale[kMine];
    u32x4 copy[kCopies], fcopy[kFactorCopies];
    T vt[4][4];
    const auto load_next = [&](int c) {
        const int count = min(kC, span.count - c * kC);
        const char* record =
            p.records + ((int64_t)(first_chunk + c) * p.v_heads + h) * p.record_bytes;
        const float* f = reinterpret_cast<const float*>(record);
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            const int unit = threadIdx.x + i * kThreads;
            if (kUnits % kThreads != 0 && unit >= kUnits) continue;
            ku[i].load(k + (int64_t)c * kC * p.k.token, p.k.token, unit, count, p.k_size, p.wide);
            kscale[i] = reinterpret_cast<const f32x4*>(f + 64 * DeltaRecord::kKeyScale)[unit / (kK / 8)];
            if (kMode == kOutputs) {
                qu[i].load(q + (int64_t)c * kC * p.q.token, p.q.token, unit, count, p.k_size, p.wide);
                qscale[i] = reinterpret_cast<const f32x4*>(f + 64 * DeltaRecord::kQueryScale)[unit / (kK / 8)];
            }
        }
#pragma unroll
        for (int i = 0; i < kCopies; ++i) {
            const int at = threadIdx.x + i * kThreads;
            if (at < kCopy) copy[i] = reinterpret_cast<const u32x4*>(record + DeltaRecord::kAtT)[at];
        }
#pragma unroll
        for (int i = 0; i < kFactorCopies; ++i) {
            const int at = threadIdx.x + i * kThreads;
            if (at < kFactors) fcopy[i] = reinterpret_cast<const u32x4*>(record)[at];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int t = 16 * i + 4 * g + r;
                vt[i][r] = in && t < count ? v[(int64_t)(c * kC + t) * p.v.token] : from_f32<T>(0.0f);
            }
    };
    const auto store_next = [&](char* to) {
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            const int unit = threadIdx.x + i * kThreads;
            if (kUnits % kThreads != 0 && unit >= kUnits) continue;
            ku[i].template store<true, true>(to + L::kAtK, to + L::kAtKt, unit, kscale[i]);
            if (kMode == kOutputs)
                qu[i].template store<true, false>(to + L::kAtQ, nullptr, unit, qscale[i]);
        }
#pragma unroll
        for (int i = 0; i < kCopies; ++i) {
            const int at = threadIdx.x + i * kThreads;
            if (at < kCopy) reinterpret_cast<u32x4*>(to + L::kAtT)[at] = copy[i];
        }
#pragma unroll
        for (int i = 0; i < kFactorCopies; ++i) {
            const int at = threadIdx.x + i * kThreads;
            if (at < kFactors) reinterpret_cast<u32x4*>(to + L::kAtF)[at] = fcopy[i];
        }
    };

    if (chunks > 0) {
        load_next(0);
        store_next(lds);
    }
    for (int c = 0; c < chunks; ++c) {
        const char* at = lds + (L::kBuffers == 2 ? (c & 1) * L::kBytes : 0);
        const float* f = reinterpret_cast<const float*>(at + L::kAtF);
        const auto factor = [&](int which, int tile) {
            return reinterpret_cast<const f32x4*>(f + 64 * which)[4 * tile + g];
        };
        const int count = min(kC, span.count - c * kC);
        float vc[4][4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) vc[i][r] = to_f32(vt[i][r]);
        __syncthreads();  // the chunk is in LDS
        if (c + 1 < chunks) load_next(c + 1);

        if (kMode == kStates) {
            float* to = p.states + ((int64_t)(first_chunk + c) * p.v_heads + h) * p.k_size * p.v_size + col;
#pragma unroll
            for (int i = 0; i < L::kTiles; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int row = 16 * i + 4 * g + r;
                    if (in && row < p.k_size) to[(int64_t)row * p.v_size] = S[i][r];
                }
        }

        // K S and Q S
        const Scale ss = scale_of(max_groups(largest(S)));
        f32x4 x[4] = {}, y[4] = {};
#pragma unroll
        for (int j = 0; j < L::kSteps; ++j) {
            const Frag<2> b = split<2>(S[2 * j], S[2 * j + 1], ss.up);
            Frag<L::kOut> bo;
            bo.part[0] = b.part[0];
            if (L::kOut == 2) bo.part[L::kOut - 1] = b.part[1];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[i] = multiply(row_fragment<T, kK>(at + L::kAtK, i, j, lane), b, x[i]);
                if (kMode == kOutputs)
                    y[i] = multiply(row_fragment<T, kK>(at + L::kAtQ, i, j, lane), bo, y[i]);
            }
        }
        // beta (V - e^G K S)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f32x4 rise = factor(DeltaRecord::kRise, i), beta = factor(DeltaRecord::kBeta, i);
#pragma unroll
            for (int r = 0; r < 4; ++r)
                x[i][r] = beta[r] * __builtin_fmaf(-(rise[r] * ss.down), x[i][r], vc[i][r]);
        }
        // U
        f32x4 u[4] = {};
        {
            const Scale xs = scale_of(max_groups(largest(x)));
            const Frag<2> b[2] = {split<2>(x[0], x[1], xs.up), split<2>(x[2], x[3], xs.up)};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
#pragma unroll
                for (int j = 0; j <= i / 2; ++j)
                    u[i] = multiply(matrix_fragment<2>(at + L::kAtT, lower_at(i, j), lane), b[j], u[i]);
                const f32x4 t = factor(DeltaRecord::kT, i);
#pragma unroll
                for (int r = 0; r < 4; ++r) u[i][r] *= t[r] * xs.down;
            }
        }
        if (kMode == kStates) {
            float* to = p.updates + ((int64_t)(first_chunk + c) * p.v_heads + h) * kC * p.v_size + col;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (in) to[(int64_t)(16 * i + 4 * g + r) * p.v_size] = u[i][r];
        }
        // S
        {
            f32x4 w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = u[i] * factor(DeltaRecord::kTail, i);
            const Scale ws = scale_of(max_groups(largest(w)));
            const Frag<2> b[2] = {split<2>(w[0], w[1], ws.up), split<2>(w[2], w[3], ws.up)};
            const float decay = f[64 * DeltaRecord::kDecay];
#pragma unroll
            for (int i = 0; i < L::kTiles; ++i) {
                f32x4 a{};
#pragma unroll
                for (int j = 0; j < 2; ++j)  // lo.lo too: updates of like keys cancel
                    a = multiply<true>(column_fragment<T, kK>(at + L::kAtKt, i, j, lane), b[j], a);
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    S[i][r] = __builtin_fmaf(a[r], ws.down, decay * S[i][r]);
            }
        }
        // O
        if (kMode == kOutputs) {
            const Scale us = scale_of(max_groups(largest(u)));
            const Frag<L::kOut> b[2] = {split<L::kOut>(u[0], u[1], us.up),
                                        split<L::kOut>(u[2], u[3], us.up)};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                f32x4 a{};
#pragma unroll
                for (int j = 0; j <= i / 2; ++j)
                    a = multiply(matrix_fragment<L::kOut>(at + L::kAtP, lower_at(i, j), lane), b[j], a);
                const f32x4 pf = factor(DeltaRecord::kP, i), qf = factor(DeltaRecord::kQueryRise, i);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int t = 16 * i + 4 * g + r;
                    const float out = __builtin_fmaf(qf[r] * ss.down, y[i][r], pf[r] * us.down * a[r]);
                    if (in && t < count) o[(int64_t)(c * kC + t) * p.o.token] = from_f32<T>(out);
                }
            }
        }
        if (c + 1 < chunks) {
            if (L::kBuffers == 1) __syncthreads();  // all waves are through with the chunk
            store_next(lds + (L::kBuffers == 2 ? ((c + 1) & 1) * L::kBytes : 0));
        }
    }
    if (p.final_state && in)
#pragma unroll
        for (int i = 0; i < L::kTiles; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = 16 * i + 4 * g + r;
                if (row < p.k_size) p.final_state[state + (int64_t)row * p.v_size] = S[i][r];
            }
}

template <class T, int kK, int kWaves, int kMode>
hipError_t launch(const DeltaChunks& a, hipStream_t stream) {
    using L = Layout<T, kK, kMode>;
    constexpr int kBytes = L::kBuffers * L::kBytes;
    const int64_t slices = (a.v_size + 16 * kWaves - 1) / (16 * kWaves);
    const void* kernel = reinterpret_cast<const void*>(delta_chain_kernel<T, kK, kWaves, kMode>);
    if (hipError_t e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, kBytes))
        return e;
    hipLaunchKernelGGL((delta_chain_kernel<T, kK, kWaves, kMode>),
                       dim3((unsigned)(slices * a.v_heads * a.batch)), dim3(64 * kWaves), kBytes,
                       stream, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_delta_chain(const DeltaChunks& a, hipStream_t stream) {
    return by_dtype(a.dtype, [&](auto t) {
        using T = decltype(t);
        const bool small = a.k_size <= 64;
        if (a.backward)
            return small ? launch<T, 64, 4, kStates>(a, stream) : launch<T, 128, 4, kStates>(a, stream);
        return small ? launch<T, 64, 4, kOutputs>(a, stream) : launch<T, 128, 4, kOutputs>(a, stream);
    });
}

}  // namespace sgemm_emu
