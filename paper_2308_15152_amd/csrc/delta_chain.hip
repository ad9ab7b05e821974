// The gated delta rule, second kernel: the walk over a sequence's chunks that
// carries the state,
//   U = T diag(beta) (V - diag(e^G) K S),
//   O = scale diag(e^G) Q S + P U,   S' = e^{G_64} S + K^T diag(e^{G_64 - G}) U.
//
// Columns of S are independent: a wave owns 16 of them (all rows, in the
// accumulator layout) and carries them through the whole sequence, so the
// chunk's chain of products never leaves its registers.  What bounds it is how
// fast one such wave gets through its instructions, so it is left with those of the
// chain only.  The block's other waves help: they bring K, Q, T, P and V of the next
// chunk into LDS as fragments (each is loaded into registers a chunk ahead), and
// make O from the S and U that the walking waves leave in LDS.  Two barriers a
// chunk: after the first (A) the chunk's K and T are there, after the second (B)
// its S and Q are:
//   walking  A: V to registers, S split and put down.  B: U, put down; next S.
//   helping  A: O of the last chunk finished; Q down.  B: Q S; next K, T, V, this P down.
#include "delta_chunk.hpp"

namespace sgemm_emu {

namespace {

enum { kOutputs, kStates };  // what the walk writes: O, or S and U per chunk

constexpr int kHelpers = 4;

// LDS, in bytes.
template <class T, int kK, int kWalkers, int kMode>
struct Layout {
    static constexpr int kParts = kPartsOf<T>;  // of K and Q
    // of P, and of S and U where they make O: rounding them to fp16 alone costs
    // 2^-12 relative, unseen in a bfloat16 result (2^-8) but not in others
    static constexpr int kOut = __is_same(T, bf16_t) ? 1 : 2;
    static constexpr int kSteps = kK / 32, kTiles = kK / 16;
    static constexpr int kRows = kParts * 4 * kSteps * 1024;  // K or Q
    static constexpr int kMatrices = 2 * DeltaRecord::kMatrix;
    // two buffers of these
    static constexpr int kAtK = 0;
    static constexpr int kAtT = kAtK + kRows;
    static constexpr int kAtF = kAtT + kMatrices;
    static constexpr int kBuffer = kAtF + DeltaRecord::kFactorBytes;
    // one of these
    static constexpr int kAtV = 2 * kBuffer;
    static constexpr int kEachV = kC * 16 * sizeof(T);
    static constexpr int kAtQ = kAtV + kWalkers * kEachV;
    static constexpr int kAtP = kAtQ + (kMode == kOutputs ? kRows : 0);
    static constexpr int kBytesP = kMode == kOutputs ? kOut * DeltaRecord::kMatrix : 0;
    static constexpr int kAtS = kAtP + kBytesP;
    static constexpr int kEachS = kOut * kSteps * 1024 + 256;  // and its scale
    static constexpr int kAtU = kAtS + (kMode == kOutputs ? kWalkers * kEachS : 0);
    static constexpr int kEachU = kC * 16 * 4;
    static constexpr int kBytes = kAtU + (kMode == kOutputs ? kWalkers * kEachU : 0);
};

template <class T, int kK, int kWalkers, int kMode>
__global__ __launch_bounds__(64 * (kWalkers + kHelpers), 1) void delta_chain_kernel(DeltaChunks p) {
    using L = Layout<T, kK, kWalkers, kMode>;
    constexpr int kOut = L::kOut;
    extern __shared__ __attribute__((aligned(16))) char lds[];

    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int g = lane >> 4;
    const int slices = (p.v_size + 16 * kWalkers - 1) / (16 * kWalkers);
    const int slice = blockIdx.x % slices;
    const int h = (blockIdx.x / slices) % p.v_heads, n = blockIdx.x / slices / p.v_heads;
    const int kh = h / (p.v_heads / p.k_heads);
    const bool packed = p.cu_seqlens != nullptr;
    const Span span = span_of(p.cu_seqlens, n, p.tokens);
    const int chunks = (span.count + kC - 1) / kC;
    const int first_chunk = packed ? chunk_base(p.cu_seqlens, n, p.tokens)
                                   : n * ((p.tokens + kC - 1) / kC);
    const int col0 = slice * kWalkers * 16;
    const char* records = p.records + ((int64_t)first_chunk * p.v_heads + h) * p.record_bytes;
    const int64_t record_step = (int64_t)p.v_heads * p.record_bytes;

    if (wave < kWalkers) {
        const int col = col0 + 16 * wave + (lane & 15);
        const bool in = col < p.v_size;
        f32x4 S[L::kTiles];  // rows 16 i + 4 g + r
        const int64_t state = ((int64_t)n * p.v_heads + h) * p.k_size * p.v_size + col;
#pragma unroll
        for (int i = 0; i < L::kTiles; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = 16 * i + 4 * g + r;
                S[i][r] = p.initial && in && row < p.k_size
                              ? p.initial[state + (int64_t)row * p.v_size] : 0.0f;
            }
        const char* v_at = lds + L::kAtV + wave * L::kEachV + lane * 4 * (int)sizeof(T);
        char* s_at = lds + L::kAtS + wave * L::kEachS;
        char* u_at = lds + L::kAtU + wave * L::kEachU + lane * 16;

        for (int c = 0; c < chunks; ++c) {
            const char* at = lds + (c & 1) * L::kBuffer;
            const float* f = reinterpret_cast<const float*>(at + L::kAtF);
            const auto factor = [&](int which, int tile) {
                return reinterpret_cast<const f32x4*>(f + 64 * which)[4 * tile + g];
            };
            lds_barrier();  // A
            T vt[4][4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                __builtin_memcpy(vt[i], v_at + i * 64 * 4 * sizeof(T), 4 * sizeof(T));
            if (kMode == kStates) {
                const int64_t task = (int64_t)(first_chunk + c) * p.v_heads + h;
                const __amdgpu_buffer_rsrc_t to =
                    buffer_at(p.states + task * ((p.k_size + 15) / 16 * 16) * p.v_size);
                const uint32_t off = in ? 4u * (4 * g * p.v_size + col) : kPastEnd;
#pragma unroll
                for (int i = 0; i < L::kTiles; ++i)
                    if (16 * i < p.k_size)
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            __builtin_amdgcn_raw_buffer_store_b32(
                                __builtin_bit_cast(uint32_t, (float)S[i][r]), to, off,
                                4 * (16 * i + r) * p.v_size, 0);
            }
            const Scale ss = scale_of(max_groups(largest(S)));
            Frag<2> sb[L::kSteps];
#pragma unroll
            for (int j = 0; j < L::kSteps; ++j) {
                sb[j] = split<2>(S[2 * j], S[2 * j + 1], ss.up);
                if (kMode == kOutputs)
#pragma unroll
                    for (int q = 0; q < kOut; ++q)
                        *reinterpret_cast<half8_t*>(s_at + (q * L::kSteps + j) * 1024 + lane * 16) =
                            sb[j].part[q];
            }
            if (kMode == kOutputs)
                reinterpret_cast<float*>(s_at + kOut * L::kSteps * 1024)[lane] = ss.down;
            lds_barrier();  // B
            // beta (V - e^G K S)
            f32x4 x[4] = {};
#pragma unroll
            for (int j = 0; j < L::kSteps; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    x[i] = multiply(row_fragment<T, kK>(at + L::kAtK, i, j, lane), sb[j], x[i]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f32x4 rise = factor(DeltaRecord::kRise, i) * ss.down;
                const f32x4 beta = factor(DeltaRecord::kBeta, i);
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    x[i][r] = beta[r] * __builtin_fmaf(-rise[r], x[i][r], to_f32(vt[i][r]));
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
                        u[i] = multiply(matrix_fragment<2>(at + L::kAtT, lower_at(i, j), lane), b[j],
                                        u[i]);
                    u[i] *= factor(DeltaRecord::kT, i) * xs.down;
                    if (kMode == kOutputs) *reinterpret_cast<f32x4*>(u_at + i * 1024) = u[i];
                }
            }
            if (kMode == kStates) {
                const int64_t task = (int64_t)(first_chunk + c) * p.v_heads + h;
                const __amdgpu_buffer_rsrc_t to = buffer_at(p.updates + task * kC * p.v_size);
                const uint32_t off = in ? 4u * (4 * g * p.v_size + col) : kPastEnd;
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        __builtin_amdgcn_raw_buffer_store_b32(
                            __builtin_bit_cast(uint32_t, (float)u[i][r]), to, off,
                            4 * (16 * i + r) * p.v_size, 0);
            }
            // S
#pragma unroll
            for (int i = 0; i < 4; ++i) u[i] *= factor(DeltaRecord::kTail, i);
            const Scale us = scale_of(max_groups(largest(u)));
            const Frag<2> b[2] = {split<2>(u[0], u[1], us.up), split<2>(u[2], u[3], us.up)};
            const float decay = f[64 * DeltaRecord::kDecay];
#pragma unroll
            for (int i = 0; i < L::kTiles; ++i) {
                f32x4 a{};
#pragma unroll
                for (int j = 0; j < 2; ++j)  // lo.lo too: updates of like keys cancel
                    a = multiply<true>(column_fragment<T, kK>(at + L::kAtK, i, j, lane), b[j], a);
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    S[i][r] = __builtin_fmaf(a[r], us.down, decay * S[i][r]);
            }
        }
        if (kMode == kOutputs && chunks > 0) lds_barrier();  // the last U
        if (p.final_state && in)
#pragma unroll
            for (int i = 0; i < L::kTiles; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int row = 16 * i + 4 * g + r;
                    if (row < p.k_size) p.final_state[state + (int64_t)row * p.v_size] = S[i][r];
                }
        return;
    }

    // ---- the helping waves
    constexpr int kThreads = 64 * kHelpers;
    constexpr int kMine = (Unit<T, kK>::kUnits + kThreads - 1) / kThreads;
    const int id = threadIdx.x - 64 * kWalkers;
    const T* k = row_of<const T>(p.k, packed, n, span, kh);
    const T* q = row_of<const T>(p.q, packed, n, span, kh);
    const T* v = row_of<const T>(p.v, packed, n, span, h);
    // V goes down as the walking waves hold it: a thread takes 4 tokens x 4 columns
    constexpr int kVUnits = 16 * 4 * kWalkers;
    const int v_four = id / (4 * kWalkers), v_cols = id % (4 * kWalkers) * 4;

    Unit<T, kK> ku[kMine], qu[kMine];
    f32x4 kscale[kMine], qscale[kMine];
    Copy<L::kMatrices, kThreads> tcopy;
    Copy<DeltaRecord::kFactorBytes, kThreads> fcopy;
    Copy<L::kBytesP == 0 ? 16 : L::kBytesP, kThreads> pcopy;
    T vu[4][4];
    const auto load_k = [&](int c) {
        const int count = min(kC, span.count - c * kC);
        const char* record = records + c * record_step;
        const float* f = reinterpret_cast<const float*>(record);
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            const int unit = id + i * kThreads;
            if (Unit<T, kK>::kUnits % kThreads != 0 && unit >= Unit<T, kK>::kUnits) continue;
            ku[i].load(k + (int64_t)c * kC * p.k.token, p.k.token, unit, count, p.k_size, p.wide);
            kscale[i] = reinterpret_cast<const f32x4*>(f + 64 * DeltaRecord::kKeyScale)[unit / (kK / 8)];
        }
        tcopy.load(record + DeltaRecord::kAtT, id);
        fcopy.load(record, id);
        if (kVUnits >= kThreads || id < kVUnits) {
            const __amdgpu_buffer_rsrc_t r = buffer_at(v + (int64_t)c * kC * p.v.token + col0);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int t = 4 * v_four + i;
                const uint32_t off = (t * (uint32_t)p.v.token + v_cols) * sizeof(T);
                if (p.wide_values) {
                    const uint32_t o = t < count && col0 + v_cols < p.v_size ? off : kPastEnd;
                    if (sizeof(T) == 2) {
                        const u32x2 w = __builtin_amdgcn_raw_buffer_load_b64(r, o, 0, 0);
                        __builtin_memcpy(vu[i], &w, 8);
                    } else {
                        const u32x4 w = __builtin_amdgcn_raw_buffer_load_b128(r, o, 0, 0);
                        __builtin_memcpy(vu[i], &w, 4 * sizeof(T));
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        vu[i][e] = load_word<T>(r, t < count && col0 + v_cols + e < p.v_size
                                                       ? off + e * (uint32_t)sizeof(T) : kPastEnd);
                }
            }
        }
    };
    const auto store_k = [&](int c) {
        char* to = lds + (c & 1) * L::kBuffer;
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            const int unit = id + i * kThreads;
            if (Unit<T, kK>::kUnits % kThreads != 0 && unit >= Unit<T, kK>::kUnits) continue;
            ku[i].store(to + L::kAtK, unit, kscale[i]);
        }
        tcopy.store(to + L::kAtT, id);
        fcopy.store(to + L::kAtF, id);
        if (kVUnits >= kThreads || id < kVUnits) {
            char* at = lds + L::kAtV + v_cols / 16 * L::kEachV +
                       (v_four / 4 * 64 + v_four % 4 * 16 + v_cols % 16) * 4 * sizeof(T);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const T w[4] = {vu[0][e], vu[1][e], vu[2][e], vu[3][e]};
                __builtin_memcpy(at + e * 4 * sizeof(T), w, 4 * sizeof(T));
            }
        }
    };
    const auto load_q = [&](int c) {
        const int count = min(kC, span.count - c * kC);
        const char* record = records + c * record_step;
        const float* f = reinterpret_cast<const float*>(record);
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            const int unit = id + i * kThreads;
            if (Unit<T, kK>::kUnits % kThreads != 0 && unit >= Unit<T, kK>::kUnits) continue;
            qu[i].load(q + (int64_t)c * kC * p.q.token, p.q.token, unit, count, p.k_size, p.wide);
            qscale[i] = reinterpret_cast<const f32x4*>(f + 64 * DeltaRecord::kQueryScale)[unit / (kK / 8)];
        }
        pcopy.load(record + DeltaRecord::kAtP, id);
    };

    // O: 16 columns and kOwn token tiles of a chunk to a wave
    constexpr int kOwn = 4 * kWalkers / kHelpers;
    const int helper = wave - kWalkers;
    const int block = helper % kWalkers, own = helper / kWalkers * kOwn;
    const int col = col0 + 16 * block + (lane & 15);
    const bool in = col < p.v_size;
    T* o = kMode == kOutputs ? row_of<T>(p.o, packed, n, span, h) : nullptr;
    f32x4 y[kOwn];

    if (chunks > 0) {
        load_k(0);
        store_k(0);
        if (chunks > 1) load_k(1);
        if (kMode == kOutputs) load_q(0);
    }
    for (int c = 0; c < chunks; ++c) {
        lds_barrier();  // A
        const auto finish = [&](int c) {
            const float* f = reinterpret_cast<const float*>(lds + (c & 1) * L::kBuffer + L::kAtF);
            const char* u_at = lds + L::kAtU + block * L::kEachU + lane * 16;
            f32x4 u[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) u[i] = *reinterpret_cast<const f32x4*>(u_at + i * 1024);
            const Scale us = scale_of(max_groups(largest(u)));
            const Frag<kOut> b[2] = {split<kOut>(u[0], u[1], us.up), split<kOut>(u[2], u[3], us.up)};
            const int count = min(kC, span.count - c * kC);
            const __amdgpu_buffer_rsrc_t to = buffer_at(o + (int64_t)c * kC * p.o.token);
#pragma unroll
            for (int i = 0; i < kOwn; ++i) {
                const int tile = own + i;
                f32x4 a{};
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    if (j <= tile / 2)
                        a = multiply(matrix_fragment<kOut>(lds + L::kAtP, lower_at(tile, j), lane),
                                     b[j], a);
                const f32x4 pf = reinterpret_cast<const f32x4*>(f + 64 * DeltaRecord::kP)[4 * tile + g] * us.down;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int t = 16 * tile + 4 * g + r;
                    store_word(from_f32<T>(__builtin_fmaf(pf[r], a[r], y[i][r])), to,
                               in && t < count ? (t * (uint32_t)p.o.token + col) * (uint32_t)sizeof(T)
                                               : kPastEnd);
                }
            }
        };
        if (kMode == kOutputs) {
            if (c > 0) finish(c - 1);
#pragma unroll
            for (int i = 0; i < kMine; ++i) {
                const int unit = id + i * kThreads;
                if (Unit<T, kK>::kUnits % kThreads != 0 && unit >= Unit<T, kK>::kUnits) continue;
                qu[i].store(lds + L::kAtQ, unit, qscale[i]);
            }
        }
        lds_barrier();  // B
        if (kMode == kOutputs) {
            pcopy.store(lds + L::kAtP, id);
            if (c + 1 < chunks) load_q(c + 1);
        }
        if (c + 1 < chunks) store_k(c + 1);
        if (c + 2 < chunks) load_k(c + 2);
        if (kMode == kOutputs) {
            const float* f = reinterpret_cast<const float*>(lds + (c & 1) * L::kBuffer + L::kAtF);
            const char* s_at = lds + L::kAtS + block * L::kEachS;
            const float down = reinterpret_cast<const float*>(s_at + kOut * L::kSteps * 1024)[lane];
#pragma unroll
            for (int i = 0; i < kOwn; ++i) y[i] = f32x4{};
#pragma unroll
            for (int j = 0; j < L::kSteps; ++j) {
                Frag<kOut> b;
#pragma unroll
                for (int r = 0; r < kOut; ++r)
                    b.part[r] = *reinterpret_cast<const half8_t*>(
                        s_at + (r * L::kSteps + j) * 1024 + lane * 16);
#pragma unroll
                for (int i = 0; i < kOwn; ++i)
                    y[i] = multiply(row_fragment<T, kK>(lds + L::kAtQ, own + i, j, lane), b, y[i]);
            }
#pragma unroll
            for (int i = 0; i < kOwn; ++i)
                y[i] *= reinterpret_cast<const f32x4*>(f + 64 * DeltaRecord::kQueryRise)[4 * (own + i) + g] * down;
            if (c + 1 == chunks) {
                lds_barrier();  // the last U
                finish(c);
            }
        }
    }
}

template <class T, int kK, int kWalkers, int kMode>
hipError_t launch(const DeltaChunks& a, hipStream_t stream) {
    constexpr int kBytes = Layout<T, kK, kWalkers, kMode>::kBytes;
    static_assert(kBytes <= 160 * 1024, "LDS of a CU");
    const int64_t slices = (a.v_size + 16 * kWalkers - 1) / (16 * kWalkers);
    const void* kernel = reinterpret_cast<const void*>(delta_chain_kernel<T, kK, kWalkers, kMode>);
    if (hipError_t e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, kBytes))
        return e;
    hipLaunchKernelGGL((delta_chain_kernel<T, kK, kWalkers, kMode>),
                       dim3((unsigned)(slices * a.v_heads * a.batch)),
                       dim3(64 * (kWalkers + kHelpers)), kBytes, stream, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_delta_chain(const DeltaChunks& a, hipStream_t stream) {
    return by_dtype(a.dtype, [&](auto t) {
        using T = decltype(t);
        constexpr bool kF32 = sizeof(T) == 4;
        if (a.backward)
            return a.k_size <= 64 ? launch<T, 64, 2, kStates>(a, stream)
                                  : launch<T, 128, 2, kStates>(a, stream);
        return a.k_size <= 64 ? launch<T, 64, 2, kOutputs>(a, stream)
                              : launch<T, 128, kF32 ? 1 : 2, kOutputs>(a, stream);
    });
}

}  // namespace sgemm_emu
