// The gated delta rule's gradient, the walk back over a sequence's chunks with
// the gradient D of the state after the chunk:
//   dU = P^T dO + diag(e^{G_64 - G}) K D,   dY = T^T dU,   dV = diag(beta) dY,
//   D before = e^{G_64} D + scale (diag(e^G) Q)^T dO - (diag(e^G) K)^T dV.
// Columns are independent here too: laid out, staged and bound like the walk
// forward (delta_chain.hip).  Leaves D after and dY of every chunk.
#include "delta_chunk.hpp"

namespace sgemm_emu {

namespace {

template <class T, int kK>
struct Layout {
    static constexpr int kParts = kPartsOf<T>;
    static constexpr int kSteps = kK / 32, kTiles = kK / 16;
    static constexpr int kRows = 4 * kSteps * 1024;
    static constexpr int kAtK = 0;
    static constexpr int kAtQt = kAtK + kParts * kRows;
    static constexpr int kAtTt = kAtQt + kParts * kRows;
    static constexpr int kAtPt = kAtTt + 2 * DeltaRecord::kMatrix;
    static constexpr int kAtF = kAtPt + 2 * DeltaRecord::kMatrix;
    static constexpr int kBytes = kAtF + DeltaRecord::kFactorBytes;
    static constexpr int kBuffers = 2 * kBytes <= 160 * 1024 ? 2 : 1;
};

template <class T, int kK, int kWaves>
__global__ __launch_bounds__(64 * kWaves, 1) void delta_back_kernel(DeltaChunks p) {
    using L = Layout<T, kK>;
    constexpr int kThreads = 64 * kWaves;
    constexpr int kUnits = 16 * kK / 8;
    constexpr int kMine = (kUnits + kThreads - 1) / kThreads;
    constexpr int kCopy = (L::kAtF - L::kAtTt) / 16;  // 16-byte pieces of T^T and P^T
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
    const T* d_o = row_of<const T>(p.d_o, packed, n, span, h) + col;
    T* dv = row_of<T>(p.dv, packed, n, span, h) + col;

    f32x4 D[L::kTiles];
    const int64_t state = ((int64_t)n * p.v_heads + h) * p.k_size * p.v_size + col;
#pragma unroll
    for (int i = 0; i < L::kTiles; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int row = 16 * i + 4 * g + r;
            D[i][r] = p.dfinal && in && row < p.k_size ? p.dfinal[state + (int64_t)row * p.v_size]
                                                       : 0.0f;
        }

    Unit<T, kK> ku[kMine], qu[kMine];
    f32x4 kscale[kMine], qscale[kMine];
    u32x4 copy[kCopies], fcopy[kFactorCopies];
    T dt[4][4];
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
            qu[i].load(q + (int64_t)c * kC * p.q.token, p.q.token, unit, count, p.k_size, p.wide);
            kscale[i] = reinterpret_cast<const f32x4*>(f + 64 * DeltaRecord::kKeyScale)[unit / (kK / 8)];
            qscale[i] = reinterpret_cast<const f32x4*>(f + 64 * DeltaRecord::kQueryScale)[unit / (kK / 8)];
        }
#pragma unroll
        for (int i = 0; i < kCopies; ++i) {
            const int at = threadIdx.x + i * kThreads;
            if (at < kCopy) copy[i] = reinterpret_cast<const u32x4*>(record + DeltaRecord::kAtTt)[at];
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
                dt[i][r] = in && t < count ? d_o[(int64_t)(c * kC + t) * p.d_o.token]
                                           : from_f32<T>(0.0f);
            }
    };
    const auto store_next = [&](char* to) {
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            const int unit = threadIdx.x + i * kThreads;
            if (kUnits % kThreads != 0 && unit >= kUnits) continue;
            ku[i].store(to + L::kAtK, unit, kscale[i]);
            qu[i].store(to + L::kAtQt, unit, qscale[i]);
        }
#pragma unroll
        for (int i = 0; i < kCopies; ++i) {
            const int at = threadIdx.x + i * kThreads;
            if (at < kCopy) reinterpret_cast<u32x4*>(to + L::kAtTt)[at] = copy[i];
        }
#pragma unroll
        for (int i = 0; i < kFactorCopies; ++i) {
            const int at = threadIdx.x + i * kThreads;
            if (at < kFactors) reinterpret_cast<u32x4*>(to + L::kAtF)[at] = fcopy[i];
        }
    };

    if (chunks > 0) {
        load_next(chunks - 1);
        store_next(lds + (L::kBuffers == 2 ? ((chunks - 1) & 1) * L::kBytes : 0));
    }
    for (int c = chunks - 1; c >= 0; --c) {
        const char* at = lds + (L::kBuffers == 2 ? (c & 1) * L::kBytes : 0);
        const float* f = reinterpret_cast<const float*>(at + L::kAtF);
        const auto factor = [&](int which, int tile) {
            return reinterpret_cast<const f32x4*>(f + 64 * which)[4 * tile + g];
        };
        const int count = min(kC, span.count - c * kC);
        const int64_t task = (int64_t)(first_chunk + c) * p.v_heads + h;
        f32x4 o[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) o[i][r] = to_f32(dt[i][r]);
        __syncthreads();  // the chunk is in LDS
        if (c > 0) load_next(c - 1);

        float* to = p.dstates + task * p.k_size * p.v_size + col;
#pragma unroll
        for (int i = 0; i < L::kTiles; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = 16 * i + 4 * g + r;
                if (in && row < p.k_size) to[(int64_t)row * p.v_size] = D[i][r];
            }

        // dU
        f32x4 u[4] = {};
        {
            const Scale s = scale_of(max_groups(largest(D)));
#pragma unroll
            for (int j = 0; j < L::kSteps; ++j) {
                const Frag<2> b = split<2>(D[2 * j], D[2 * j + 1], s.up);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    u[i] = multiply(row_fragment<T, kK>(at + L::kAtK, i, j, lane), b, u[i]);
            }
            const Scale os = scale_of(max_groups(largest(o)));
            const Frag<L::kParts> b[2] = {split<L::kParts>(o[0], o[1], os.up),
                                          split<L::kParts>(o[2], o[3], os.up)};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                f32x4 a{};
#pragma unroll
                for (int j = i / 2; j < 2; ++j)
                    a = multiply(matrix_fragment<2>(at + L::kAtPt, upper_at(i, j), lane), b[j], a);
                const f32x4 tail = factor(DeltaRecord::kTail, i), pf = factor(DeltaRecord::kPt, i);
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    u[i][r] = __builtin_fmaf(tail[r] * s.down, u[i][r], pf[r] * os.down * a[r]);
            }
        }
        // dY, and dV
        f32x4 y[4] = {};
        {
            const Scale s = scale_of(max_groups(largest(u)));
            const Frag<2> b[2] = {split<2>(u[0], u[1], s.up), split<2>(u[2], u[3], s.up)};
            float* dy = p.dsides + task * kC * p.v_size + col;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
#pragma unroll
                for (int j = i / 2; j < 2; ++j)
                    y[i] = multiply(matrix_fragment<2>(at + L::kAtTt, upper_at(i, j), lane), b[j], y[i]);
                const f32x4 tf = factor(DeltaRecord::kTt, i), beta = factor(DeltaRecord::kBeta, i);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int t = 16 * i + 4 * g + r;
                    y[i][r] *= tf[r] * s.down;
                    if (in) dy[(int64_t)t * p.v_size] = y[i][r];
                    y[i][r] *= beta[r];
                    if (in && t < count)
                        dv[(int64_t)(c * kC + t) * p.dv.token] = from_f32<T>(y[i][r]);
                }
            }
        }
        // D: both products in one accumulator, under one scale
        {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                o[i] *= factor(DeltaRecord::kQueryRise, i);
                y[i] *= -factor(DeltaRecord::kRise, i);
            }
            const Scale s = scale_of(max_groups(fmaxf(largest(o), largest(y))));
            const Frag<2> bo[2] = {split<2>(o[0], o[1], s.up), split<2>(o[2], o[3], s.up)};
            const Frag<2> by[2] = {split<2>(y[0], y[1], s.up), split<2>(y[2], y[3], s.up)};
            const float decay = f[64 * DeltaRecord::kDecay];
#pragma unroll
            for (int i = 0; i < L::kTiles; ++i) {
                f32x4 a{};
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    a = multiply<true>(column_fragment<T, kK>(at + L::kAtQt, i, j, lane), bo[j], a);
                    a = multiply<true>(column_fragment<T, kK>(at + L::kAtK, i, j, lane), by[j], a);
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) D[i][r] = __builtin_fmaf(a[r], s.down, decay * D[i][r]);
            }
        }
        if (c > 0) {
            if (L::kBuffers == 1) __syncthreads();
            store_next(lds + (L::kBuffers == 2 ? ((c - 1) & 1) * L::kBytes : 0));
        }
    }
    if (p.dinitial && in)
#pragma unroll
        for (int i = 0; i < L::kTiles; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = 16 * i + 4 * g + r;
                if (row < p.k_size) p.dinitial[state + (int64_t)row * p.v_size] = D[i][r];
            }
}

template <class T, int kK, int kWaves>
hipError_t launch(const DeltaChunks& a, hipStream_t stream) {
    using L = Layout<T, kK>;
    constexpr int kBytes = L::kBuffers * L::kBytes;
    const int64_t slices = (a.v_size + 16 * kWaves - 1) / (16 * kWaves);
    const void* kernel = reinterpret_cast<const void*>(delta_back_kernel<T, kK, kWaves>);
    if (hipError_t e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, kBytes))
        return e;
    hipLaunchKernelGGL((delta_back_kernel<T, kK, kWaves>),
                       dim3((unsigned)(slices * a.v_heads * a.batch)), dim3(64 * kWaves), kBytes,
                       stream, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_delta_chain_back(const DeltaChunks& a, hipStream_t stream) {
    return by_dtype(a.dtype, [&](auto t) {
        using T = decltype(t);
        return a.k_size <= 64 ? launch<T, 64, 4>(a, stream) : launch<T, 128, 4>(a, stream);
    });
}

}  // namespace sgemm_emu
