// The gated delta rule, first kernel: for every chunk of 64 tokens of every
// value head, the two triangular matrices of the chunk form,
//   T = (I + A)^-1,  A_ts = beta_t e^{G_t - G_s} k_t.k_s (s < t),
//   P_ts = scale e^{G_t - G_s} q_t.k_s (s <= t),
// as operand fragments, and the row factors of the walk over the chunks.
//
// G is summed in FP64: decays of e^-200 and less (a reset) would leave FP32
// sums too coarse for the differences after them.  The inverse starts from
// the four 16 x 16 diagonal blocks (forward substitution, a column to a
// lane) and joins them with FP32 matrix products, two sizes up:
//   [A 0; C D]^-1 = [A^-1 0; -D^-1 C A^-1, D^-1].
// The walk forward takes T diag(beta), the one back T^T.
//
// A block makes one chunk of one head, a wave 16 rows of it.  Bound by the records that it
// writes (27 KB a chunk, or 39 for the gradient) and, in part, by the latency of the
// triangular inverse: 4 x 4096 tokens of 16 heads of 128 in bfloat16 take 60 us,
// 4.1 TB/s of K, Q and records.
#include "delta_chunk.hpp"

namespace sgemm_emu {

namespace {

constexpr int kThreads = 256;
constexpr int kPitch = 68;  // floats of a row of the matrices in LDS

// Row r of a 16 x 16 block of X (in LDS) as the A operand of the four
// FP32 products of a 16 x 16 x 16 one: step i contracts columns 4 g + i.
__device__ inline f32x4 block_rows(const float* X, int lane) {
    return *reinterpret_cast<const f32x4*>(X + (lane & 15) * kPitch + 4 * (lane >> 4));
}
__device__ inline f32x4 block_columns(const float* X, int lane) {
    f32x4 b;
#pragma unroll
    for (int i = 0; i < 4; ++i) b[i] = X[(4 * (lane >> 4) + i) * kPitch + (lane & 15)];
    return b;
}
__device__ inline f32x4 block_product(f32x4 a, f32x4 b, f32x4 c) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
    return c;
}
__device__ inline void block_store(float* X, int lane, f32x4 d) {
#pragma unroll
    for (int i = 0; i < 4; ++i) X[(4 * (lane >> 4) + i) * kPitch + (lane & 15)] = d[i];
}

// Fragments of tile `tile`'s rows of the matrix M (or its transpose), with the
// rows' inverse scales; its columns times `columns`, if given.  Blocks on the
// empty side of the diagonal are zero whatever M holds there.
template <bool kTransposed>
__device__ inline void write_fragments(const float* M, int tile, int lane, char* to, float* inverse,
                                       const float* columns = nullptr) {
    const int row = lane & 15, g = lane >> 4;
    float x[2][8], m = 0.0f;
#pragma unroll
    for (int step = 0; step < 2; ++step)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int other = 2 * step + half;
            const bool full = kTransposed ? other >= tile : other <= tile;
            const int a = 16 * tile + row, b = 16 * other + 4 * g;
            f32x4 v{};
            if (full) {
                if (kTransposed)
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[i] = M[(b + i) * kPitch + a];
                else
                    v = *reinterpret_cast<const f32x4*>(M + a * kPitch + b);
                if (columns) v *= *reinterpret_cast<const f32x4*>(columns + b);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[step][4 * half + i] = v[i];
                m = fmaxf(m, fabsf(v[i]));
            }
        }
    const Scale s = scale_of(max_groups(m));
    if (g == 0) inverse[16 * tile + row] = s.down;
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

template <class T, int kK, bool kBackward, bool kWide>
__global__ __launch_bounds__(kThreads, sizeof(T) == 4 ? 2 : 4) void delta_prep_kernel(DeltaChunks p) {
    constexpr int kSteps = kK / 32;
    // A and P; before them, in the same place, k's rows as operands
    __shared__ __attribute__((aligned(16))) float lds[2 * kC * kPitch];
    float *A = lds, *P = lds + kC * kPitch;
    static_assert(sizeof(Operand<T>) * 64 * 4 * kSteps <= sizeof(lds), "k's rows");
    __shared__ double G[kC];
    __shared__ __attribute__((aligned(16))) float beta[kC], key_down[kC];

    const int h = blockIdx.x % p.v_heads, c = blockIdx.x / p.v_heads;
    const Place at = place_of(p.cu_seqlens, c, p.batch, p.tokens);
    if (at.count <= 0) return;  // the whole block
    const bool packed = p.cu_seqlens != nullptr;
    const int kh = h / (p.v_heads / p.k_heads);
    char* record = p.records + ((int64_t)c * p.v_heads + h) * p.record_bytes;
    float* factors = reinterpret_cast<float*>(record);
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row = lane & 15, g = lane >> 4;

    // This wave's 16 rows of k and q, in operand order, on their way (after the
    // decays, which are waited for first).
    double sum = 0.0;
    float strength = lane < at.count ? 1.0f : 0.0f;
    if (wave == 0 && lane < at.count) {
        const int t = at.first + lane;
        if (p.g.p)
            sum = log_decay(row_of<const float>(p.g, packed, at.n, at.span, h)[t * p.g.token]);
        if (p.beta.p)
            strength = row_of<const float>(p.beta, packed, at.n, at.span, h)[t * p.beta.token];
    }
    const T* k = row_of<const T>(p.k, packed, at.n, at.span, kh) + (int64_t)at.first * p.k.token;
    const T* q = row_of<const T>(p.q, packed, at.n, at.span, kh) + (int64_t)at.first * p.q.token;
    const auto load_tile = [&](const T* from, int64_t stride, int tile, Eight<T>(&x)[kSteps])
                               __attribute__((always_inline)) {
        const int t = 16 * tile + row;
        const __amdgpu_buffer_rsrc_t r = buffer_at(from);
#pragma unroll
        for (int j = 0; j < kSteps; ++j)
            x[j] = load_eight<T>(r, t * (uint32_t)stride * (uint32_t)sizeof(T), 32 * j + 8 * g, p.k_size,
                                 t < at.count, kWide);
    };
    const auto take_tile = [&](const Eight<T>(&x)[kSteps], Operand<T>(&f)[kSteps])
                               __attribute__((always_inline)) {
        float m = 0.0f;
#pragma unroll
        for (int j = 0; j < kSteps; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) m = fmaxf(m, fabsf(to_f32(x[j].x[i])));
        const Scale s = scale_of(max_groups(m));
#pragma unroll
        for (int j = 0; j < kSteps; ++j) f[j].set(x[j], s.up);
        return s;
    };
    Eight<T> kx[kSteps], qx[kSteps];
    load_tile(k, p.k.token, wave, kx);
    load_tile(q, p.q.token, wave, qx);

    if (wave == 0) {  // running sums of the decays, and the strengths
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const double u = __shfl_up(sum, d, 64);
            if (lane >= d) sum += u;
        }
        G[lane] = sum;
        if (kBackward) reinterpret_cast<double*>(record + DeltaRecord::kAtSums)[lane] = sum;
        beta[lane] = strength;
    }
    Operand<T> kw[kSteps], qf[kSteps];
    Scale mine = take_tile(kx, kw), qs = take_tile(qx, qf);
    Operand<T>* rows = reinterpret_cast<Operand<T>*>(lds);
#pragma unroll
    for (int j = 0; j < kSteps; ++j) rows[(wave * kSteps + j) * 64 + lane] = kw[j];
    if (g == 0) key_down[16 * wave + row] = mine.down;
    __syncthreads();

    // this wave's rows of A and P
    f32x4 d{};
    double Gt[4];
    float bt[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        Gt[r] = G[16 * wave + 4 * g + r];
        bt[r] = beta[16 * wave + 4 * g + r];
        // scales of the rows this lane holds of a result
        d[r] = __shfl(mine.down, 4 * g + r, 64);
    }
    f32x4 dq;
#pragma unroll
    for (int r = 0; r < 4; ++r) dq[r] = __shfl(qs.down, 4 * g + r, 64);
    f32x4 kk[4] = {}, qk[4] = {};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (i > wave) continue;
#pragma unroll
        for (int j = 0; j < kSteps; ++j) {
            const Operand<T> kf = rows[(i * kSteps + j) * 64 + lane];
            kk[i] = product(kw[j], kf, kk[i]);
            qk[i] = product(qf[j], kf, qk[i]);
        }
    }
    __syncthreads();  // k's rows are used
    int bad = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (i > wave) continue;
        const float down = key_down[16 * i + row];
        const int s = 16 * i + row;
        const double Gs = G[s];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int t = 16 * wave + 4 * g + r;
            const float e = s <= t ? expf((float)(Gt[r] - Gs)) : 0.0f;
            float a = kk[i][r], b = qk[i][r];
            if (sizeof(T) == 4) {  // FP32 rows were scaled
                a = a * d[r] * down;
                b = b * dq[r] * down;
            }
            a *= bt[r] * e;
            // a value that is not finite must not reach rows before it
            const bool spoilt = s < t && !finite(a);
            bad |= spoilt ? 1 << r : 0;
            A[t * kPitch + s] = s < t && !spoilt ? a : 0.0f;
            P[t * kPitch + s] = s <= t ? p.scale * e * b : 0.0f;
        }
    }
    if (bad != 0)
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (bad >> r & 1) beta[16 * wave + 4 * g + r] = __builtin_nanf("");
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
    // row factors
    if (g == 0) {
        const int t = 16 * wave + row;
        const double last = G[kC - 1];
        if (__is_same(T, f16_t)) mine = qs = Scale{1.0f, 1.0f};  // taken as they are
        factors[64 * DeltaRecord::kKeyScale + t] = mine.up;
        factors[64 * DeltaRecord::kQueryScale + t] = qs.up;
        // (where beta is not finite, what a walk makes of the row is not either)
        const bool in = finite(beta[t]);
        factors[64 * DeltaRecord::kRise + t] =
            in ? expf((float)G[t]) * mine.down : __builtin_nanf("");
        factors[64 * DeltaRecord::kBeta + t] = beta[t];
        if (!in) beta[t] = 0.0f;
        factors[64 * DeltaRecord::kTail + t] = expf((float)(last - G[t])) * mine.down;
        factors[64 * DeltaRecord::kQueryRise + t] = p.scale * expf((float)G[t]) * qs.down;
        factors[64 * DeltaRecord::kDecay + t] = expf((float)last);
    }

    // the diagonal block, whose rows and columns are all this wave's: column
    // `row` of its inverse, in every group of lanes
    float* D = A + 16 * wave * (kPitch + 1);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
    float x[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        float v = i == row ? 1.0f : 0.0f;
#pragma unroll
        for (int j = 0; j < i; ++j) v = __builtin_fmaf(-D[i * kPitch + j], x[j], v);
        x[i] = v;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
    if (g == 0)
#pragma unroll
        for (int i = 0; i < 16; ++i) D[i * kPitch + row] = x[i];
    __syncthreads();
    const auto block = [&](int i, int j) __attribute__((always_inline)) {
        return A + 16 * (i * kPitch + j);
    };
    // 32 x 32: blocks (1, 0) and (3, 2), read and written by one wave each
    if (wave & 1) {
        f32x4 y = block_product(block_rows(block(wave, wave - 1), lane),
                                block_columns(block(wave - 1, wave - 1), lane), f32x4{});
        y = block_product(-block_rows(block(wave, wave), lane), y, f32x4{});
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
        block_store(block(wave, wave - 1), lane, y);
    }
    __syncthreads();
    {  // 64 x 64: wave (i, j) makes block (2 + i, j)
        const int i = 2 + (wave >> 1), j = wave & 1;
        f32x4 y[2], z{};
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            y[r] = f32x4{};
            if (2 + r > i) continue;
            if (j == 0)
                y[r] = block_product(block_rows(block(2 + r, 0), lane),
                                     block_columns(block(0, 0), lane), y[r]);
            y[r] = block_product(block_rows(block(2 + r, 1), lane),
                                 block_columns(block(1, j), lane), y[r]);
            z = block_product(-block_rows(block(i, 2 + r), lane), y[r], z);
        }
        __syncthreads();
        block_store(block(i, j), lane, z);
    }
    __syncthreads();

    write_fragments<false>(A, wave, lane, record + DeltaRecord::kAtT,
                              factors + 64 * DeltaRecord::kT, beta);
    if (kBackward) {
        write_fragments<true>(A, wave, lane, record + DeltaRecord::kAtTt,
                                 factors + 64 * DeltaRecord::kTt);
        write_fragments<true>(P, wave, lane, record + DeltaRecord::kAtPt,
                                 factors + 64 * DeltaRecord::kPt);
    } else {
        write_fragments<false>(P, wave, lane, record + DeltaRecord::kAtP,
                               factors + 64 * DeltaRecord::kP);
    }
}

template <class T, int kK, bool kWide>
void launch_rows(const DeltaChunks& a, hipStream_t stream) {
    const dim3 grid((unsigned)(a.chunks * a.v_heads));
    if (a.backward)
        hipLaunchKernelGGL((delta_prep_kernel<T, kK, true, kWide>), grid, dim3(kThreads), 0,
                           stream, a);
    else
        hipLaunchKernelGGL((delta_prep_kernel<T, kK, false, kWide>), grid, dim3(kThreads), 0,
                           stream, a);
}

template <class T, int kK>
void launch(const DeltaChunks& a, hipStream_t stream) {
    if (a.wide)
        launch_rows<T, kK, true>(a, stream);
    else
        launch_rows<T, kK, false>(a, stream);
}

}  // namespace

hipError_t launch_delta_prep(const DeltaChunks& a, hipStream_t stream) {
    if (a.chunks == 0) return hipSuccess;
    return by_dtype(a.dtype, [&](auto t) {
        using T = decltype(t);
        if (a.k_size <= 64)
            launch<T, 64>(a, stream);
        else
            launch<T, 128>(a, stream);
        return hipGetLastError();
    });
}

}  // namespace sgemm_emu
