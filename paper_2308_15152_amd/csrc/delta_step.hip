// The gated delta rule token by token (its recurrent form):
//   S <- e^g S + k u^T,  u = beta (v - e^g S^T k),  o = scale S^T q.
//
// The columns of S are independent, so a block owns kCols columns of one
// head's state and holds them in registers across the tokens: thread (x, y) has
// kVec columns from kVec x and the rows y, y + kRows, ... .  With S before the
// token, S^T k and S^T q are both sums over the rows, taken together: o = scale (e^g
// S^T q + u (k.q)), so a token costs one reduction over the block.
//
// Bound by memory at large batches: the state is read and written once for
// all tokens of the call (8 bytes an element); q, k and v are small.  At small
// batches the launch and the state's latency bound it, and narrow column
// slices spread a head over more CUs.  Measured (128 x 128 states): 256 sequences of 32
// heads 219 us, 4.9 TB/s; one sequence of 16 heads 4.7 us, a further token 0.9.
#include "mixing.hpp"

namespace sgemm_emu {

namespace {

constexpr int kThreads = 256;
constexpr int kMaxK = 128;

// Sum over the lanes of a wave that agree in l % kX, in every one of them.
template <int kX>
__device__ inline float sum_rows(float x) {
    if (kX <= 8)
        x += __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), 0x128,
                                                                0xf, 0xf, true));  // 8 lanes on
    if (kX <= 16) {
        const uint32_t u = __builtin_bit_cast(uint32_t, x);
        const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
        const uint32_t a0 = a[0], a1 = a[1];
        x = __builtin_bit_cast(float, a0) + __builtin_bit_cast(float, a1);
    }
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    const uint32_t a0 = a[0], a1 = a[1];
    return __builtin_bit_cast(float, a0) + __builtin_bit_cast(float, a1);
}

// kVec columns a thread, kX threads along the columns.
template <class T, int kVec, int kX>
__global__ __launch_bounds__(kThreads) void delta_step_kernel(DeltaStep p,
                                                              int64_t first) {
    constexpr int kCols = kVec * kX;
    constexpr int kRows = kThreads / kX;       // threads along the rows
    constexpr int kEach = kMaxK / kRows;       // rows of a thread
    constexpr int kWaves = kThreads / 64;
    typedef typename Pack<float, kVec>::type Vec;
    static_assert(kX >= 8 && kX <= 32, "lanes of a row");
    __shared__ __attribute__((aligned(16))) float sums[2][kWaves][2 * kCols + 4];
    __shared__ float keys[2][2][kMaxK];

    const int x = threadIdx.x % kX, y = threadIdx.x / kX;
    const int wave = threadIdx.x >> 6;
    const int slices = (p.v_size + kCols - 1) / kCols;
    int64_t task = first + blockIdx.x;
    const int slice = (int)(task % slices);
    task /= slices;
    const int h = (int)(task % p.v_heads), n = (int)(task / p.v_heads);
    const int kh = h / (p.v_heads / p.k_heads);
    const Span s = span_of(nullptr, n, p.tokens);
    const int col = slice * kCols + kVec * x;
    const bool in = col < p.v_size;  // kVec divides v_size or is 1

    const T* q = row_of<const T>(p.q, false, n, s, kh);
    const T* k = row_of<const T>(p.k, false, n, s, kh);
    const T* v = row_of<const T>(p.v, false, n, s, h);
    T* o = row_of<T>(p.o, false, n, s, h);
    const int slot = p.slots ? p.slots[n] : n;
    if (slot < 0 || slot >= p.n_slots) {  // the whole block
        if (in && y == 0)
            for (int t = 0; t < p.tokens; ++t)
                for (int i = 0; i < kVec; ++i) o[t * p.o.token + col + i] = from_f32<T>(0.0f);
        return;
    }
    const int64_t at = slot * p.state_stride + (int64_t)h * p.k_size * p.v_size + col;
    float S[kEach][kVec];
#pragma unroll
    for (int r = 0; r < kEach; ++r) {
        const int row = y + kRows * r;
        Vec w{};
        if (in && row < p.k_size && p.from)
            w = *reinterpret_cast<const Vec*>(p.from + at + (int64_t)row * p.v_size);
        __builtin_memcpy(S[r], &w, sizeof(Vec));
    }
    const float* g = p.g.p ? row_of<const float>(p.g, false, n, s, h) : nullptr;
    const float* beta = p.beta.p ? row_of<const float>(p.beta, false, n, s, h) : nullptr;

    // the next token's values, on their way while one is computed
    const int e = threadIdx.x % kMaxK;
    const bool is_key = threadIdx.x < kMaxK, has_key = e < p.k_size;
    const T* key_row = is_key ? k + e : q + e;
    const int64_t key_step = is_key ? p.k.token : p.q.token;
    T key{}, value[kVec]{};
    float gate = 0.0f, strength = 1.0f;
    const auto load_token = [&](int t) __attribute__((always_inline)) {
        if (has_key) key = key_row[t * key_step];
#pragma unroll
        for (int i = 0; i < kVec; ++i)
            if (in) value[i] = v[t * p.v.token + col + i];
        if (g) gate = g[t * p.g.token];
        if (beta) strength = beta[t * p.beta.token];
    };
    if (p.tokens > 0) load_token(0);
    for (int t = 0; t < p.tokens; ++t) {
        const int buf = t & 1;
        keys[buf][threadIdx.x / kMaxK][e] = has_key ? to_f32(key) : 0.0f;
        float vt[kVec];
#pragma unroll
        for (int i = 0; i < kVec; ++i) vt[i] = in ? to_f32(value[i]) : 0.0f;
        const float decay = g ? expf(log_decay(gate)) : 1.0f, b = strength;
        if (t + 1 < p.tokens) load_token(t + 1);
        lds_barrier();
        float kr[kEach], qr[kEach], sk[kVec] = {}, sq[kVec] = {}, kq = 0.0f;
#pragma unroll
        for (int r = 0; r < kEach; ++r) {
            kr[r] = keys[buf][0][y + kRows * r];
            qr[r] = keys[buf][1][y + kRows * r];
            kq = __builtin_fmaf(kr[r], qr[r], kq);
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
                sk[i] = __builtin_fmaf(S[r][i], kr[r], sk[i]);
                sq[i] = __builtin_fmaf(S[r][i], qr[r], sq[i]);
            }
        }
        // over the wave's rows, then over the waves
        kq = sum_rows<kX>(kq);
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            sk[i] = sum_rows<kX>(sk[i]);
            sq[i] = sum_rows<kX>(sq[i]);
        }
        Vec out_k, out_q;
        __builtin_memcpy(&out_k, sk, sizeof(Vec));
        __builtin_memcpy(&out_q, sq, sizeof(Vec));
        if ((threadIdx.x & 63) < kX) {
            float* to = sums[buf][wave];
            *reinterpret_cast<Vec*>(to + kVec * x) = out_k;
            *reinterpret_cast<Vec*>(to + kCols + kVec * x) = out_q;
            if (x == 0) to[2 * kCols] = kq;
        }
        lds_barrier();
        float tk[kVec] = {}, tq[kVec] = {}, tkq = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float* from = sums[buf][w];
            tkq += from[2 * kCols];
            float a[kVec], c[kVec];
            __builtin_memcpy(a, from + kVec * x, sizeof(a));
            __builtin_memcpy(c, from + kCols + kVec * x, sizeof(c));
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
                tk[i] += a[i];
                tq[i] += c[i];
            }
        }
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const float u = b * __builtin_fmaf(-decay, tk[i], vt[i]);
#pragma unroll
            for (int r = 0; r < kEach; ++r) S[r][i] = __builtin_fmaf(kr[r], u, decay * S[r][i]);
            tq[i] = p.scale * __builtin_fmaf(u, tkq, decay * tq[i]);
        }
        if (in && y == 0)
#pragma unroll
            for (int i = 0; i < kVec; ++i) o[t * p.o.token + col + i] = from_f32<T>(tq[i]);
    }
    if (p.to && in)
#pragma unroll
        for (int r = 0; r < kEach; ++r) {
            const int row = y + kRows * r;
            if (row < p.k_size) {
                Vec w;
                __builtin_memcpy(&w, S[r], sizeof(Vec));
                *reinterpret_cast<Vec*>(p.to + at + (int64_t)row * p.v_size) = w;
            }
        }
}

template <class T, int kVec, int kX>
hipError_t launch(const DeltaStep& a, hipStream_t stream) {
    const int64_t slices = (a.v_size + kVec * kX - 1) / (kVec * kX);
    const int64_t blocks = slices * a.v_heads * a.batch;
    for (int64_t first = 0; first < blocks; first += kMostBlocks) {
        const int64_t count = blocks - first < kMostBlocks ? blocks - first : kMostBlocks;
        hipLaunchKernelGGL((delta_step_kernel<T, kVec, kX>), dim3((unsigned)count), dim3(kThreads),
                           0, stream, a, first);
        if (hipError_t e = hipGetLastError()) return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_delta_step(const DeltaStep& a, hipStream_t stream) {
    if (a.batch == 0 || a.v_size == 0) return hipSuccess;
    // 16-byte accesses of the state's rows; otherwise one column a thread
    const bool wide = a.v_size % 4 == 0 && a.state_stride % 4 == 0 &&
                      (uintptr_t)a.from % 16 == 0 && (uintptr_t)a.to % 16 == 0;
    return by_dtype(a.dtype, [&](auto t) {
        using T = decltype(t);
        if (!wide) return launch<T, 1, 32>(a, stream);
        return launch<T, 4, 8>(a, stream);
    });
}

}  // namespace sgemm_emu
