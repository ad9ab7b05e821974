// The gated delta rule, sequences cut into parts: the state before every part
// from the one before the first (and, back, the gradient after every part from
// the one after the last),
//   S_{p+1} = M_p S_p + N_p,      D_{p-1} = M_p^T D_p + N'_p.
// A block takes 16 columns of one head of one sequence, and a wave 32 rows of them,
// which stay in its registers from part to part.  A wave's rows of M are loaded a part
// ahead and split in registers; of S the waves exchange split fragments through LDS, one
// barrier a part.  Bound by the latency of that loop: the parts follow one another.  8
// parts of 8 heads of 128 x 128 take 25 us; with M shared through LDS and all rows of 16
// columns to a wave they took 50.
#include "delta_chunk.hpp"

namespace sgemm_emu {

namespace {

template <int kK, bool kBack>
__global__ __launch_bounds__(2 * kK, 1) void delta_join_kernel(DeltaChunks p) {
    constexpr int kSteps = kK / 32;  // of a contraction, and waves
    __shared__ __attribute__((aligned(16))) char fragments[2][kSteps][2 * 1024];
    __shared__ float scales[2][kSteps][16];
    __shared__ __attribute__((aligned(16))) float down[kK];

    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row = lane & 15, g = lane >> 4;
    const int slices = (p.v_size + 15) / 16;
    const int slice = blockIdx.x % slices;
    const int h = (blockIdx.x / slices) % p.v_heads, n = blockIdx.x / slices / p.v_heads;
    const Span span = span_of(p.cu_seqlens, n, p.tokens);
    const int chunks = (span.count + kC - 1) / kC;
    const int parts = max((chunks + p.part_chunks - 1) / p.part_chunks, 1);
    const int first = p.cu_seqlens ? part_base(p, n) : n * parts;
    const int rows = (p.k_size + 15) / 16 * 16;
    const int col = slice * 16 + row;
    const bool in = col < p.v_size;
    const auto part_at = [&](int j) __attribute__((always_inline)) {
        return ((int64_t)(first + j) * p.v_heads + h);
    };
    const auto of = [&](int step) __attribute__((always_inline)) {  // part of a step
        return kBack ? parts - 1 - step : step;
    };

    // this wave's two tiles of rows of M, in operand order
    f32x4 x[2][kSteps][2];
    const auto load = [&](int j) __attribute__((always_inline)) {
        const __amdgpu_buffer_rsrc_t M = buffer_at(p.part_steps + part_at(j) * rows * rows);
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int s = 0; s < kSteps; ++s)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const int a = 32 * wave + 16 * t + row, b = 32 * s + 16 * half + 4 * g;
                    const bool there = 32 * wave + 16 * t < rows && 32 * s + 16 * half < rows;
                    if (kBack)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            x[t][s][half][i] =
                                load_word<float>(M, there ? 4u * ((b + i) * rows + a) : kPastEnd);
                    else
                        x[t][s][half] = __builtin_bit_cast(
                            f32x4, __builtin_amdgcn_raw_buffer_load_b128(
                                       M, there ? 4u * (a * rows + b) : kPastEnd, 0, 0));
                }
    };
    // Byte of row 32 wave + 16 i + 4 g + r in this lane's column of a state
    const auto place = [&](int i, int r) __attribute__((always_inline)) -> uint32_t {
        const int e = 32 * wave + 16 * i + 4 * g + r;
        return in && e < p.k_size ? 4u * (e * p.v_size + col) : kPastEnd;
    };
    const auto load_state = [&](const float* from, f32x4(&to)[2]) __attribute__((always_inline)) {
        const __amdgpu_buffer_rsrc_t r = buffer_at(from);
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) to[i][e] = load_word<float>(r, place(i, e));
    };
    f32x4 S[2] = {};
    const float* start = kBack ? p.dfinal : p.initial;
    const int64_t state = (int64_t)p.k_size * p.v_size;
    if (start) load_state(start + ((int64_t)n * p.v_heads + h) * state, S);
    float* states = kBack ? p.part_dstates : p.part_states;
    f32x4 next[2];  // N of the step
    const auto load_n = [&](int j) __attribute__((always_inline)) {
        load_state(states + part_at(j) * state, next);
    };
    const auto store_state = [&](int step) __attribute__((always_inline)) {
        const __amdgpu_buffer_rsrc_t to = buffer_at(states + part_at(of(step)) * state);
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) store_word((float)S[i][r], to, place(i, r));
    };
    if (parts > 1) {
        load(of(0));
        load_n(of(0));
    }
    // (Loads without conditions, as in delta_chain.hip: the last part's are made twice.)
    for (int step = 0; step + 1 < parts; ++step) {
        const int ahead = min(step + 1, parts - 2);
        // S to the others
        const Scale ss = scale_of(max_groups(largest(S)));
        const Frag<2> own = split<2>(S[0], S[1], ss.up);
        char* to = fragments[step & 1][wave] + lane * 16;
        *reinterpret_cast<half8_t*>(to) = own.part[0];
        *reinterpret_cast<half8_t*>(to + 1024) = own.part[1];
        scales[step & 1][wave][row] = ss.down;
        // M
        Frag<2> m[2][kSteps];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            float top = 0.0f;
#pragma unroll
            for (int s = 0; s < kSteps; ++s) top = fmaxf(top, largest(x[t][s]));
            const Scale up = scale_of(max_groups(top));
            if (g == 0) down[32 * wave + 16 * t + row] = up.down;
#pragma unroll
            for (int s = 0; s < kSteps; ++s) m[t][s] = split<2>(x[t][s][0], x[t][s][1], up.up);
        }
        f32x4 N[2] = {next[0], next[1]};
        store_state(step);  // N has been read
        load(of(ahead));
        load_n(of(ahead));
        lds_barrier();
        f32x4 sum[2] = {};
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            Frag<2> b;
#pragma unroll
            for (int q = 0; q < 2; ++q)
                b.part[q] = *reinterpret_cast<const half8_t*>(fragments[step & 1][s] + q * 1024 +
                                                              lane * 16);
            const float scale = scales[step & 1][s][row];
#pragma unroll
            for (int t = 0; t < 2; ++t)
                sum[t] += multiply<true>(m[t][s], b, f32x4{}) * scale;
        }
#pragma unroll
        for (int t = 0; t < 2; ++t)
            S[t] = N[t] + sum[t] * *reinterpret_cast<const f32x4*>(down + 32 * wave + 16 * t + 4 * g);
    }
    store_state(parts - 1);
}

template <int kK, bool kBack>
hipError_t launch(const DeltaChunks& a, hipStream_t stream) {
    const int64_t slices = (a.v_size + 15) / 16;
    hipLaunchKernelGGL((delta_join_kernel<kK, kBack>),
                       dim3((unsigned)(slices * a.v_heads * a.batch)), dim3(2 * kK), 0, stream, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_delta_join(const DeltaChunks& a, bool back, hipStream_t stream) {
    if (a.k_size <= 64) return back ? launch<64, true>(a, stream) : launch<64, false>(a, stream);
    return back ? launch<128, true>(a, stream) : launch<128, false>(a, stream);
}

}  // namespace sgemm_emu
