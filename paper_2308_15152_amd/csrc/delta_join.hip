// The gated delta rule, sequences cut into parts: the state before every part
// from the one before the first (and, back, the gradient after every part from
// the one after the last),
//   S_{p+1} = M_p S_p + N_p,      D_{p-1} = M_p^T D_p + N'_p.
// A block takes 32 columns of one head of one sequence, a wave 16 of them, which
// stay in its registers from part to part.  M is split once per block into
// fragments in LDS; the next part's M and N are loaded meanwhile.  Bound by that
// loop's latency: a part's M is 64 KiB, and the parts follow one another: 6.3 us a part
// for 8 heads.  (With 128 columns to a block, a fourth of the CUs, a part takes 15 us.)
#include "delta_chunk.hpp"

namespace sgemm_emu {

namespace {

constexpr int kWaves = 2;

template <int kK, bool kBack>
__global__ __launch_bounds__(64 * kWaves, 1) void delta_join_kernel(DeltaChunks p) {
    constexpr int kSteps = kK / 32, kTiles = kK / 16;
    __shared__ __attribute__((aligned(16))) char fragments[2 * kTiles * kSteps * 1024];
    __shared__ __attribute__((aligned(16))) float down[kK];

    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row = lane & 15, g = lane >> 4;
    const int slices = (p.v_size + 16 * kWaves - 1) / (16 * kWaves);
    const int slice = blockIdx.x % slices;
    const int h = (blockIdx.x / slices) % p.v_heads, n = blockIdx.x / slices / p.v_heads;
    const Span span = span_of(p.cu_seqlens, n, p.tokens);
    const int chunks = (span.count + kC - 1) / kC;
    const int parts = max((chunks + p.part_chunks - 1) / p.part_chunks, 1);
    const int first = p.cu_seqlens ? part_base(p, n) : n * parts;
    const int rows = (p.k_size + 15) / 16 * 16;
    const int col = (slice * kWaves + wave) * 16 + row;
    const bool in = col < p.v_size;
    const auto part_at = [&](int j) __attribute__((always_inline)) {
        return ((int64_t)(first + j) * p.v_heads + h);
    };
    const auto of = [&](int step) __attribute__((always_inline)) {  // part of a step
        return kBack ? parts - 1 - step : step;
    };

    // this wave's rows of M, in operand order: kOwn tiles of 16 rows
    constexpr int kOwn = kTiles / kWaves;
    f32x4 x[kOwn][kSteps][2];
    const auto load = [&](int j) __attribute__((always_inline)) {
        const __amdgpu_buffer_rsrc_t M = buffer_at(p.part_steps + part_at(j) * rows * rows);
#pragma unroll
        for (int t = 0; t < kOwn; ++t)
#pragma unroll
            for (int s = 0; s < kSteps; ++s)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const int tile = kOwn * wave + t, other = 2 * s + half;
                    x[t][s][half] = f32x4{};
                    if (16 * tile >= rows || 16 * other >= rows) continue;  // (of all lanes)
                    const int a = 16 * tile + row, b = 16 * other + 4 * g;
                    if (kBack)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            x[t][s][half][i] = load_word<float>(M, 4u * ((b + i) * rows + a));
                    else
                        x[t][s][half] = __builtin_bit_cast(
                            f32x4, __builtin_amdgcn_raw_buffer_load_b128(M, 4u * (a * rows + b), 0, 0));
                }
    };
    // Byte of row 16 i + 4 g + r in this lane's column of a state
    const auto place = [&](int i, int r) __attribute__((always_inline)) -> uint32_t {
        const int e = 16 * i + 4 * g + r;
        return in && (16 * i + 16 <= p.k_size || e < p.k_size) ? 4u * (e * p.v_size + col) : kPastEnd;
    };
    const auto load_state = [&](const float* from, f32x4(&to)[kTiles])
        __attribute__((always_inline)) {
        const __amdgpu_buffer_rsrc_t r = buffer_at(from);
#pragma unroll
        for (int i = 0; i < kTiles; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) to[i][e] = load_word<float>(r, place(i, e));
    };
    f32x4 S[kTiles];
    const float* start = kBack ? p.dfinal : p.initial;
    const int64_t state = (int64_t)p.k_size * p.v_size;
    if (start)
        load_state(start + ((int64_t)n * p.v_heads + h) * state, S);
    else
#pragma unroll
        for (int i = 0; i < kTiles; ++i) S[i] = f32x4{};
    float* states = kBack ? p.part_dstates : p.part_states;
    f32x4 next[kTiles];  // N of the step
    const auto load_n = [&](int j) __attribute__((always_inline)) {
        load_state(states + part_at(j) * state, next);
    };
    if (parts > 1) {
        load(of(0));
        load_n(of(0));
    }
    for (int step = 0; step < parts; ++step) {
        const bool last = step + 1 == parts;
        if (!last) {
            lds_barrier();  // the last part's fragments are used
#pragma unroll
            for (int t = 0; t < kOwn; ++t) {
                const int tile = kOwn * wave + t;
                float m = 0.0f;
#pragma unroll
                for (int s = 0; s < kSteps; ++s) m = fmaxf(m, largest(x[t][s]));
                const Scale up = scale_of(max_groups(m));
                if (g == 0) down[16 * tile + row] = up.down;
#pragma unroll
                for (int s = 0; s < kSteps; ++s) {
                    const Frag<2> f = split<2>(x[t][s][0], x[t][s][1], up.up);
#pragma unroll
                    for (int q = 0; q < 2; ++q)
                        *reinterpret_cast<half8_t*>(
                            fragments + ((q * kTiles + tile) * kSteps + s) * 1024 + lane * 16) =
                            f.part[q];
                }
            }
            if (step + 2 < parts) load(of(step + 1));
        }
        {  // N has been read
            const __amdgpu_buffer_rsrc_t to = buffer_at(states + part_at(of(step)) * state);
#pragma unroll
            for (int i = 0; i < kTiles; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) store_word((float)S[i][r], to, place(i, r));
        }
        if (last) break;
        lds_barrier();
        const Scale ss = scale_of(max_groups(largest(S)));
        Frag<2> b[kSteps];
#pragma unroll
        for (int s = 0; s < kSteps; ++s) b[s] = split<2>(S[2 * s], S[2 * s + 1], ss.up);
#pragma unroll
        for (int i = 0; i < kTiles; ++i) {
            f32x4 a{};
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                Frag<2> f;
#pragma unroll
                for (int q = 0; q < 2; ++q)
                    f.part[q] = *reinterpret_cast<const half8_t*>(
                        fragments + ((q * kTiles + i) * kSteps + s) * 1024 + lane * 16);
                a = multiply<true>(f, b[s], a);
            }
            S[i] = next[i] + a * reinterpret_cast<const f32x4*>(down)[4 * i + g] * ss.down;
        }
        if (step + 2 < parts) load_n(of(step + 1));
    }
}

template <int kK, bool kBack>
hipError_t launch(const DeltaChunks& a, hipStream_t stream) {
    const int64_t slices = (a.v_size + 16 * kWaves - 1) / (16 * kWaves);
    hipLaunchKernelGGL((delta_join_kernel<kK, kBack>), dim3((unsigned)(slices * a.v_heads * a.batch)),
                       dim3(64 * kWaves), 0, stream, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_delta_join(const DeltaChunks& a, bool back, hipStream_t stream) {
    if (a.k_size <= 64) return back ? launch<64, true>(a, stream) : launch<64, false>(a, stream);
    return back ? launch<128, true>(a, stream) : launch<128, false>(a, stream);
}

}  // namespace sgemm_emu
