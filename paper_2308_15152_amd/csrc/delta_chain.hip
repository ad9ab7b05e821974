// The gated delta rule, second kernel: the walk over a sequence's chunks that
// carries the state,
//   U = T diag(beta) (V - diag(e^G) K S),
//   O = scale diag(e^G) Q S + P U,   S' = e^{G_64} S + K^T diag(e^{G_64 - G}) U.
//
// Columns of S are independent: a pair of waves owns 16 of them, half of the rows
// each in the accumulator layout, and carries them through the whole sequence.  What
// bounds it is the chain of a chunk's products, in which one wave issues an
// instruction every 4 to 6 cycles and nothing else can help, so that only the chain is
// left to the pair: each makes K S of its rows, the first adds the other's and goes on to U,
// and both update their rows of S with the split U that it gives the other.  The
// block's other waves help: four bring K, Q, T, P and V of the next chunk into
// LDS as fragments (loaded into registers a chunk before), and four make O from the S and U
// that the walking waves leave in LDS.
//
// One barrier a chunk (A): behind it the chunk's K, T, V and Q are there, and
// the last chunk's U.  Inside a chunk a walking wave posts when its S is down and
// its V is taken; the helpers wait for that before they read S and write the next V.  In
// FP32, for whose two parts LDS holds Q only once, the post is a second barrier (B),
// before which the chunk's Q goes down.
//
// Measured (bfloat16, 128 x 128): 4 x 4096 tokens of 16 heads 212 us, 3.3 us a
// chunk on all CUs (the four that bring and the pair take about as long); 32768 tokens of 8
// heads, not cut, 2.3 us a chunk.
//
// A long sequence of few heads leaves most CUs idle.  It is cut into parts, and
// walked three times less deep: first every part but the last from S = 0, and, as
// further columns with V = 0, from the columns of the identity, which gives N and M of
// S -> M S + N; then the states before the parts follow one from another
// (delta_join.hip); then all parts are walked for their outputs.
#include "delta_chunk.hpp"

namespace sgemm_emu {

namespace {

constexpr int kOutputs = kDeltaOutputs, kStates = kDeltaStates, kPartSteps = kDeltaParts;

// LDS, in bytes, and the number of helping waves.
// kWalkers: groups of 16 columns, a pair of walking waves each.
template <class T, int kK, int kWalkers, int kMode>
struct Layout {
    static constexpr bool kPosts = sizeof(T) == 2 || kMode != kOutputs;
    // Four bring the operands, four make O.  (Stores of O among a wave's loads
    // would be waited for with them.)
    static constexpr int kHelpers = kMode == kOutputs ? 8 : 4;
    static constexpr int kParts = kPartsOf<T>;  // of K and Q
    static constexpr int kSteps = kK / 32, kTiles = kK / 16;
    static constexpr int kHalf = kTiles / 2;                  // row tiles of a wave of a pair
    static constexpr int kRows = kParts * 4 * kSteps * 1024;  // K or Q
    static constexpr int kMatrices = 2 * DeltaRecord::kMatrix;
    static constexpr int kBytesP = kMode == kOutputs ? kMatrices : 0;
    // two buffers of these
    static constexpr int kAtK = 0;
    static constexpr int kAtT = kAtK + kRows;
    static constexpr int kAtF = kAtT + kMatrices;
    static constexpr int kFactorBytes = 256 * DeltaRecord::kChain;
    static constexpr int kBuffer = kAtF + kFactorBytes;
    // one or two of Q and P
    static constexpr int kAtQ = 2 * kBuffer;
    static constexpr int kAtP = kAtQ + (kMode == kOutputs ? kRows : 0);
    static constexpr int kBufferQ = kAtP + kBytesP - kAtQ;
    // one of these
    static constexpr int kAtV = kAtQ + (kPosts ? 2 : 1) * kBufferQ;
    using V = Values<T, kWalkers, 256>;
    static constexpr int kAtS = kAtV + kWalkers * V::kEach;
    static constexpr int kEachS = 2 * kSteps * 1024 + 128;  // and the scales of its halves
    static constexpr int kAtU = kAtS + (kMode == kOutputs ? kWalkers * kEachS : 0);
    static constexpr int kEachU = kC * 16 * 4 + 128;  // and each column's rows that count, and scale
    static constexpr int kBufferU = kMode == kOutputs ? kWalkers * kEachU : 0;  // one or two
    // what the waves of a pair give each other
    static constexpr int kAtX = kAtU + (kPosts ? 2 : 1) * kBufferU;
    static constexpr int kEachX = 4 * 1024 + 64;
    // chunks done: [wave] S is down, V taken; [2 kWalkers + wave] given to the other
    static constexpr int kAtPosts = kAtX + kWalkers * kEachX;
    static constexpr int kBytes = kAtPosts + 16 * kWalkers;
};

// kWide: all rows can be loaded 16 bytes at a time (8 of V's).  (Decided here, not where
// they are loaded: loads of two kinds into the same registers would be waited for
// as if both were under way.)
template <class T, int kK, int kWalkers, int kMode, bool kWide>
__global__ __launch_bounds__(64 * (2 * kWalkers + Layout<T, kK, kWalkers, kMode>::kHelpers), 1)
void delta_chain_kernel(DeltaChunks p) {
    using L = Layout<T, kK, kWalkers, kMode>;
    constexpr bool kPosts = L::kPosts;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    int* posts = reinterpret_cast<int*>(lds + L::kAtPosts);

    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int g = lane >> 4;
    const int v_slices = (p.v_size + 16 * kWalkers - 1) / (16 * kWalkers);
    const int slices =
        v_slices + (kMode == kPartSteps ? (p.k_size + 16 * kWalkers - 1) / (16 * kWalkers) : 0);
    const WalkTask w = walk_task(slices);
    int slice = w.slice;
    const int h = w.task % p.v_heads, index = w.task / p.v_heads;
    if (index >= (p.part_chunks > 0 ? p.parts : p.batch)) return;  // the whole block
    const int kh = h / (p.v_heads / p.k_heads);
    const bool packed = p.cu_seqlens != nullptr;
    const Walk walk = walk_of(p, index);
    const int chunks = walk.count;
    // (the whole block)
    if (chunks < 0 || (kMode == kPartSteps && !p.backward && walk.part + 1 == walk.parts)) return;
    const int n = walk.n;
    const Span span = {walk.span.first, walk.span.count - walk.first * kC};  // from the part on
    // columns of S, or (kPartSteps, later slices) of M, which has no V
    const bool of_m = kMode == kPartSteps && slice >= v_slices;
    if (of_m) slice -= v_slices;
    const int columns = of_m ? p.k_size : p.v_size;
    const int col0 = slice * kWalkers * 16;
    const int first_chunk = walk.base + walk.first;
    const char* records = p.records + ((int64_t)first_chunk * p.v_heads + h) * p.record_bytes;
    const int64_t record_step = (int64_t)p.v_heads * p.record_bytes;
    const int64_t skip = (int64_t)walk.first * kC;  // tokens of the parts before
    if (threadIdx.x < 4 * kWalkers) posts[threadIdx.x] = 0;

    if (wave < 2 * kWalkers) {
        const int group = wave >> 1, half = wave & 1;
        const bool leads = half == 0;
        const int row0 = half * 16 * L::kHalf;
        const int col = col0 + 16 * group + (lane & 15);
        const bool in = col < columns;
        f32x4 S[L::kHalf];  // rows row0 + 16 i + 4 g + r
        const int64_t sequence = ((int64_t)n * p.v_heads + h) * p.k_size * p.v_size;
        const int64_t part = ((int64_t)index * p.v_heads + h) * p.k_size * p.v_size;
        const float* from = kMode == kPartSteps    ? nullptr
                            : p.part_chunks > 0 ? p.part_states + part
                            : p.initial         ? p.initial + sequence
                                                : nullptr;
#pragma unroll
        for (int i = 0; i < L::kHalf; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = row0 + 16 * i + 4 * g + r;
                S[i][r] = from && in && row < p.k_size ? from[(int64_t)row * p.v_size + col] : 0.0f;
                if (of_m && row == col) S[i][r] = 1.0f;
            }
        const char* v_at = lds + L::kAtV + group * L::V::kEach + 
                           value_slot(lane, group) * 4 * (int)sizeof(T);
        char* s_at = lds + L::kAtS + group * L::kEachS;
        char* u_at = lds + L::kAtU + group * L::kEachU + lane * 16;
        char* x_at = lds + L::kAtX + group * L::kEachX;
        int* given = posts + 2 * kWalkers;

        for (int c = 0; c < chunks; ++c) {
            const char* at = lds + (c & 1) * L::kBuffer;
            const float* f =
                reinterpret_cast<const float*>(at + L::kAtF) - 64 * DeltaRecord::kFirstChain;
            const auto factor = [&](int which, int tile) __attribute__((always_inline)) {
                return reinterpret_cast<const f32x4*>(f + 64 * which)[4 * tile + g];
            };
            lds_barrier();  // A
            f32x4 vt[4];
            if (leads)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    T w[4];
                    __builtin_memcpy(w, v_at + i * 64 * sizeof(w), sizeof(w));
                    vt[i] = f32x4{to_f32(w[0]), to_f32(w[1]), to_f32(w[2]), to_f32(w[3])};
                }
            if (kMode == kStates) {
                const int64_t task = (int64_t)(first_chunk + c) * p.v_heads + h;
                const __amdgpu_buffer_rsrc_t to =
                    buffer_at(p.states + task * ((p.k_size + 15) / 16 * 16) * p.v_size);
                const uint32_t off = in ? 4u * ((row0 + 4 * g) * p.v_size + col) : kPastEnd;
#pragma unroll
                for (int i = 0; i < L::kHalf; ++i)
                    if (row0 + 16 * i < p.k_size)
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            __builtin_amdgcn_raw_buffer_store_b32(
                                __builtin_bit_cast(uint32_t, (float)S[i][r]), to, off,
                                4 * (16 * i + r) * p.v_size, 0);
            }
            const Scale ss = scale_of(max_groups(largest(S)));
            Frag<2> sb[L::kSteps / 2];
#pragma unroll
            for (int j = 0; j < L::kSteps / 2; ++j) {
                sb[j] = split<2>(S[2 * j], S[2 * j + 1], ss.up);
                if (kMode == kOutputs)
#pragma unroll
                    for (int q = 0; q < 2; ++q)
                        *reinterpret_cast<half8_t*>(
                            s_at + (q * L::kSteps + half * (L::kSteps / 2) + j) * 1024 + lane * 16) =
                            sb[j].part[q];
            }
            if (kMode == kOutputs)
                reinterpret_cast<float*>(s_at + 2 * L::kSteps * 1024)[16 * half + (lane & 15)] =
                    ss.down;
            if (kPosts) {
                __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
                __hip_atomic_store(posts + wave, c + 1, __ATOMIC_RELAXED,
                                   __HIP_MEMORY_SCOPE_WORKGROUP);
            } else {
                lds_barrier();  // B
            }
            // V - e^G K S
            f32x4 x[4] = {};
#pragma unroll
            for (int j = 0; j < L::kSteps / 2; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    x[i] = multiply(row_fragment<T, kK>(at + L::kAtK, i, half * (L::kSteps / 2) + j,
                                                        lane), sb[j], x[i]);
            Frag<2> b[2];
            float down;
            if (!leads) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    *reinterpret_cast<f32x4*>(x_at + i * 1024 + lane * 16) = x[i] * ss.down;
                give(given + wave, c + 1);
                wait_given(given + wave - 1, c + 1);
                take(given + wave - 1, c + 1, [&]() __attribute__((always_inline)) {
#pragma unroll
                    for (int j = 0; j < 2; ++j)
#pragma unroll
                        for (int q = 0; q < 2; ++q)
                            b[j].part[q] = *reinterpret_cast<const half8_t*>(
                                x_at + (2 * j + q) * 1024 + lane * 16);
                    down = reinterpret_cast<const float*>(x_at + 4096)[lane & 15];
                });
            } else {
            f32x4 other[4];
            take(given + wave + 1, c + 1, [&]() __attribute__((always_inline)) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    other[i] = *reinterpret_cast<const f32x4*>(x_at + i * 1024 + lane * 16);
            });
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f32x4 rise = factor(DeltaRecord::kRise, i);
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    x[i][r] = __builtin_fmaf(
                        -rise[r], __builtin_fmaf(x[i][r], ss.down, other[i][r]), vt[i][r]);
            }
            // U
            f32x4 u[4] = {};
            int cut = kC;
            float u_down;  // U: u times it
            {
                float top = column_largest(x);
                const bool cuts = __any(!finite(top));
                if (cuts) cut = cut_column(x, top);
                const Scale xs = scale_of(top);
                const Frag<2> xb[2] = {split<2>(x[0], x[1], xs.up), split<2>(x[2], x[3], xs.up)};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
#pragma unroll
                    for (int j = 0; j <= i / 2; ++j)
                        u[i] = multiply(matrix_fragment<2>(at + L::kAtT, lower_at(i, j), lane), xb[j],
                                        u[i]);
                    u[i] *= kMode == kStates ? factor(DeltaRecord::kT, i) * xs.down
                                             : factor(DeltaRecord::kT, i);
                    if (kMode == kStates && cuts)
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (16 * i + 4 * g + r >= cut) u[i][r] = __builtin_nanf("");
                    if (kMode == kOutputs)
                        *reinterpret_cast<f32x4*>(u_at + (kPosts ? (c & 1) * L::kBufferU : 0) +
                                                  i * 1024) = u[i];
                }
                u_down = kMode == kStates ? 1.0f : xs.down;
                if (kMode == kOutputs) {
                    char* to = u_at + (kPosts ? (c & 1) * L::kBufferU : 0) - lane * 16 + kC * 16 * 4;
                    reinterpret_cast<int*>(to)[lane & 15] = cut;
                    reinterpret_cast<float*>(to)[16 + (lane & 15)] = u_down;
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
            b[0] = split<2>(u[0], u[1], us.up);
            b[1] = split<2>(u[2], u[3], us.up);
            down = cut == kC ? us.down * u_down : __builtin_nanf("");
            asm("" : "+v"(down));  // one select, not one for every product with it
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int q = 0; q < 2; ++q)
                    *reinterpret_cast<half8_t*>(x_at + (2 * j + q) * 1024 + lane * 16) = b[j].part[q];
            reinterpret_cast<float*>(x_at + 4096)[lane & 15] = down;
            give(given + wave, c + 1);
            }
            const float decay = f[64 * DeltaRecord::kDecay];
#pragma unroll
            for (int i = 0; i < L::kHalf; ++i) {
                f32x4 a{};
#pragma unroll
                for (int j = 0; j < 2; ++j)  // lo.lo too: updates of like keys cancel
                    a = multiply<true>(
                        column_fragment<T, kK>(at + L::kAtK, half * L::kHalf + i, j, lane), b[j], a);
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    S[i][r] = __builtin_fmaf(a[r], down, decay * S[i][r]);
            }
        }
        if (kMode == kOutputs && chunks > 0) lds_barrier();  // the last U
        const int rows = (p.k_size + 15) / 16 * 16;
        float* to = kMode == kPartSteps
                        ? (of_m ? p.part_steps + ((int64_t)index * p.v_heads + h) * rows * rows
                                : p.part_states + part)
                    : p.final_state && walk.part + 1 == walk.parts ? p.final_state + sequence
                                                                   : nullptr;
        const int stride = of_m ? rows : p.v_size;
        if (to && (in || (of_m && col < rows)))
#pragma unroll
            for (int i = 0; i < L::kHalf; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int row = row0 + 16 * i + 4 * g + r;
                    if (row < (of_m ? rows : p.k_size)) to[(int64_t)row * stride + col] = S[i][r];
                }
        return;
    }

    // ---- the helping waves
    const int helper = wave - 2 * kWalkers;
    const auto buffer_q = [&](int c) __attribute__((always_inline)) {
        return lds + (kPosts ? (c & 1) * L::kBufferQ : 0);
    };
    // until every walking wave, which is in chunk c and posts on its way, has posted
    const auto wait_posts = [&](int c) __attribute__((always_inline)) {
        if (kPosts) {
#pragma unroll
            for (int w = 0; w < 2 * kWalkers; ++w) wait_given(posts + w, c + 1);
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
        } else {
            lds_barrier();  // B
        }
    };

    if (helper < 4) {  // bring the operands
        int id = threadIdx.x - 128 * kWalkers;
        const T* k = row_of<const T>(p.k, packed, n, span, kh) + skip * p.k.token;
        const T* q = row_of<const T>(p.q, packed, n, span, kh) + skip * p.q.token;
        const T* v = row_of<const T>(p.v, packed, n, span, h) + skip * p.v.token + col0;
        Rows<T, kK, 256> ku, qu;
        Copy<L::kMatrices, 256> tcopy;
        Copy<L::kFactorBytes, 256> fcopy;
        Copy<L::kBytesP == 0 ? 16 : L::kBytesP, 256> pcopy;
        typename L::V vu;
        const auto load_k = [&](int c) __attribute__((always_inline)) {
            const int count = min(kC, span.count - c * kC);
            const char* record = records + c * record_step;
            ku.load(k + (int64_t)c * kC * p.k.token, p.k.token, count, p.k_size, kWide,
                    reinterpret_cast<const float*>(record) + 64 * DeltaRecord::kKeyScale, id);
            tcopy.load(record + DeltaRecord::kAtT, id);
            fcopy.load(record + 256 * DeltaRecord::kFirstChain, id);
        };
        const auto load_v = [&](int c) __attribute__((always_inline)) {
            vu.load(v + (int64_t)c * kC * p.v.token, p.v.token, min(kC, span.count - c * kC),
                    of_m ? 0 : p.v_size - col0, kWide, id);
        };
        const auto store_k = [&](int c) __attribute__((always_inline)) {
            char* to = lds + (c & 1) * L::kBuffer;
            ku.store(to + L::kAtK, id);
            tcopy.store(to + L::kAtT, id);
            fcopy.store(to + L::kAtF, id);
        };
        const auto store_v = [&]() __attribute__((always_inline)) { vu.store(lds + L::kAtV, id); };
        const auto load_q = [&](int c) __attribute__((always_inline)) {
            if (kMode != kOutputs) return;
            const char* record = records + c * record_step;
            qu.load(q + (int64_t)c * kC * p.q.token, p.q.token, min(kC, span.count - c * kC),
                    p.k_size, kWide,
                    reinterpret_cast<const float*>(record) + 64 * DeltaRecord::kQueryScale, id);
        };
        const auto load_p = [&](int c) __attribute__((always_inline)) {
            if (kMode == kOutputs) pcopy.load(records + c * record_step + DeltaRecord::kAtP, id);
        };
        const auto store_q = [&](int c) __attribute__((always_inline)) {
            if (kMode == kOutputs) qu.store(buffer_q(c) + L::kAtQ, id);
        };
        const auto store_p = [&](int c) __attribute__((always_inline)) {
            if (kMode == kOutputs) pcopy.store(buffer_q(c) + L::kAtP, id);
        };
        // A chunk's operands are loaded as soon as the registers are free, a chunk before
        // they go down; Q goes down a chunk ahead like K, or (FP32) in its own chunk.
        // There are no conditions, so that it is known at every wait which loads are
        // behind the one waited for: after the last chunk it is brought again.
        constexpr int kAhead = kPosts ? 1 : 0;
        const int last = chunks - 1;
        if (chunks > 0) {
            load_k(0);
            load_q(0);
            load_p(0);
            load_v(0);
            store_k(0);
            load_k(min(1, last));
            if (kAhead > 0) {
                store_q(0);
                load_q(min(1, last));
            }
            store_v();
            load_v(min(1, last));
        }
        for (int c = 0; c < chunks; ++c) {
            lds_barrier();  // A
            if (!kPosts) asm volatile("" : "+v"(id));  // places made anew, not kept
            // what the last chunk was the last to read; now, while the walking waves
            // need little of the LDS (their K S does)
            store_k(c + 1);
            load_k(min(c + 2, last));
            if (kPosts) {
                store_p(c);
                load_p(min(c + 1, last));
            }
            store_q(c + kAhead);
            load_q(min(c + kAhead + 1, last));
            wait_posts(c);
            if (!kPosts) {
                store_p(c);
                load_p(min(c + 1, last));
            }
            store_v();
            load_v(min(c + 2, last));
        }
        if (kMode == kOutputs && chunks > 0) lds_barrier();  // the last U
        return;
    }

    // O: 16 columns and kOwn token tiles of a chunk to a wave
    constexpr int kOwn = kWalkers;
    const int block = helper % kWalkers, own = (helper - 4) / kWalkers * kOwn;
    const int col = col0 + 16 * block + (lane & 15);
    const bool in = col < p.v_size;
    T* o = row_of<T>(p.o, packed, n, span, h) + skip * p.o.token;
    const uint32_t o_step = (uint32_t)p.o.token * sizeof(T);
    const uint32_t o_at = in ? (16 * own + 4 * g) * o_step + col * (uint32_t)sizeof(T) : kPastEnd;
    f32x4 y[kOwn], pf[kOwn];  // scale diag(e^G) Q S, and the scales of P's rows
    const auto finish = [&](int c) __attribute__((always_inline)) {
        const char* u_at = lds + L::kAtU + (kPosts ? (c & 1) * L::kBufferU : 0) +
                           block * L::kEachU + lane * 16;
        f32x4 u[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) u[i] = *reinterpret_cast<const f32x4*>(u_at + i * 1024);
        const char* column = u_at - lane * 16 + kC * 16 * 4 + (lane & 15) * 4;
        const int cut = *reinterpret_cast<const int*>(column);
        const float u_down = *reinterpret_cast<const float*>(column + 64);
        const Scale us = scale_of(max_groups(largest(u)));
        const Frag<2> b[2] = {split<2>(u[0], u[1], us.up), split<2>(u[2], u[3], us.up)};
        const int count = min(kC, span.count - c * kC);
        const __amdgpu_buffer_rsrc_t to = buffer_at(o + (int64_t)c * kC * p.o.token);
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            const int tile = own + i;
            f32x4 a{};
#pragma unroll
            for (int j = 0; j < 2; ++j)
                if (j <= tile / 2)
                    a = multiply(matrix_fragment<2>(buffer_q(c) + L::kAtP, lower_at(tile, j), lane),
                                 b[j], a);
            a *= pf[i] * (us.down * u_down);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int t = 16 * tile + 4 * g + r;
                const uint32_t off = o_at + (16 * i + r) * o_step;
                store_word(from_f32<T>(t < cut ? a[r] + y[i][r] : __builtin_nanf("")), to,
                           count == kC || t < count ? off : kPastEnd);
            }
        }
    };

    for (int c = 0; c < chunks; ++c) {
        lds_barrier();  // A
        if (c > 0) finish(c - 1);
        wait_posts(c);
        const float* f = reinterpret_cast<const float*>(lds + (c & 1) * L::kBuffer + L::kAtF) -
                         64 * DeltaRecord::kFirstChain;
        const char* s_at = lds + L::kAtS + block * L::kEachS;
        const float* downs =
            reinterpret_cast<const float*>(s_at + 2 * L::kSteps * 1024) + (lane & 15);
        const float first = downs[0], last = downs[16];  // of S's halves
        f32x4 z[kOwn];
#pragma unroll
        for (int i = 0; i < kOwn; ++i) y[i] = f32x4{};
#pragma unroll
        for (int j = 0; j < L::kSteps; ++j) {
            if (j == L::kSteps / 2)
#pragma unroll
                for (int i = 0; i < kOwn; ++i) {
                    z[i] = y[i] * first;
                    y[i] = f32x4{};
                }
            Frag<2> b;
#pragma unroll
            for (int r = 0; r < 2; ++r)
                b.part[r] = *reinterpret_cast<const half8_t*>(
                    s_at + (r * L::kSteps + j) * 1024 + lane * 16);
#pragma unroll
            for (int i = 0; i < kOwn; ++i)
                y[i] = multiply(row_fragment<T, kK>(buffer_q(c) + L::kAtQ, own + i, j, lane), b,
                                y[i]);
        }
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            const int at = 4 * (own + i) + g;
            y[i] = (y[i] * last + z[i]) *
                   reinterpret_cast<const f32x4*>(f + 64 * DeltaRecord::kQueryRise)[at];
            pf[i] = reinterpret_cast<const f32x4*>(f + 64 * DeltaRecord::kP)[at];
        }
    }
    if (chunks > 0) {
        lds_barrier();  // the last U
        finish(chunks - 1);
    }
}

template <class T, int kK, int kWalkers, int kMode, bool kWide>
hipError_t launch_rows(const DeltaChunks& a, hipStream_t stream) {
    using L = Layout<T, kK, kWalkers, kMode>;
    static_assert(L::kBytes <= 160 * 1024, "LDS of a CU");
    static_assert(64 * (2 * kWalkers + L::kHelpers) <= kDeltaMostThreads, "one launch");
    constexpr int kColumns = 16 * kWalkers;
    int64_t slices = (a.v_size + kColumns - 1) / kColumns;
    if (kMode == kPartSteps) slices += (a.k_size + kColumns - 1) / kColumns;
    const int64_t walks = a.part_chunks > 0 ? a.parts : a.batch;
    const void* kernel =
        reinterpret_cast<const void*>(delta_chain_kernel<T, kK, kWalkers, kMode, kWide>);
    if (hipError_t e =
            hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, L::kBytes))
        return e;
    hipLaunchKernelGGL((delta_chain_kernel<T, kK, kWalkers, kMode, kWide>),
                       dim3((unsigned)walk_blocks(walks * a.v_heads, slices)),
                       dim3(64 * (2 * kWalkers + L::kHelpers)), L::kBytes, stream, a);
    return hipGetLastError();
}

template <class T, int kK, int kWalkers, int kMode>
hipError_t launch(const DeltaChunks& a, hipStream_t stream) {
    return a.wide && a.wide_values ? launch_rows<T, kK, kWalkers, kMode, true>(a, stream)
                                   : launch_rows<T, kK, kWalkers, kMode, false>(a, stream);
}

}  // namespace

hipError_t launch_delta_chain(const DeltaChunks& a, DeltaWalk walk, hipStream_t stream) {
    return by_dtype(a.dtype, [&](auto t) {
        using T = decltype(t);
        constexpr bool kF32 = sizeof(T) == 4;
        const bool small = a.k_size <= 64;
        switch (walk) {
            case kDeltaStates:
                if (narrow(a))
                    return small ? launch<T, 64, 1, kStates>(a, stream)
                                 : launch<T, 128, 1, kStates>(a, stream);
                return small ? launch<T, 64, 2, kStates>(a, stream)
                             : launch<T, 128, 2, kStates>(a, stream);
            case kDeltaParts:
                return small ? launch<T, 64, 4, kPartSteps>(a, stream)
                             : launch<T, 128, kF32 ? 2 : 4, kPartSteps>(a, stream);
            default:
                if (narrow(a))
                    return small ? launch<T, 64, 1, kOutputs>(a, stream)
                                 : launch<T, 128, 1, kOutputs>(a, stream);
                return small ? launch<T, 64, 2, kOutputs>(a, stream)
                             : launch<T, 128, kF32 ? 1 : 2, kOutputs>(a, stream);
        }
    });
}

}  // namespace sgemm_emu
