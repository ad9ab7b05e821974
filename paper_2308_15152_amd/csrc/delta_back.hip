// The gated delta rule's gradient, the walk back over a sequence's chunks with
// the gradient D of the state after the chunk:
//   dU = P^T dO + diag(e^{G_64 - G}) K D,   dY = T^T dU,   dV = diag(beta) dY,
//   D before = e^{G_64} D + scale (diag(e^G) Q)^T dO - (diag(e^G) K)^T dV.
// Columns are independent here too, and the work is shared out as on the way
// forward (delta_chain.hip): pairs of walking waves carry 16 columns of D and
// do what waits for D; helping waves bring K and T^T of the next chunk, and make
// what does not wait, P^T dO and the product with Q, a chunk ahead from Q, P^T and dO,
// which they bring two chunks ahead.  Leaves D after and dY of every chunk.  A
// sequence cut into parts is walked twice, as on the way forward: every part
// but the first from D = 0, then all from their own (M^T takes D across a part).
// Measured: 2 x 4096 tokens of 16 heads (bfloat16, 128 x 128) 214 us, 3.3 us a chunk,
// bound by the chain like the walk forward.
//
// One barrier a chunk (A).  Inside a chunk a walking wave posts when it has taken
// its two products; then the helpers put down the next ones.  In FP32, for whose
// two parts LDS holds Q only once, the post is a second barrier (B), before which
// the helpers have read the Q that they overwrite after it.
#include <type_traits>

#include "delta_chunk.hpp"

namespace sgemm_emu {

namespace {

// LDS, in bytes, and the number of helping waves.
// kWalkers: groups of 16 columns, a pair of walking waves each.
template <class T, int kK, int kWalkers>
struct Layout {
    static constexpr bool kPosts = sizeof(T) == 2 || kK == 64;  // as LDS allows
    // with eight helpers, four bring K and T^T and four Q, P^T and dO
    static constexpr int kHelpers = kPosts && kWalkers > 1 ? 8 : 4;
    static constexpr int kParts = kPartsOf<T>;
    static constexpr int kSteps = kK / 32, kTiles = kK / 16;
    static constexpr int kHalf = kTiles / 2;  // row tiles of a wave of a pair
    static constexpr int kRows = kParts * 4 * kSteps * 1024;
    static constexpr int kMatrix = 2 * DeltaRecord::kMatrix;
    // two buffers of these
    static constexpr int kAtK = 0;
    static constexpr int kAtTt = kAtK + kRows;
    static constexpr int kAtF = kAtTt + kMatrix;
    static constexpr int kFactorBytes = 256 * DeltaRecord::kBack;
    static constexpr int kBuffer = kAtF + kFactorBytes;
    // one or two of these
    static constexpr int kAtQ = 0;
    static constexpr int kAtPt = kAtQ + kRows;
    static constexpr int kAtFq = kAtPt + kMatrix;
    static constexpr int kAheadBytes = 256 * DeltaRecord::kAhead;
    static constexpr int kAtDo = kAtFq + kAheadBytes;
    using V = Values<T, kWalkers, 256>;
    static constexpr int kBufferQ = kAtDo + kWalkers * V::kEach;
    static constexpr int kAtQs = 2 * kBuffer;
    // the products, as the walking waves hold them: 4 tiles and kTiles tiles
    static constexpr int kAtProducts = kAtQs + (kPosts ? 2 : 1) * kBufferQ;
    static constexpr int kEach = (4 + kTiles) * 1024;
    // what the waves of a pair give each other
    static constexpr int kAtX = kAtProducts + kWalkers * kEach;
    static constexpr int kEachX = 4 * 1024 + 64;
    // steps done: [wave] products taken; [2 kWalkers + wave] given to the other
    static constexpr int kAtPosts = kAtX + kWalkers * kEachX;
    static constexpr int kBytes = kAtPosts + 16 * kWalkers;
};

// kCarry: only D before every part, from zero after it; kWide: as in delta_chain.hip.
template <class T, int kK, int kWalkers, bool kCarry, bool kWide>
__global__ __launch_bounds__(64 * (2 * kWalkers + Layout<T, kK, kWalkers>::kHelpers), 1)
void delta_back_kernel(DeltaChunks p) {
    using L = Layout<T, kK, kWalkers>;
    constexpr bool kPosts = L::kPosts;
    constexpr int kHelpers = L::kHelpers;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    int* posts = reinterpret_cast<int*>(lds + L::kAtPosts);

    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int g = lane >> 4;
    const int slices = (p.v_size + 16 * kWalkers - 1) / (16 * kWalkers);
    const WalkTask w = walk_task(slices);
    const int slice = w.slice;
    const int h = w.task % p.v_heads, index = w.task / p.v_heads;
    if (index >= (p.part_chunks > 0 ? p.parts : p.batch)) return;  // the whole block
    const int kh = h / (p.v_heads / p.k_heads);
    const bool packed = p.cu_seqlens != nullptr;
    const Walk walk = walk_of(p, index);
    const int chunks = walk.count;
    if (chunks < 0 || (kCarry && walk.part == 0)) return;  // the whole block
    const int n = walk.n;
    const Span span = {walk.span.first, walk.span.count - walk.first * kC};  // from the part on
    const int first_chunk = walk.base + walk.first;
    const int col0 = slice * kWalkers * 16;
    const char* records = p.records + ((int64_t)first_chunk * p.v_heads + h) * p.record_bytes;
    const int64_t record_step = (int64_t)p.v_heads * p.record_bytes;
    const int64_t skip = (int64_t)walk.first * kC;  // tokens of the parts before
    if (threadIdx.x < 4 * kWalkers) posts[threadIdx.x] = 0;

    // Steps s = 0, 1, ... are chunks from the last to the first.
    if (wave < 2 * kWalkers) {
        const int group = wave >> 1, half = wave & 1;
        const bool leads = half == 0;
        const int row0 = half * 16 * L::kHalf;
        const int col = col0 + 16 * group + (lane & 15);
        const bool in = col < p.v_size;
        f32x4 D[L::kHalf];  // rows row0 + 16 i + 4 g + r
        const int64_t sequence = ((int64_t)n * p.v_heads + h) * p.k_size * p.v_size;
        const int64_t part = ((int64_t)index * p.v_heads + h) * p.k_size * p.v_size;
        const float* from = kCarry              ? nullptr
                            : p.part_chunks > 0 ? p.part_dstates + part
                            : p.dfinal          ? p.dfinal + sequence
                                                : nullptr;
#pragma unroll
        for (int i = 0; i < L::kHalf; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = row0 + 16 * i + 4 * g + r;
                D[i][r] = from && in && row < p.k_size ? from[(int64_t)row * p.v_size + col] : 0.0f;
            }
        const char* products = lds + L::kAtProducts + group * L::kEach + lane * 16;
        char* x_at = lds + L::kAtX + group * L::kEachX;
        int* given = posts + 2 * kWalkers;
        T* dv = row_of<T>(p.dv, packed, n, span, h) + skip * p.dv.token;
        const uint32_t v_step = (uint32_t)p.dv.token * sizeof(T);
        const uint32_t v_at = in ? 4 * g * v_step + col * (uint32_t)sizeof(T) : kPastEnd;
        const uint32_t f_at = in ? 4u * (4 * g * p.v_size + col) : kPastEnd;
        const uint32_t d_at = in ? 4u * ((row0 + 4 * g) * p.v_size + col) : kPastEnd;
        if (chunks > 0) {
            lds_barrier();
            lds_barrier();
        }
        for (int s = 0; s < chunks; ++s) {
            const int c = chunks - 1 - s;
            const char* at = lds + (s & 1) * L::kBuffer;
            const float* f =
                reinterpret_cast<const float*>(at + L::kAtF) - 64 * DeltaRecord::kFirstBack;
            const auto factor = [&](int which, int tile) __attribute__((always_inline)) {
                return reinterpret_cast<const f32x4*>(f + 64 * which)[4 * tile + g];
            };
            const int count = min(kC, span.count - c * kC);
            const int64_t task = (int64_t)(first_chunk + c) * p.v_heads + h;
            lds_barrier();  // A
            f32x4 u[4], add[L::kHalf];
            if (leads)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    u[i] = *reinterpret_cast<const f32x4*>(products + i * 1024);
#pragma unroll
            for (int i = 0; i < L::kHalf; ++i)
                add[i] = *reinterpret_cast<const f32x4*>(products + (4 + half * L::kHalf + i) * 1024);
            if (kPosts) {
                __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
                __hip_atomic_store(posts + wave, s + 1, __ATOMIC_RELAXED,
                                   __HIP_MEMORY_SCOPE_WORKGROUP);
            } else {
                lds_barrier();  // B
            }
            if (!kCarry) {
                const __amdgpu_buffer_rsrc_t to =
                    buffer_at(p.dstates + task * ((p.k_size + 15) / 16 * 16) * p.v_size);
#pragma unroll
                for (int i = 0; i < L::kHalf; ++i)
                    if (row0 + 16 * i < p.k_size)
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            __builtin_amdgcn_raw_buffer_store_b32(
                                __builtin_bit_cast(uint32_t, (float)D[i][r]), to, d_at,
                                4 * (16 * i + r) * p.v_size, 0);
            }
            // dU
            Frag<2> b[2];
            float down;
            f32x4 a[4] = {};
            const Scale ds = scale_of(max_groups(largest(D)));
#pragma unroll
            for (int j = 0; j < L::kSteps / 2; ++j) {
                const Frag<2> db = split<2>(D[2 * j], D[2 * j + 1], ds.up);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    a[i] = multiply(row_fragment<T, kK>(at + L::kAtK, i, half * (L::kSteps / 2) + j,
                                                        lane), db, a[i]);
            }
            if (!leads) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    *reinterpret_cast<f32x4*>(x_at + i * 1024 + lane * 16) = a[i] * ds.down;
                give(given + wave, s + 1);
                wait_given(given + wave - 1, s + 1);
                take(given + wave - 1, s + 1, [&]() __attribute__((always_inline)) {
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
                take(given + wave + 1, s + 1, [&]() __attribute__((always_inline)) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        other[i] = *reinterpret_cast<const f32x4*>(x_at + i * 1024 + lane * 16);
                });
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const f32x4 tail = factor(DeltaRecord::kTail, i);
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        u[i][r] = __builtin_fmaf(
                            tail[r], __builtin_fmaf(a[i][r], ds.down, other[i][r]), u[i][r]);
                }
                // dY, and dV
                f32x4 y[4] = {};
                int cut = 0;
                {
                    float top = column_largest(u);
                    const bool cuts = __any(!finite(top));
                    if (cuts) cut = cut_column_back(u, top);
                    const Scale us = scale_of(top);
                    const Frag<2> ub[2] = {split<2>(u[0], u[1], us.up), split<2>(u[2], u[3], us.up)};
                    const __amdgpu_buffer_rsrc_t dy = buffer_at(p.dsides + task * kC * p.v_size);
                    const __amdgpu_buffer_rsrc_t to = buffer_at(dv + (int64_t)c * kC * p.dv.token);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
#pragma unroll
                        for (int j = i / 2; j < 2; ++j)
                            y[i] = multiply(matrix_fragment<2>(at + L::kAtTt, upper_at(i, j), lane), ub[j],
                                            y[i]);
                        y[i] *= factor(DeltaRecord::kTt, i) * us.down;
                        const f32x4 beta = factor(DeltaRecord::kBeta, i);
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            if (!kCarry)
                                __builtin_amdgcn_raw_buffer_store_b32(
                                    __builtin_bit_cast(uint32_t, (float)y[i][r]), dy, f_at,
                                    4 * (16 * i + r) * p.v_size, 0);
                            y[i][r] *= beta[r];
                            if (kCarry) continue;
                            store_word(from_f32<T>(y[i][r]), to,
                                       count == kC || 16 * i + 4 * g + r < count
                                           ? v_at + (16 * i + r) * v_step : kPastEnd);
                        }
                        y[i] *= -factor(DeltaRecord::kRise, i);
                    }
                    if (cuts && !kCarry)  // over what was stored
#pragma unroll 1
                        for (int t = fresh(4 * g); t < cut; t += t % 4 == 3 ? 13 : 1) {
                            store_word(__builtin_nanf(""), dy,
                                       in ? 4u * (t * p.v_size + col) : kPastEnd);
                            store_word(from_f32<T>(__builtin_nanf("")), to,
                                       in && t < count
                                           ? t * v_step + col * (uint32_t)sizeof(T) : kPastEnd);
                        }
                }
                const Scale ys = scale_of(max_groups(largest(y)));
                b[0] = split<2>(y[0], y[1], ys.up);
                b[1] = split<2>(y[2], y[3], ys.up);
                down = cut == 0 ? ys.down : __builtin_nanf("");
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int q = 0; q < 2; ++q)
                        *reinterpret_cast<half8_t*>(x_at + (2 * j + q) * 1024 + lane * 16) =
                            b[j].part[q];
                reinterpret_cast<float*>(x_at + 4096)[lane & 15] = down;
                give(given + wave, s + 1);
            }
            // D
            const float decay = f[64 * DeltaRecord::kDecay];
#pragma unroll
            for (int i = 0; i < L::kHalf; ++i) {
                f32x4 a{};
#pragma unroll
                for (int j = 0; j < 2; ++j)  // lo.lo too: as for S
                    a = multiply<true>(
                        column_fragment<T, kK>(at + L::kAtK, half * L::kHalf + i, j, lane), b[j], a);
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    D[i][r] = __builtin_fmaf(a[r], down,
                                             __builtin_fmaf(decay, D[i][r], add[i][r]));
            }
        }
        float* to = kCarry                            ? p.part_dstates + part
                    : p.dinitial && walk.part == 0 ? p.dinitial + sequence
                                                   : nullptr;
        if (to && in)
#pragma unroll
            for (int i = 0; i < L::kHalf; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int row = row0 + 16 * i + 4 * g + r;
                    if (row < p.k_size) to[(int64_t)row * p.v_size + col] = D[i][r];
                }
        return;
    }

    // ---- the helping waves
    if (chunks == 0) return;
    const int helper = wave - 2 * kWalkers, last = chunks - 1;
    const int id = (threadIdx.x - 128 * kWalkers) & 255;
    const T* k = row_of<const T>(p.k, packed, n, span, kh) + skip * p.k.token;
    const T* q = row_of<const T>(p.q, packed, n, span, kh) + skip * p.q.token;
    const T* d_o = row_of<const T>(p.d_o, packed, n, span, h) + skip * p.d_o.token + col0;
    Rows<T, kK, 256> ku, qu;
    Copy<L::kMatrix, 256> tcopy, pcopy;
    Copy<L::kFactorBytes, 256> fcopy;
    Copy<L::kAheadBytes, 256> fqcopy;
    typename L::V vu;
    const auto load_k = [&](int s) __attribute__((always_inline)) {
        const int c = chunks - 1 - s;
        const char* record = records + c * record_step;
        ku.load(k + (int64_t)c * kC * p.k.token, p.k.token, min(kC, span.count - c * kC), p.k_size,
                kWide, reinterpret_cast<const float*>(record) + 64 * DeltaRecord::kKeyScale, id);
        tcopy.load(record + DeltaRecord::kAtTt, id);
        fcopy.load(record + 256 * DeltaRecord::kFirstBack, id);
    };
    const auto store_k = [&](int s) __attribute__((always_inline)) {
        char* to = lds + (s & 1) * L::kBuffer;
        ku.store(to + L::kAtK, id);
        tcopy.store(to + L::kAtTt, id);
        fcopy.store(to + L::kAtF, id);
    };
    const auto load_q = [&](int s) __attribute__((always_inline)) {
        const int c = chunks - 1 - s, count = min(kC, span.count - c * kC);
        const char* record = records + c * record_step;
        qu.load(q + (int64_t)c * kC * p.q.token, p.q.token, count, p.k_size, kWide,
                reinterpret_cast<const float*>(record) + 64 * DeltaRecord::kQueryScale, id);
        pcopy.load(record + DeltaRecord::kAtPt, id);
        fqcopy.load(record + 256 * DeltaRecord::kFirstAhead, id);
        vu.load(d_o + (int64_t)c * kC * p.d_o.token, p.d_o.token, count, p.v_size - col0,
                kWide, id);
    };
    const auto buffer_q = [&](int s) __attribute__((always_inline)) {
        return lds + L::kAtQs + (kPosts ? (s & 1) * L::kBufferQ : 0);
    };
    const auto store_q = [&](int s) __attribute__((always_inline)) {
        char* to = buffer_q(s);
        qu.store(to + L::kAtQ, id);
        pcopy.store(to + L::kAtPt, id);
        fqcopy.store(to + L::kAtFq, id);
        vu.store(to + L::kAtDo, id);
    };

    // P^T dO and the product with Q: 16 columns to a wave, kOwn of the 4 token
    // tiles and kOwnK of the kTiles element tiles
    constexpr int kOwn = 4 * kWalkers / kHelpers, kOwnK = L::kTiles * kWalkers / kHelpers;
    static_assert(kOwn >= 1 && kOwnK >= 1, "every wave has a part");
    const int block = helper % kWalkers, part = helper / kWalkers;
    f32x4 pd[kOwn], qd[kOwnK];
    const auto make = [&](int s) __attribute__((always_inline)) {
        const char* at = buffer_q(s);
        const float* f =
            reinterpret_cast<const float*>(at + L::kAtFq) - 64 * DeltaRecord::kFirstAhead;
        const char* v_at = at + L::kAtDo + block * L::V::kEach +
                           value_slot(lane, block) * 4 * (int)sizeof(T);
        f32x4 o[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            T x[4];
            __builtin_memcpy(x, v_at + i * 64 * 4 * sizeof(T), 4 * sizeof(T));
#pragma unroll
            for (int r = 0; r < 4; ++r) o[i][r] = to_f32(x[r]);
        }
        float top = column_largest(o);
        const bool cuts = __any(!finite(top));
        int cut = 0;
        if (cuts) cut = cut_column_back(o, top);
        const Scale os = scale_of(top);
        {
            const Frag<L::kParts> b[2] = {split<L::kParts>(o[0], o[1], os.up),
                                          split<L::kParts>(o[2], o[3], os.up)};
#pragma unroll
            for (int i = 0; i < kOwn; ++i) {
                const int tile = part * kOwn + i;
                f32x4 a{};
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    if (j >= tile / 2)
                        a = multiply(matrix_fragment<2>(at + L::kAtPt, upper_at(tile, j), lane), b[j], a);
                pd[i] = a * reinterpret_cast<const f32x4*>(f + 64 * DeltaRecord::kPt)[4 * tile + g] * os.down;
            }
            if (cuts) {
                const int first = fresh(cut - 16 * part * kOwn - 4 * g);
#pragma unroll
                for (int i = 0; i < kOwn; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (16 * i + r < first) pd[i][r] = __builtin_nanf("");
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            o[i] *= reinterpret_cast<const f32x4*>(f + 64 * DeltaRecord::kQueryRise)[4 * i + g];
        const Scale qs = scale_of(max_groups(largest(o)));
        const Frag<2> b[2] = {split<2>(o[0], o[1], qs.up), split<2>(o[2], o[3], qs.up)};
#pragma unroll
        for (int i = 0; i < kOwnK; ++i) {
            f32x4 a{};
#pragma unroll
            for (int j = 0; j < 2; ++j)
                a = multiply<true>(column_fragment<T, kK>(at + L::kAtQ, part * kOwnK + i, j, lane), b[j], a);
            qd[i] = a * (cut == 0 ? qs.down : __builtin_nanf(""));
        }
    };
    const auto put = [&]() __attribute__((always_inline)) {
        char* to = lds + L::kAtProducts + block * L::kEach + lane * 16;
#pragma unroll
        for (int i = 0; i < kOwn; ++i)
            *reinterpret_cast<f32x4*>(to + (part * kOwn + i) * 1024) = pd[i];
#pragma unroll
        for (int i = 0; i < kOwnK; ++i)
            *reinterpret_cast<f32x4*>(to + (4 + part * kOwnK + i) * 1024) = qd[i];
    };

    // Loads are a step ahead of the stores and without conditions, as in delta_chain.hip.
    const auto run = [&](auto brings_k, auto brings_q) __attribute__((always_inline)) {
        if (brings_k) {
            load_k(0);
            store_k(0);
            load_k(min(1, last));
        }
        if (brings_q) {
            load_q(0);
            store_q(0);
            load_q(min(1, last));
        }
        lds_barrier();
        make(0);
        lds_barrier();
        put();
        if (brings_q) {
            store_q(1);
            load_q(min(2, last));
        }
        for (int s = 0; s < chunks; ++s) {
            lds_barrier();  // A
            if (brings_k) {
                store_k(s + 1);
                load_k(min(s + 2, last));
            }
            if (kPosts && brings_q) {
                store_q(s + 2);
                load_q(min(s + 3, last));
            }
            make(s + 1);
            if (kPosts) {
                // every walking wave is in this step and posts on its way
#pragma unroll
                for (int w = 0; w < 2 * kWalkers; ++w) wait_given(posts + w, s + 1);
                __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
            } else {
                lds_barrier();  // B
            }
            put();
            if (!kPosts && brings_q) {
                store_q(s + 2);
                load_q(min(s + 3, last));
            }
        }
    };
    if constexpr (kHelpers == 4)
        run(std::true_type{}, std::true_type{});
    else if (helper < 4)
        run(std::true_type{}, std::false_type{});
    else
        run(std::false_type{}, std::true_type{});
}

template <class T, int kK, int kWalkers, bool kCarry, bool kWide>
hipError_t launch_rows(const DeltaChunks& a, hipStream_t stream) {
    using L = Layout<T, kK, kWalkers>;
    static_assert(L::kBytes <= 160 * 1024, "LDS of a CU");
    static_assert(64 * (2 * kWalkers + L::kHelpers) * 2 <= kDeltaMostThreads * kWalkers,
                  "32 columns: one launch");
    const int64_t slices = (a.v_size + 16 * kWalkers - 1) / (16 * kWalkers);
    const int64_t walks = a.part_chunks > 0 ? a.parts : a.batch;
    const void* kernel =
        reinterpret_cast<const void*>(delta_back_kernel<T, kK, kWalkers, kCarry, kWide>);
    if (hipError_t e =
            hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, L::kBytes))
        return e;
    hipLaunchKernelGGL((delta_back_kernel<T, kK, kWalkers, kCarry, kWide>),
                       dim3((unsigned)walk_blocks(walks * a.v_heads, slices)),
                       dim3(64 * (2 * kWalkers + L::kHelpers)), L::kBytes, stream, a);
    return hipGetLastError();
}

template <class T, int kK, int kWalkers, bool kCarry>
hipError_t launch(const DeltaChunks& a, hipStream_t stream) {
    return a.wide && a.wide_values ? launch_rows<T, kK, kWalkers, kCarry, true>(a, stream)
                                   : launch_rows<T, kK, kWalkers, kCarry, false>(a, stream);
}

}  // namespace

hipError_t launch_delta_chain_back(const DeltaChunks& a, DeltaWalk walk, hipStream_t stream) {
    return by_dtype(a.dtype, [&](auto t) {
        using T = decltype(t);
        constexpr int kLarge = sizeof(T) == 4 ? 1 : 2;  // walking waves, keys above 64
        if (narrow(a)) {
            if (walk == kDeltaParts)
                return a.k_size <= 64 ? launch<T, 64, 1, true>(a, stream)
                                      : launch<T, 128, 1, true>(a, stream);
            return a.k_size <= 64 ? launch<T, 64, 1, false>(a, stream)
                                  : launch<T, 128, 1, false>(a, stream);
        }
        if (walk == kDeltaParts)
            return a.k_size <= 64 ? launch<T, 64, 2, true>(a, stream)
                                  : launch<T, 128, kLarge, true>(a, stream);
        return a.k_size <= 64 ? launch<T, 64, 2, false>(a, stream)
                              : launch<T, 128, kLarge, false>(a, stream);
    });
}

}  // namespace sgemm_emu
