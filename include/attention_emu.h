/*
 * attention_emu.h -- C ABI of the softmax attention operators of
 * libsgemm_emu.so.  Status codes, streams, graph capture, threads and ownership
 * of memory are as in sgemm_emu.h; types, views and what is asked of strides and
 * spans as in mixing_emu.h.
 */
#ifndef ATTENTION_EMU_H
#define ATTENTION_EMU_H

#include "mixing_emu.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Attention over whole sequences.  q, o: (batch, tokens, q_heads, size), k, v:
 * (batch, keys, k_heads, size), all of one dtype; query head h reads key head h /
 * (q_heads / k_heads).  Per sequence and query head, for token i:
 *   s_j = scale q_i k_j,  lse_i = log sum_j e^{s_j},  o_i = sum_j e^{s_j - lse_i} v_j
 * over the keys that it sees: all of its sequence's n keys, or, if `causal`, keys 0 to
 * i + n - t of a sequence of t tokens (the last token sees all).  A token that sees
 * no key (or only scores of -infinity) has o = 0 and lse = -infinity.
 * lse (FP32, view `lse`: batch, token and head strides, p NULL: not wanted) is what
 * the gradient needs.
 *   cu_seqlens NULL: `batch` sequences of `tokens` tokens and `keys` keys.
 *   else: packed sequences; the views' batch stride is not used, `tokens` is the
 *     number of rows in all, and sequence n is rows cu_seqlens[n] to
 *     cu_seqlens[n+1] - 1 of q, o and lse, and rows cu_keys[n] to cu_keys[n+1] - 1 of k
 *     and v (`keys` rows in all; cu_keys NULL: cu_seqlens, with keys == tokens).
 *     Both are device int32 with batch + 1 values, not decreasing; values
 *     outside the rows are clamped to them; where they decrease, results are unspecified, and
 *     nothing outside the tensors is touched.  Rows of no sequence are not written.
 * A key or value that is not finite reaches only tokens that see it (as NaN, it may be, where the
 * formula says infinity).
 * Scores, statistics and sums are FP32; weights below 2^-126 are zeros.  With 16-bit types the
 * weights e^{s_j - m} are rounded to the type before they multiply v (FP16: to 2^-32 of the row's
 * largest where they are small), the results once.  FP32 operands are taken as
 * two FP16 parts with a power of two for each row (22 bits of an element, down to 2^-39 of its
 * row's largest), and weights, times their value's power of two, in the same way with one for each
 * token (22 bits, down to 2^-34 of the largest such product that the token has), or both as they are
 * in short calls.
 * workspace: device memory, 256-byte aligned, at least what the _workspace query
 *   for the same arguments returns (for parts of the keys where the query rows alone do not fill
 *   the device, and for FP32's parts; 0 bytes where neither is); its contents need not be kept.
 * Sizes: size <= 128, q_heads a multiple of k_heads, with FP32 at most 2^14, token strides <=
 * 2^22, scale finite and not zero, tokens x q_heads and keys below 2^31 for a sequence, and blocks of 32
 * rows or keys below 2^30 in all.
 * Errors: _DIM (also keys != tokens without cu_keys), _UNSUPPORTED (dtype, sizes, scale,
 * strides and head counts above), _NULL, _STRIDE, _ALIAS, _HIP.
 */
typedef struct {
    int32_t dtype, batch, tokens, keys, q_heads, k_heads, size, causal;
    float scale;
    int32_t reserved;
    const int32_t* cu_seqlens;
    const int32_t* cu_keys;
    sgemm_emu_view_t q, k, v, o, lse;
    void* workspace;
    int64_t workspace_bytes;
} attention_emu_forward_t;

/* Bytes of workspace, or a negative error; pointers are not looked at except for being
 * NULL. */
int64_t attention_emu_forward_workspace(const attention_emu_forward_t* a);
int attention_emu_forward(const attention_emu_forward_t* a, hipStream_t stream);

/* Its gradient: from o and lse of the forward pass and d_o (like o) to dq, dk, dv
 * (the inputs' type):
 *   p_ij = e^{s_ij - lse_i},  dv_j = sum_i p_ij do_i,
 *   ds_ij = p_ij (do_i v_j - do_i o_i),  dq_i = scale sum_j ds_ij k_j,
 *   dk_j = scale sum_i ds_ij q_i,
 * sums over tokens and over a key head's query heads in FP32 in a fixed order; with 16-bit
 * types p and ds are rounded to the type before they multiply.  p is taken as one at most, for
 * it is off by the last bit of lse, which is not small beside one where scores are of 2^20 and
 * more.  o and lse may be those of more
 * keys than are given here (keys in parts: dq is the sum of the parts').  Gradients of
 * tokens that see no key and of keys that no token sees are zero.  Where q, k, v, o or d_o is
 * not finite, any gradient of its sequence's key head may not be; other sequences and
 * heads are not reached.
 * workspace: as above, and for a number for each query row. */
typedef struct {
    int32_t dtype, batch, tokens, keys, q_heads, k_heads, size, causal;
    float scale;
    int32_t reserved;
    const int32_t* cu_seqlens;
    const int32_t* cu_keys;
    sgemm_emu_view_t q, k, v, o, lse, d_o, dq, dk, dv;
    void* workspace;
    int64_t workspace_bytes;
} attention_emu_backward_t;

int64_t attention_emu_backward_workspace(const attention_emu_backward_t* a);
int attention_emu_backward(const attention_emu_backward_t* a, hipStream_t stream);

/* The form for single tokens: `tokens` new tokens (one, or a few drafted ones) of each
 * of `batch` sequences, whose keys and values are a prefix that all of them share
 * followed by a cache of their own:
 *   q, o: (batch, tokens, q_heads, size),
 *   prefix_k, prefix_v: (prefix, k_heads, size) (views; the batch stride is not used;
 *     prefix 0: none), read once for the whole batch,
 *   k, v: (n_slots, capacity, k_heads, size); sequence b has row slots[b] (device,
 *     int32) or b if slots is NULL, and of it the first lengths[b] positions (device, int32;
 *     clamped to 0 .. capacity), the new tokens' own keys and values among them: token i
 *     sees the whole prefix and the cache's positions 0 to lengths[b] - tokens + i.
 * A slot outside [0, n_slots) leaves its sequence out (o = 0 there).  Positions behind
 * lengths[b] are not used, whatever they hold.
 * workspace as above (for the tokens' shares of the prefix and of parts of the caches; 0
 *   bytes where one part is all there is). */
typedef struct {
    int32_t dtype, batch, tokens, prefix, capacity, n_slots, q_heads, k_heads, size;
    float scale;
    sgemm_emu_view_t q, prefix_k, prefix_v, k, v, o;
    const int32_t* lengths;
    const int32_t* slots;
    void* workspace;
    int64_t workspace_bytes;
} attention_emu_step_t;

int64_t attention_emu_step_workspace(const attention_emu_step_t* a);
int attention_emu_step(const attention_emu_step_t* a, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* ATTENTION_EMU_H */
