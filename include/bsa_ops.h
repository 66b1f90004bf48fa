/*
 * bsa_ops.h - operators that stand beside block-sparse attention on AMD
 *             Instinct MI355X (gfx950): rotary positions on up to three axes,
 *             and attention over a sliding window with first tokens that stay
 *             visible, forward and backward.
 *
 * They live in libbsa_ops.so and keep the conventions of bsa.h: every entry
 * point returns a bsa_status and never throws; bsa_ops_last_error() tells
 * more about the calling thread's last failure; "device" pointers belong to
 * the current device; streams are hipStream_t values passed as void* (NULL:
 * the legacy default stream); calls are asynchronous on `stream`.  No entry
 * point allocates, frees, synchronises or reads device memory on the host, so
 * all of them can be captured into a HIP graph.
 *
 * Tensors are [batch, tokens, heads, head_dim] in general strided form:
 * strides are in elements and ordered (batch, head, token), none negative,
 * the head-dim stride is 1, and every token row starts 16-byte aligned.
 * Inputs may repeat rows (a stride of 0); the rows of an output must not
 * overlap.  Outputs do not overlap inputs unless an entry point says so.
 */
#ifndef BSA_OPS_H_
#define BSA_OPS_H_

#include "bsa.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Detail of the last failure on the calling thread (thread-local storage,
 * valid until the next call on this thread). */
BSA_API const char* bsa_ops_last_error(void);

/* ---------------------------------------------------------------------------
 * Rotary positions
 *
 * The first pairs[0] + pairs[1] + pairs[2] pairs of a head are turned, pair i
 * by the angle position[axis of i] * freq[i]: the first pairs[0] pairs by the
 * position on axis 0 (time), the next pairs[1] by axis 1 (height), the next
 * pairs[2] by axis 2 (width).  With P turned pairs, pair i is elements
 * (2i, 2i + 1) when interleaved, else (i, i + P); the elements from 2P on are
 * copied.  (x, y) becomes (x cos t - y sin t, x sin t + y cos t).  Angles are
 * formed in 64 bits and reduced before the sine and cosine are taken in 32, so
 * far positions lose nothing; the rotation is computed in 32 bits and rounded
 * once.
 *
 * inverse != 0 turns by the opposite angle.  That is the backward pass: given
 * the gradients of the rotated tensors as q and k, it returns those of the
 * originals.
 *
 * Positions come from a device array, or from a grid.  positions is int32,
 * axis a of token n of batch b at a * pos_stride[0] + b * pos_stride[1] + n
 * (axes with no pairs are not read).  Without it, token n lies at
 * (n / (grid[1] * grid[2]), n / grid[2] % grid[1], n % grid[2]) + origin; the
 * tokens past the grid's last (text behind a clip, say) are copied unturned.
 */
typedef struct {
  int32_t batch, heads, kv_heads, seq, head_dim, dtype; /* kv_heads 0: q alone */
  int32_t pairs[3];
  int32_t interleaved, inverse;
  int32_t grid[3], origin[3]; /* used when positions is NULL */
  int32_t kv_rows;            /* tokens that k_out and v_out have room for (seq or more without rows) */
  int64_t pos_stride[2];      /* (axis, batch), elements */
  int64_t q_stride[3], k_stride[3], v_stride[3];             /* (batch, head, token), elements */
  int64_t q_out_stride[3], k_out_stride[3], v_out_stride[3]; /* (batch, head, token), elements */
} bsa_rope_shapes;

/*
 * q_out and k_out from q and k; v, when given, is copied to v_out.
 *   freq     device double [P], angle per position in radians.
 *   lengths  device int32 [batch] or NULL: tokens of each sequence; output rows
 *            of the tokens from there on keep what they held.
 *   rows     device int32 [batch] or NULL: the row of k_out and v_out that a
 *            sequence's first token goes to, the others following it (a cache
 *            that the new tokens are appended to); NULL means row 0.  Rows
 *            outside [0, kv_rows) are not written.
 * q_out may be q itself, and k_out k itself when rows is NULL (same strides);
 * v_out may be v itself likewise.  No tensor is the output of another.
 * dtype bf16, f16 or f32; head_dim a multiple of 8 up to 256.  k may be NULL
 * with kv_heads 0; v may be NULL.  batch and seq may be 0.
 */
BSA_API bsa_status bsa_rope(const bsa_rope_shapes* shapes, const double* freq, const int32_t* positions,
                            const int32_t* lengths, const int32_t* rows, const void* q, const void* k, const void* v,
                            void* q_out, void* k_out, void* v_out, void* stream);

/* ---------------------------------------------------------------------------
 * Window attention
 *
 * Query i of a sequence with q_len queries and kv_len keys has position
 * p = i + kv_len - q_len (the last query looks from the last key).  It sees
 * the keys j of the sequence with p - left <= j <= p + right, and of the first
 * `sinks` keys those with j <= p + right as well:
 *     O = softmax(scale * Q K^T over the visible keys) V.
 * A query that sees no key gets O = 0 and LSE = -inf.  heads is a multiple of
 * kv_heads; query head h reads key head h / (heads / kv_heads).  The token
 * strides of K and V, and in the backward pass of Q and dout, are below 2^23
 * elements where there is more than one token.
 */
typedef struct {
  int32_t batch, heads, kv_heads, seq_q, seq_kv, head_dim, dtype;
  int32_t left, right; /* keys before and after the position; -1: all of them */
  int32_t sinks;       /* first keys that stay visible */
  float scale;         /* 0: 1 / sqrt(head_dim) */
  int32_t reserved;    /* 0 */
  int64_t q_stride[3], k_stride[3], v_stride[3], o_stride[3]; /* (batch, head, token), elements */
} bsa_window_shapes;

/* Strides of the backward pass's tensors, laid out like Q (dout, dq) and K
 * (dk, dv). */
typedef struct {
  int64_t do_stride[3], dq_stride[3], dk_stride[3], dv_stride[3];
} bsa_window_grads;

/* Bytes of device workspace that a forward (backward == 0) or backward call of
 * these shapes needs; 0 means none.  Host only. */
BSA_API bsa_status bsa_window_workspace(const bsa_window_shapes* shapes, int32_t backward, size_t* bytes);

/*
 * O and LSE.  One entry point for every number of queries: prompts, drafted
 * tokens, single tokens over a long cache.
 *   q_len, kv_len  device int32 [batch] or NULL (seq_q, seq_kv): lengths of
 *                  each sequence, taken as 0 below 0 and as seq_q or seq_kv
 *                  above it.  Keys from kv_len on are not read; O and LSE rows
 *                  from q_len on keep what they held.
 *   lse            float32 [batch, heads, seq_q] or NULL: natural-log
 *                  log-sum-exp of the scaled scores.
 *   workspace      device memory of bsa_window_workspace's size (NULL when that
 *                  is 0), 16-byte aligned, used until the call's work is done;
 *                  calls that overlap in time need workspaces of their own.
 * dtype bf16 or f16, head_dim 64 or 128.  batch, seq_q and seq_kv may be 0.
 * Probabilities are rounded to the tensors' type for their product with V; their
 * sum, the maximum and O are 32 bits (O before its division by the sum: values
 * of V of 2^127 / (256 kv_len) and more may overflow it).  Values of K and V
 * that are not finite reach the queries that see them and no others.  (Rows that
 * meet such a value of V are formed a second time: up to twelve times the time
 * of the call, if they are all of them.)  Results do not depend on the order in
 * which workgroups run.
 */
BSA_API bsa_status bsa_window_forward(const bsa_window_shapes* shapes, const void* q, const void* k, const void* v,
                                      void* o, float* lse, const int32_t* q_len, const int32_t* kv_len,
                                      void* workspace, size_t workspace_bytes, void* stream);

/*
 * Gradients of Q, K and V from dout, the gradient of O; o and lse are what
 * bsa_window_forward gave for the same q, k, v, lengths and shapes.  The
 * gradient of a key head that several query heads share is their sum.  Rows of
 * dq from q_len on and of dk and dv from kv_len on keep what they held; keys
 * that no query sees get 0.  Sums are taken in a fixed order (no atomics).
 * Probabilities and the scores' gradients are rounded to the tensors' type for
 * their products; float16 holds the latter to 2^-25 below 2^-14, so the loss is
 * scaled where they are smaller.  What the rows behind a sequence's end and the
 * keys that no query sees hold does not affect results, but a value that is not
 * finite anywhere else may reach the gradients of neighbouring rows and keys that
 * it is not visible to.
 */
BSA_API bsa_status bsa_window_backward(const bsa_window_shapes* shapes, const bsa_window_grads* grads, const void* q,
                                       const void* k, const void* v, const void* o, const float* lse,
                                       const void* dout, void* dq, void* dk, void* dv, const int32_t* q_len,
                                       const int32_t* kv_len, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* BSA_OPS_H_ */
