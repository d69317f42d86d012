/*
 * skipffn.h - C ABI of the MI355X (gfx950) Skip-FFN block.
 *
 * The block is the feed-forward half of one decoder layer under Skip-Vision (its first half,
 * attention, is here too: skipffn_attn_*)
 * (Section 4.2 of the paper):
 *
 *     retained token :  h_out = h_attn + FFN(h_attn)
 *     skipped  token :  h_out = h_attn
 *
 * with FFN the pre-norm SwiGLU MLP of the paper's LLaMA-3-8B backbone
 * (Section 5.4; three C x M matrices, cf. the 3*N2*C*M term of Section 5.2 and
 * Table 1):  FFN(x) = W_down( silu(W_gate n(x)) * (W_up n(x)) ),
 * n(x) = x * rsqrt(mean(x^2) + eps) * gain.
 *
 * Conventions common to every call
 * --------------------------------
 *  - All tensor pointers are DEVICE pointers (HBM of the current HIP device)
 *    unless a parameter says "host".  Tensors are dense row-major.
 *  - bf16 tensors are passed as `const void*` / `void*` to 16-bit elements
 *    (the upper half of an IEEE binary32).  Accumulation is fp32.
 *  - T = tokens in the flattened (packed, unpadded) batch, R = retained rows,
 *    C = hidden size, I = intermediate size (the paper's M).
 *    C % 8 == 0, I % 8 == 0; every tensor pointer is 16-byte aligned.
 *  - Weights use the [out_features, in_features] layout: w_gate, w_up [I, C],
 *    w_down [C, I]  (y = x W^T).  No pre-packing.
 *  - skip_mask: one byte per token, non-zero = the token skips the FFN.
 *  - idx: ascending token indices of the retained rows (what skipffn_compact
 *    writes).  `R` is given by the host (R >= 0); or R = -1 and `num_retained`
 *    points at the device-side count written by skipffn_compact, in which case
 *    no host synchronisation happens and buffers must be sized for R = T.
 *  - Ownership: the caller owns every buffer.  The library allocates no
 *    device memory, keeps no pointer after a call returns, never synchronises
 *    the device and enqueues work only on `stream` (a hipStream_t passed as
 *    void*; NULL = the default stream).  Results are complete when the stream
 *    reaches the end of the enqueued work.
 *  - Every function returns a skipffn_status; 0 is success.  Argument errors
 *    are detected on the host before anything is enqueued.  Nothing aborts,
 *    throws or prints.
 */
#ifndef SKIPFFN_H
#define SKIPFFN_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum skipffn_status {
    SKIPFFN_OK = 0,
    SKIPFFN_EINVAL = 1,       /* null / misaligned pointer, negative size, R > T */
    SKIPFFN_ESHAPE = 2,       /* C or I not a multiple of 8, or a tensor >= 2 GiB */
    SKIPFFN_EWORKSPACE = 3,   /* workspace (or saved buffer) too small */
    SKIPFFN_EHIP = 4,         /* a HIP call failed; see skipffn_last_hip_error */
    SKIPFFN_EUNSUPPORTED = 5, /* unknown flag bit */
    SKIPFFN_EIDX = 6          /* SKIPFFN_FLAG_VALIDATE_IDX: idx is not strictly ascending inside [0, T) */
} skipffn_status;

/* flags (bitwise or) */
#define SKIPFFN_FLAG_DW_FP32        0x1u  /* backward: dw_* are float32, not bf16 */
#define SKIPFFN_FLAG_DW_ACCUMULATE  0x2u  /* backward: dw_* += instead of = */
#define SKIPFFN_FLAG_NO_RESIDUAL    0x4u  /* forward: retained rows get bf16(FFN(x)), not bf16(x + FFN(x)) - a debugging view */
#define SKIPFFN_FLAG_BALANCED_SPLIT  0x8u  /* use the balanced K split of the down / dXn GEMMs whenever it applies
                                             (by default a cost model picks between it, plain split-K and no split) */
#define SKIPFFN_FLAG_VALIDATE_IDX    0x10u /* forward / backward, debugging: check idx[0..R) on the device first (strictly
                                             ascending, inside [0, T)) and return SKIPFFN_EIDX, with nothing else
                                             enqueued, when it is not.  The ONE case in which a call waits for the
                                             stream (it reads the verdict back), so not for use under graph capture.
                                             Without the flag idx is trusted: a wrong entry is an out-of-bounds write. */
#define SKIPFFN_FLAG_ALL            0x1Fu  /* what forward / backward take */
#define SKIPFFN_FLAG_QK_NORM         0x20u /* qk_rope: an RMS norm of every head of q and k before the rotation */
#define SKIPFFN_FLAG_ROPE_PAIRS      0x40u /* qk_rope: columns 2 j and 2 j + 1 are rotated together, not j and j + rot / 2 */

/* ---- step 1: mask -> ascending retained indices -------------------------
 * Section 4.1 decides which visual tokens are retained; the block consumes
 * that partition.  Writes idx[0..R) = positions t with skip_mask[t] == 0 in
 * increasing t (entries beyond R are left untouched), *num_retained = R and,
 * if pos != NULL, pos[t] = compacted row of token t or -1 if skipped.
 *   skip_mask  u8  [T]  device, 16-byte aligned
 *   idx        i32 [T]  device OUT (capacity T)
 *   num_retained i32 [1] device OUT
 *   pos        i32 [T]  device OUT or NULL
 *   workspace  device scratch of at least skipffn_compact_workspace_bytes(T)
 * T == 0 is valid (writes *num_retained = 0).  Deterministic. */
size_t skipffn_compact_workspace_bytes(int64_t T);
int skipffn_compact(const uint8_t* skip_mask, int64_t T, int32_t* idx,
                    int32_t* num_retained, int32_t* pos,
                    void* workspace, size_t workspace_bytes, void* stream);

/* skipffn_compact for callers that cannot allocate device memory and so have no workspace to
 * hand over: code running under HIP graph capture, tight serving loops, harnesses that forbid
 * hipMalloc.  Same arguments, outputs and guarantees as skipffn_compact minus the workspace: the
 * few kilobytes of scratch the multi-block path needs (T above 262144) live in a 32 KB array
 * inside the library, one copy per GPU, held until the process ends.  The call allocates and
 * frees nothing.  T may be at most skipffn_compact_static_max_tokens() (2^28); a larger T returns
 * SKIPFFN_ESHAPE with nothing enqueued.  Every call on a GPU uses that GPU's one array: calls
 * that may overlap in time on the same GPU (different streams without ordering) race - give
 * those skipffn_compact with a workspace each. */
int64_t skipffn_compact_static_max_tokens(void);
int skipffn_compact_static(const uint8_t* skip_mask, int64_t T, int32_t* idx,
                           int32_t* num_retained, int32_t* pos, void* stream);

/* The same check as SKIPFFN_FLAG_VALIDATE_IDX, asynchronous (Section 4.2's retained set must be
 * a set of token positions: the block scatters through it).  Enqueues two small kernels that
 * write status[0] = 0 if idx[0..R) is strictly ascending and inside [0, T), else 1, and
 * status[1] = the first offending position (INT32_MAX if none).
 *   status  i32 [2] device OUT;  idx, R, num_retained as in the conventions.  No host wait. */
int skipffn_validate_idx(const int32_t* idx, int64_t R, const int32_t* num_retained, int64_t T,
                         int32_t* status, void* stream);

/* ---- steps 2-4: forward of the block (Section 4.2, both equations) --------
 *   hidden  bf16 [T, C]  input (h_attn)
 *   out     bf16 [T, C]  output; may be the same pointer as hidden (in place:
 *                        skipped rows are then not touched at all).  When
 *                        out != hidden, skipped rows are copied bit for bit.
 *                        Partial overlap is not allowed.
 *   idx, R, num_retained : see conventions
 *   rms_gain bf16 [C] or NULL (= all ones)
 *   w_gate, w_up bf16 [I, C]; w_down bf16 [C, I]
 *   saved   NULL, or a buffer of skipffn_saved_bytes(R_max, C, I) bytes that
 *           receives what backward needs (gathered input rows, normalised
 *           rows, 1/rms, gate, up and hidden activations, and row-contiguous copies of the
 *           normalised rows and of the hidden activations); required for
 *           training because an in-place forward overwrites its input.
 *   workspace: at least skipffn_forward_workspace_bytes(R_max, C, I, saved != NULL)
 * where R_max = R if R >= 0 else T.  The size queries never decrease as R_max grows, so
 * buffers sized once for a bound serve every call with fewer rows.
 * R == 0 or T == 0: no arithmetic (out-of-place: plain copy).
 * Results are deterministic: every reduction has a fixed order.  The GEMMs pick their tile
 * height and K split from the row bound of the call (R, or T when R = -1), C and I, so the
 * same data may round differently in the last bit under a different bound. */
size_t skipffn_saved_bytes(int64_t R_max, int64_t C, int64_t I);
size_t skipffn_forward_workspace_bytes(int64_t R_max, int64_t C, int64_t I, int has_saved);
int skipffn_forward(int64_t T, int64_t C, int64_t I, float eps,
                    const void* hidden, void* out,
                    const int32_t* idx, int64_t R, const int32_t* num_retained,
                    const void* rms_gain,
                    const void* w_gate, const void* w_up, const void* w_down,
                    void* saved, void* workspace, size_t workspace_bytes,
                    uint32_t flags, void* stream);

/* ---- step 5: backward over retained rows only -----------------------------
 * The paper applies the skip during supervised fine-tuning (Section 4.2), so
 * gradients flow through the FFN for retained tokens only; a skipped token has
 * an identity Jacobian through this block.
 *   grad_out    bf16 [T, C]  upstream gradient
 *   grad_hidden bf16 [T, C]  OUT; may alias grad_out (skipped rows untouched);
 *                            otherwise skipped rows are bit copies of grad_out
 *   saved       what the matching forward wrote (same R, C, I)
 *   dw_gate, dw_up [I, C]; dw_down [C, I]: bf16, overwritten, unless
 *       SKIPFFN_FLAG_DW_FP32 (float32) / SKIPFFN_FLAG_DW_ACCUMULATE (+=).
 *       With R == 0 they are zero-filled (or left as they are when
 *       accumulating).
 *   d_rms_gain  NULL, or float32 [C] OUT: gradient of the RMSNorm gain (of an all-ones gain
 *       when rms_gain is NULL), overwritten or += like dw_*; always float32.  It is summed
 *       over rows in a fixed order (deterministic).
 *   workspace: at least skipffn_backward_workspace_bytes(R_max, C, I) */
size_t skipffn_backward_workspace_bytes(int64_t R_max, int64_t C, int64_t I);
int skipffn_backward(int64_t T, int64_t C, int64_t I, float eps,
                     const void* grad_out, void* grad_hidden,
                     const int32_t* idx, int64_t R, const int32_t* num_retained,
                     const void* rms_gain,
                     const void* w_gate, const void* w_up, const void* w_down,
                     const void* saved,
                     void* dw_gate, void* dw_up, void* dw_down, void* d_rms_gain,
                     void* workspace, size_t workspace_bytes,
                     uint32_t flags, void* stream);

/* ---- skip KV-cache (Section 4.3, the set-difference equation) -------------
 * After prefill the key / value rows of FFN-skipped tokens are dropped:
 * dst[r, :] = src[idx[r], :] for r < R.  row_bytes % 16 == 0.
 *   src  [T, row_bytes] device;  dst [R, row_bytes] device OUT (no overlap) */
int skipffn_gather_rows(const void* src, void* dst, int64_t T, int64_t row_bytes,
                        const int32_t* idx, int64_t R, const int32_t* num_retained,
                        void* stream);

/* Whole-cache form of the same set difference: a cache holds n_slabs slabs (one per layer,
 * key/value, batch entry and head - whatever precedes the token axis in the caller's
 * layout), each [T, row_bytes]; slab s starts at src + s * src_slab_bytes.  For every slab
 *     dst[s][r, :] = src[s][idx[r], :]   for r < R,
 * slab s of dst starting at dst + s * dst_slab_bytes (dst_slab_bytes >= R_max * row_bytes,
 * so the compacted cache may keep the prefill capacity or be packed).  One launch for the
 * whole cache.  row_bytes, src_slab_bytes, dst_slab_bytes are multiples of 16; src and dst
 * must not overlap (compacting in place would race: row r is a source for an earlier
 * destination).  n_slabs == 0 or R == 0: nothing is done. */
int skipffn_kv_compact(const void* src, void* dst, int64_t n_slabs, int64_t T, int64_t row_bytes,
                       int64_t src_slab_bytes, int64_t dst_slab_bytes,
                       const int32_t* idx, int64_t R, const int32_t* num_retained, void* stream);

/* ---- adaptive summary layer (Section 4.2, the summary-token equation) ------------------
 *     x^s = softmax(X w^T)^T X
 * X [n, C] a set of visual tokens, w [1, C] the layer's weight, the softmax taken over the
 * n tokens: one summary row per token set.  A call handles S sets at once:
 *   hidden  bf16 [T, C]          token features
 *   tok     i32 [n_tok] device   token indices, the sets laid one after the other
 *   seg     i32 [S + 1] device   set s is tok[seg[s] .. seg[s+1]); sizes need not be known
 *                                on the host.  Entries of tok outside [0, T) and segment
 *                                bounds outside [0, n_tok] are ignored, never dereferenced.
 *   w       bf16 [C]
 *   out     bf16 [S, C] OUT      the summary tokens (an empty set gives a zero row)
 *   saved   NULL (inference) or skipffn_summary_saved_bytes(n_tok, S, C) bytes OUT:
 *           scores f32 [n_tok], log-sum-exp f32 [S], x^s in f32 [S, C]
 *   workspace: at least skipffn_summary_workspace_bytes(n_tok, S, C)
 * Backward, for L with dL/dx^s = grad_out bf16 [S, C]:
 *   grad_hidden bf16 [T, C] IN/OUT: row t of every listed token becomes
 *       bf16(grad_hidden[t] + p_t * grad_out[s] + ds_t * w), ds_t = p_t (grad_out[s] . X_t -
 *       grad_out[s] . x^s); rows not listed are not touched.  The sets must be disjoint.
 *   dw  f32 [C] OUT: sum_t ds_t X_t over all sets, overwritten, or += with
 *       SKIPFFN_FLAG_DW_ACCUMULATE (the only flag accepted); summed in a fixed order.
 * C % 8 == 0; pointers 16-byte aligned (tok, seg: 4-byte).  S == 0 or n_tok == 0: only the
 * zero rows / zero dw are written. */
size_t skipffn_summary_saved_bytes(int64_t n_tok, int64_t S, int64_t C);
size_t skipffn_summary_workspace_bytes(int64_t n_tok, int64_t S, int64_t C);
int skipffn_summary_forward(int64_t T, int64_t C, const void* hidden,
                            const int32_t* tok, const int32_t* seg, int64_t n_tok, int64_t S,
                            const void* w, void* out, void* saved,
                            void* workspace, size_t workspace_bytes, void* stream);
int skipffn_summary_backward(int64_t T, int64_t C, const void* hidden,
                             const int32_t* tok, const int32_t* seg, int64_t n_tok, int64_t S,
                             const void* w, const void* saved, const void* grad_out,
                             void* grad_hidden, void* dw,
                             void* workspace, size_t workspace_bytes, uint32_t flags, void* stream);

/* ---- retained-token selection (Section 4.1) --------------------------------------------
 * For a backbone without global / local views the paper retains, per sequence, the n visual
 * tokens most similar to the CLS token and skips the rest.  Similarity is the cosine of the
 * vision features; a token is retained iff fewer than n tokens of its sequence have a larger
 * similarity (equal similarities: the lower index first), so the mask is unique for the
 * float32 similarities computed, which are returned.
 *   features  bf16 [n_feat, Cv]  visual tokens of all sequences, packed
 *   cls       bf16 [B, Cv]       one CLS row per sequence
 *   seq_off   i32 [B + 1] device rows of sequence b: seq_off[b] .. seq_off[b+1]) (clamped to n_feat)
 *   n_keep / n_keep_dev          retained count n: one host value, or i32 [B] on the device
 *   mask      u8 [n_feat] OUT    0 = retained, 1 = skipped, in feature order
 *   sim       f32 [n_feat] OUT   the similarities (also the kernels' scratch: required)
 *   token_pos, skip_mask, T      optional pair: token_pos i32 [n_feat] gives each visual token's
 *       position in a flat token sequence of length T and skip_mask u8 [T] receives the same
 *       value there (other entries, e.g. text tokens, are not touched; positions outside
 *       [0, T) are ignored) - the mask skipffn_compact consumes, without a host round trip.
 * Cv % 8 == 0; features, cls 16-byte aligned. */
int skipffn_select_retained(const void* features, const void* cls, const int32_t* seq_off,
                            int64_t n_feat, int64_t B, int64_t Cv, int64_t n_keep,
                            const int32_t* n_keep_dev, uint8_t* mask, float* sim,
                            const int32_t* token_pos, uint8_t* skip_mask, int64_t T, void* stream);

/* ---- token merge (Section 4.1, the three steps) ----------------------------------------
 * Reduces each set of (local, skipped) visual tokens to k tokens: pairwise cosine
 * similarities and their average per token (over the other tokens of the set); the k tokens
 * of lowest average similarity are kept; every other token is merged into the kept token it
 * is most similar to.  A kept token becomes the plain mean of itself and the tokens merged
 * into it (the paper leaves the merge itself open).  Equal averages / similarities go to the
 * lower index; decisions are taken on the float32 values computed, which are returned.
 *   x         bf16 [n_tok, C]     tokens of all sets, set s = rows seg_host[s] .. seg_host[s+1])
 *   seg_host  i32 [S + 1] HOST    ascending, seg_host[0] >= 0; at most 4096 rows per set
 *   k                             tokens kept per set (<= 4096); a set of n <= k rows is kept whole
 *   out       bf16 [S, k, C] OUT  merged tokens in the index order of the kept tokens; rows past
 *                                 a set's kept count are zero
 *   kept_idx  i32 [S, k] OUT      row index (in x) of every kept token, -1 padding
 *   assign    i32 [n_tok] OUT     slot (0 .. k-1 within its set) each token ends up in
 *   avg_sim   f32 [n_tok] OUT     the average similarities
 *   workspace: at least skipffn_token_merge_workspace_bytes(n_tok, n_max, C), n_max = rows of
 *              the largest set (it does not change the size)
 * Sets are processed in groups of even size, up to 64 per launch, in order on the stream. */
size_t skipffn_token_merge_workspace_bytes(int64_t n_tok, int64_t n_max, int64_t C);
int skipffn_token_merge(const void* x, const int32_t* seg_host, int64_t S, int64_t C, int64_t k,
                        void* out, int32_t* kept_idx, int32_t* assign, float* avg_sim,
                        void* workspace, size_t workspace_bytes, void* stream);

/* Gradient of the token merge with respect to x (Section 4.1; the merged tokens feed the
 * language model during training).  Which tokens are kept and where a token goes are piecewise
 * constant in x and carry no gradient; a kept slot is the mean of its m members, so every
 * member receives grad_out[slot] / m, rounded once to bf16.
 *   grad_out  bf16 [S, k, C]      gradient of `out` (rows past a set's kept count are ignored)
 *   seg_host, S, C, k             as in the forward call
 *   assign    i32 [n_tok]         the forward call's output; a value outside 0 .. min(k, n)-1
 *                                 gives a zero row
 *   grad_x    bf16 [n_tok, C] OUT every row is written
 * No workspace. */
int skipffn_token_merge_backward(const void* grad_out, const int32_t* seg_host, int64_t S, int64_t C,
                                 int64_t k, const int32_t* assign, void* grad_x, void* stream);

/* ---- attention over whole prompts (the first half of the decoder layer) -----------------
 * The block's input h_attn comes from attention, which every token takes part in, skipped ones
 * too (Section 4.2).  For every sequence of a packed batch and every query head
 *     out_i = sum_j P_ij v_j,   P_ij = softmax over j of (scale * q_i . k_j)
 * over the keys j that query i sees: all nk of its sequence, or with causal != 0 those with
 * j <= i + (nk - nq), i.e. the nq queries are the last of nk tokens (nk > nq: new tokens after a
 * cached beginning; nk < nq: the first nq - nk queries see nothing).  A query that sees no key
 * gives a zero row and zero gradients.  Query head h reads key/value head h / (Hq / Hkv).
 *   skipffn_heads  a bf16 tensor by token, head and column, element (t, h, d) at
 *                  data[t * token_stride + h * head_stride + d]: [T, H, D], a column range of the
 *                  projections' output [T, (Hq + 2 Hkv) D], or a cache [H, capacity, D].  Strides are
 *                  in elements, multiples of 8, not negative (0 repeats an input's rows or heads);
 *                  token_stride < 2^22.  data is 16-byte aligned.  The struct is read on the host
 *                  during the call.
 *   q [Tq, Hq, D], k and v [Tk, Hkv, D], out [Tq, Hq, D] OUT (memory of its own: what it spans meets none
 *                  of q, k, v; heads and rows of it are apart)
 *   seg_q, seg_k   i32 [n_seq + 1] device: sequence s has the queries seg_q[s] .. seg_q[s+1]) and the
 *                  keys seg_k[s] .. seg_k[s+1]); seg_k = NULL: the same as seg_q.  Lengths need not be
 *                  known on the host, may be 0; bounds are clamped to [0, Tq], [0, Tk].  Rows of out
 *                  that belong to no sequence are left as they were.
 *   scale          > 0, finite (1 / sqrt(D))
 *   saved          NULL (inference) or skipffn_attn_saved_bytes(Tq, Hq) bytes OUT (log-sum-exp, f32)
 *   workspace      at least skipffn_attn_forward_workspace_bytes(...) bytes (NULL where that is 0)
 * D % 8 == 0, 8 <= D <= 128, Hq a multiple of Hkv, n_seq <= 65535, (max(Tq, Tk) / 32 + 2 n_seq) Hq < 2^25.
 * Scores, softmax sums and products are accumulated in fp32; the weights P are rounded to bf16 before they
 * meet v (the matrix cores' operand type).  Deterministic: every sum has a fixed order.
 * A k_j or v_j that is not finite reaches the queries that see key j, and no others: a score of minus infinity is a
 * weight of 0, and a query that sees keys, but such scores alone, is NaN.  Rows that belong to no sequence may hold anything.
 * The workspace is for the keys of few queries, which are cut into parts: ask for the sizes of the call (more
 * queries may need less), or for the largest answer of the calls to come.  As everywhere, calls that may
 * overlap in time need workspaces of their own. */
typedef struct skipffn_heads {
    void* data;
    int64_t token_stride, head_stride;
} skipffn_heads;
size_t skipffn_attn_saved_bytes(int64_t Tq, int64_t Hq);
size_t skipffn_attn_forward_workspace_bytes(int64_t Tq, int64_t Tk, int64_t n_seq, int64_t Hq, int64_t Hkv, int64_t D);
int skipffn_attn_forward(int64_t Tq, int64_t Tk, int64_t n_seq, int64_t Hq, int64_t Hkv, int64_t D,
                         const skipffn_heads* q, const skipffn_heads* k, const skipffn_heads* v,
                         const skipffn_heads* out, const int32_t* seg_q, const int32_t* seg_k,
                         int causal, float scale, void* saved,
                         void* workspace, size_t workspace_bytes, void* stream);

/* Gradients of the above for L with dL/dout = grad_out [Tq, Hq, D]: with dP_ij = grad_out_i . v_j and
 * dS_ij = P_ij (dP_ij - grad_out_i . out_i),
 *     grad_q_i = scale sum_j dS_ij k_j,  grad_k_j = scale sum_i dS_ij q_i,  grad_v_j = sum_i P_ij grad_out_i,
 * the last two summed over the query heads of a key/value head too (in fp32, rounded once).
 *   out, saved     what the forward call wrote for the same inputs
 *   grad_q [Tq, Hq, D], grad_k and grad_v [Tk, Hkv, D] OUT, overwritten; rows that belong to no sequence
 *                  are left as they were.  They may be column ranges of one tensor (no element
 *                  is shared); what they span meets none of the inputs.
 *   workspace      at least skipffn_attn_backward_workspace_bytes(...)
 * Shapes as above, and ((Tq / 32 + n_seq) (Hq / Hkv) / 4 + n_seq) Hkv < 2^24, (Tk / 128 + n_seq) Hkv < 2^24.
 * Deterministic.  What is not finite in one sequence may reach any gradient of that sequence, and none of another. */
size_t skipffn_attn_backward_workspace_bytes(int64_t Tq, int64_t Tk, int64_t n_seq, int64_t Hq, int64_t Hkv, int64_t D);
int skipffn_attn_backward(int64_t Tq, int64_t Tk, int64_t n_seq, int64_t Hq, int64_t Hkv, int64_t D,
                          const skipffn_heads* q, const skipffn_heads* k, const skipffn_heads* v,
                          const skipffn_heads* out, const skipffn_heads* grad_out,
                          const int32_t* seg_q, const int32_t* seg_k, int causal, float scale,
                          const void* saved, const skipffn_heads* grad_q, const skipffn_heads* grad_k,
                          const skipffn_heads* grad_v, void* workspace, size_t workspace_bytes, void* stream);

/* Attention of one new token a sequence over the cache that is left (Section 4.3): the rows of a prefix
 * that the sequences of a group share (several questions about one image), then each sequence's own rows
 * (its tokens so far, the new one's key and value among them).  The prefix is read once for the sequences that
 * fit one product (32 rows of query heads), not once a sequence.
 *   q, out [n_seq, Hq, D]     token = sequence; q's head_stride < 2^24
 *   prefix_k, prefix_v        [Tp, Hkv, D], e.g. one layer of what skipffn_kv_compact wrote: head_stride =
 *                             capacity * D.  Read only where n_groups > 0 and Tp > 0
 *   prefix_seg  i32 [n_groups + 1] device: group i has the prefix rows prefix_seg[i] .. prefix_seg[i+1])
 *   group_off   i32 [n_groups + 1] device, ascending from 0: group i has the sequences group_off[i] ..
 *                             group_off[i+1]); sequences from group_off[n_groups] on have no prefix.
 *                             n_groups == 0: no sequence has one (both may be NULL)
 *   suffix_k, suffix_v        [n_seq][suffix_capacity, Hkv, D], sequence s suffix_k_seq (suffix_v_seq) elements
 *                             after the one before it.  Not read where suffix_capacity == 0
 *   suffix_len  i32 [n_seq] device: own rows of every sequence (clamped to 0 .. suffix_capacity)
 * A sequence with no rows at all gives a zero row, one of nothing but scores of minus infinity NaN.  What is not finite
 * among a sequence's own rows reaches that sequence alone.  Types, scale and shapes as above, (n_seq + n_groups + 1) Hq < 2^24, strides by sequence < 2^36;
 * out may not meet q or the caches.  workspace: at least skipffn_attn_decode_workspace_bytes(...), which holds fp32 rows of the parts
 * that long caches are cut into.  The parts depend on the bounds of the call (Tp, suffix_capacity, n_groups),
 * not on the lengths on the device.  Deterministic. */
size_t skipffn_attn_decode_workspace_bytes(int64_t n_seq, int64_t n_groups, int64_t Hq, int64_t Hkv, int64_t D, int64_t Tp,
                                           int64_t suffix_capacity);
int skipffn_attn_decode(int64_t n_seq, int64_t n_groups, int64_t Hq, int64_t Hkv, int64_t D, int64_t Tp,
                        int64_t suffix_capacity, const skipffn_heads* q, const skipffn_heads* prefix_k,
                        const skipffn_heads* prefix_v, const int32_t* prefix_seg, const int32_t* group_off,
                        const skipffn_heads* suffix_k, const skipffn_heads* suffix_v, int64_t suffix_k_seq, int64_t suffix_v_seq,
                        const int32_t* suffix_len, const skipffn_heads* out, float scale,
                        void* workspace, size_t workspace_bytes, void* stream);

/* skipffn_attn_decode that also hands out what the rows of the cache receive (for evicting rows by it): with P the attention
 * weights of a sequence's token,
 *     prefix row t of a group:  w[h][t] = sum over the group's sequences and the query heads of h of P,
 *     own row t of a sequence:  w[h][t] = sum over the query heads of h of P.
 *   most_shared     most sequences that a group has (a bound that sizes the workspace).  Sequences of a group past the first most_shared
 *                   of it add nothing to its prefix's weights.  >= 1 where there is a prefix
 *   prefix_weights  f32 [Hkv, Tp] OUT, head h prefix_weights_head elements after the one before it; rows of no group left as they were.
 *                   Not read or written where n_groups == 0 or Tp == 0
 *   suffix_weights  f32 [n_seq, Hkv, suffix_capacity] OUT by strides of sequence and head (no element shared); rows past suffix_len are
 *                   left as they were.  Not read or written where suffix_capacity == 0
 * Both are overwritten, or += with SKIPFFN_FLAG_DW_ACCUMULATE (the only flag).  What they span does not meet, and no weight is an element of q, out, the
 * cache or the offsets and lengths, which other workgroups still read.  `out` has the bits that skipffn_attn_decode gives; all else as there.
 * A sequence whose row of `out` is NaN for its scores makes NaN of the weights of the rows it sees.  Deterministic.
 * Tp + 36 n_groups and suffix_capacity < 2^24 - 64, (Tp / 64 + 1 + n_groups + n_seq (suffix_capacity / 256 + 1)) Hkv + n_seq Hq / 4 < 2^24 - 1.
 * workspace: at least skipffn_attn_decode_weights_workspace_bytes(...): about 4 Hq (most_shared Tp + n_seq suffix_capacity) and what decode takes. */
size_t skipffn_attn_decode_weights_workspace_bytes(int64_t n_seq, int64_t n_groups, int64_t Hq, int64_t Hkv, int64_t D, int64_t Tp,
                                                   int64_t suffix_capacity, int64_t most_shared);
int skipffn_attn_decode_weights(int64_t n_seq, int64_t n_groups, int64_t Hq, int64_t Hkv, int64_t D, int64_t Tp, int64_t suffix_capacity,
                                const skipffn_heads* q, const skipffn_heads* prefix_k, const skipffn_heads* prefix_v,
                                const int32_t* prefix_seg, const int32_t* group_off, const skipffn_heads* suffix_k,
                                const skipffn_heads* suffix_v, int64_t suffix_k_seq, int64_t suffix_v_seq, const int32_t* suffix_len,
                                const skipffn_heads* out, float scale, int64_t most_shared, float* prefix_weights,
                                int64_t prefix_weights_head, float* suffix_weights, int64_t suffix_weights_seq,
                                int64_t suffix_weights_head, void* workspace, size_t workspace_bytes, uint32_t flags, void* stream);

/* ---- what the keys receive (for evicting cache rows by it) ------------------------------
 * For every key j and key/value head the attention weights that its queries give it,
 *     w[h][j] = sum over the query heads of h and over the queries i that count of P_ij,   P as in skipffn_attn_forward,
 * computed from the log-sum-exp that it saved (one product, no values).
 *   q, k, seg_q, seg_k, causal, scale   what skipffn_attn_forward was given; any Tq, Tk, strides it takes
 *   saved     what that call wrote: f32 [Hq, Tq], the base-2 logarithm of a row's sum of 2^(scale log2(e) q . k)
 *             (+infinity: the row sees no key).  Not read where no query counts
 *   last      queries that count: the last so many of every sequence; < 0: all
 *   weights   f32 [Hkv, Tk] OUT, head h weights_head (>= Tk) elements after the one before it: overwritten, or += with
 *             SKIPFFN_FLAG_DW_ACCUMULATE (the only flag).  Keys that no query sees get 0; keys of no sequence are left as they were
 *   workspace at least skipffn_attn_key_weights_workspace_bytes(...) bytes (NULL where that is 0)
 * A query whose scores are not finite where it sees (its log-sum-exp is NaN or minus infinity) makes NaN of the keys it
 * sees, and of no others.  fp32 throughout.  What weights spans meets none of q, k and saved, no weight is an
 * element of seg_q or seg_k.  Shapes as skipffn_attn_forward, and
 * (Tk / 256 + n_seq) Hkv < 2^24.  Deterministic. */
size_t skipffn_attn_key_weights_workspace_bytes(int64_t Tq, int64_t Tk, int64_t n_seq, int64_t Hq, int64_t Hkv, int64_t D, int64_t last);
int skipffn_attn_key_weights(int64_t Tq, int64_t Tk, int64_t n_seq, int64_t Hq, int64_t Hkv, int64_t D, const skipffn_heads* q,
                             const skipffn_heads* k, const int32_t* seg_q, const int32_t* seg_k, int causal, float scale, const void* saved,
                             int64_t last, float* weights, int64_t weights_head, void* workspace, size_t workspace_bytes, uint32_t flags,
                             void* stream);

/* ---- eviction: a cache cut down to the rows that received most ---------------------------
 * Of every sequence and key/value head, each on its own, n_keep rows stay (all of them where there are no more): the `first` first and the `recent`
 * last rows before all others (by index where n_keep holds not even these), then by weight, the larger first; equal weights by index, a
 * NaN after every number.  Kept rows stay in their order.
 * packed != 0: rows of all sequences one after the other, as a prefix of skipffn_attn_decode:
 *   k, v [T, Hkv, D], weights f32 [Hkv, T]; seg i32 [n_seq + 1] device: sequence s has the rows seg[s] .. seg[s+1])
 *   k_out, v_out [T_out, Hkv, D] OUT, weights_out f32 and keep i32 [Hkv, T_out] OUT: sequence s has the rows seg_out[s] .. seg_out[s+1])
 *   of them; seg_out i32 [n_seq + 1] device OUT.  Kept rows past T_out are dropped: T, or the sum of the budgets, holds all
 * packed == 0: a capacity of rows for every sequence, as the own rows of skipffn_attn_decode:
 *   k, v [n_seq][T, Hkv, D], weights [n_seq][Hkv, T] by strides of sequence and head; seg i32 [n_seq] device: rows in use (clamped to 0 .. T)
 *   k_out, v_out [n_seq][T_out, Hkv, D], weights_out, keep [n_seq][Hkv, T_out] OUT; seg_out i32 [n_seq] device OUT: rows left, at most T_out
 *   n_keep / n_keep_dev  one host value, or i32 [n_seq] on the device
 *   weights_out     the kept rows' weights, or NULL
 *   keep            the kept rows' numbers, counted from their sequence's first row
 * Rows past a sequence's are left as they were, in every output.  Strides in elements; those of sequences are not read where packed.
 * What k_out and v_out span meets neither k nor v, and what keep, weights_out and seg_out span meets neither weights, seg nor n_keep_dev (kept rows, and
 * heads that still read, would race).  No element of an output is one of k, v or seg, or another output's.
 * Rows are copied bit for bit.  T, T_out < 2^30, n_seq Hkv < 2^22, workgroups of 16 kept rows of a head fewer than 2^24; D and strides of k, v as
 * in skipffn_attn_forward.  Deterministic. */
int skipffn_kv_evict(int64_t n_seq, int64_t Hkv, int64_t D, int64_t T, int64_t T_out, int packed, const skipffn_heads* k, const skipffn_heads* v,
                     int64_t k_seq, int64_t v_seq, const float* weights, int64_t weights_head, int64_t weights_seq, const int32_t* seg,
                     int64_t n_keep, const int32_t* n_keep_dev, int64_t first, int64_t recent, const skipffn_heads* k_out,
                     const skipffn_heads* v_out, int64_t k_out_seq, int64_t v_out_seq, float* weights_out, int64_t weights_out_head,
                     int64_t weights_out_seq, int32_t* keep, int64_t keep_head, int64_t keep_seq, int32_t* seg_out, void* stream);

/* ---- norm and rotation of queries and keys (between the projection and the attention) ------
 * For every token t and every head x of q and k, with n = x, or with SKIPFFN_FLAG_QK_NORM
 *     n = x * rsqrt(mean(x^2) + eps) * gain          (mean over the head's D columns; gain_q, gain_k bf16 [D] or NULL = ones),
 * the first `rot` columns are rotated in pairs by the angle A_j = pos[axis_j][t] * inv_freq[j], j < rot / 2,
 *     y_a = n_a cos A_j - n_b sin A_j,   y_b = n_a sin A_j + n_b cos A_j
 * with (a, b) = (j, j + rot / 2), or (2 j, 2 j + 1) with SKIPFFN_FLAG_ROPE_PAIRS; columns from rot on leave as n.  One axis of positions
 * is the place in the text; images have several (time, height, width), each with frequencies of its own.  The angle is the exact
 * product of the two numbers (taken in 64 bits), all else is fp32, rounded once to bf16.
 *   q [T, Hq, D], k, v [T, Hkv, D]      as skipffn_heads, e.g. column ranges of the projections' output; v and v_out: both or none
 *   pos       i32 [n_axes, T] device, any sign; inv_freq f32 [rot / 2] device (neither is read where rot == 0)
 *   axis      u8 [rot / 2] HOST, every one below n_axes, or NULL: axis 0 for all
 *   q_out [T, Hq, D]; k_out, v_out OUT: [T, Hkv, D], or with row != NULL the rows of a cache [rows_out, Hkv, D]:
 *   row       i32 [T] device: token t's key and value go to row row[t] of k_out and v_out, and nowhere if that is outside
 *             [0, rows_out) (a padded batch); rows that no token has are left as they were.  Two tokens with the same row: each 8 bytes
 *             of it come from one of them.  NULL: row t (rows_out is not read)
 * An output may be its own input (same memory and strides, row == NULL); training with a norm needs the inputs again, so not then.
 * Otherwise it shares no element with an input (positions, frequencies, rows and gains are read by all workgroups) or another output: what
 * heads span does not meet, or they are column ranges of rows of one stride.  v is copied bit for bit.
 * Own rows of skipffn_attn_decode, [n_seq, capacity, Hkv, D] or [Hkv, n_seq, capacity, D], are a cache of n_seq * capacity rows: a new
 * token's is sequence * capacity + own length.
 * D % 8 == 0, 8 <= D <= 128, rot % 8 == 0, 0 <= rot <= D, n_axes <= 4, T (Hq + 2 Hkv) < 2^27 (the forward call).  eps >= 0, finite. */
int skipffn_qk_rope_forward(int64_t T, int64_t Hq, int64_t Hkv, int64_t D, int64_t rot, int64_t n_axes, const skipffn_heads* q,
                            const skipffn_heads* k, const skipffn_heads* v, const int32_t* pos, const float* inv_freq, const uint8_t* axis,
                            const void* gain_q, const void* gain_k, float eps, const int32_t* row, int64_t rows_out,
                            const skipffn_heads* q_out, const skipffn_heads* k_out, const skipffn_heads* v_out, uint32_t flags, void* stream);

/* Gradients of the above (without `row`; the values' gradient passes by) for L with dL/dq_out = grad_q_out, dL/dk_out = grad_k_out: with
 * g the gradient rotated back and r = rsqrt(mean(x^2) + eps),
 *     d_gain = sum over tokens and heads of g x r,   grad_x = r (g gain - x r^2 mean(g gain x)),   or grad_x = g without the norm.
 *   q, k             what the forward call read; NULL (not read) without SKIPFFN_FLAG_QK_NORM
 *   grad_q, grad_k   OUT, as q and k; may be grad_q_out, grad_k_out themselves, else as the outputs above
 *   d_gain_q, d_gain_k  NULL, or f32 [D] OUT (with the norm; also where the gain is NULL), overwritten, or += with
 *                    SKIPFFN_FLAG_DW_ACCUMULATE.  Summed in a fixed order that depends on the sizes of the call.  Neither shares an
 *                    element with another output
 *   workspace        for gain gradients alone: at least skipffn_qk_rope_backward_workspace_bytes(...) */
size_t skipffn_qk_rope_backward_workspace_bytes(int64_t T, int64_t Hq, int64_t Hkv, int64_t D);
int skipffn_qk_rope_backward(int64_t T, int64_t Hq, int64_t Hkv, int64_t D, int64_t rot, int64_t n_axes, const skipffn_heads* q,
                             const skipffn_heads* k, const skipffn_heads* grad_q_out, const skipffn_heads* grad_k_out, const int32_t* pos,
                             const float* inv_freq, const uint8_t* axis, const void* gain_q, const void* gain_k, float eps,
                             const skipffn_heads* grad_q, const skipffn_heads* grad_k, float* d_gain_q, float* d_gain_k,
                             void* workspace, size_t workspace_bytes, uint32_t flags, void* stream);

/* ---- layout of `saved`, for tests that compare stage by stage -------------
 * Byte offsets of the sections inside a saved buffer for (R_max, C, I):
 * offsets[0] x rows bf16 [R, C]; [1] normalised rows bf16 [R, C];
 * [2] 1/rms f32 [R]; [3] gate bf16 [R, I]; [4] up bf16 [R, I];
 * [5] silu(gate)*up bf16 [R, I]; [6] normalised rows transposed, bf16 [C, ld];
 * [7] silu(gate)*up transposed, bf16 [I, ld]; ld = R_max rounded up to a multiple of 64
 * (the weight-gradient GEMMs contract over the rows and read the copies in which the row
 * index is contiguous; columns >= R are not read).
 * `offsets` is a HOST array of 8. */
int skipffn_saved_layout(int64_t R_max, int64_t C, int64_t I, size_t* offsets);

/* ---- diagnostics ---------------------------------------------------------- */
const char* skipffn_status_string(int status);
int skipffn_last_hip_error(void);     /* hipError_t of the last SKIPFFN_EHIP on this thread */
int skipffn_version(void);            /* major * 10000 + minor * 100 + patch */

/* Measurement aid, not part of the method: a register-only loop of independent
 * v_mfma_f32_16x16x32_bf16 (no memory traffic), i.e. what the matrix cores of the chip in hand
 * sustain - the ceiling bench.py quotes next to the published peak.  `blocks` workgroups of 4
 * wavefronts issue iters * 32 MFMAs per wavefront (16384 FLOP each); operands are the constant
 * 1.0 or, with random_operands != 0, pseudo-random bf16 values (the clock a power-capped chip
 * holds depends on the data).
 *   out     f32 [blocks * 256] device OUT (keeps the arithmetic alive)
 *   clocks  i64 [2 * blocks]  device OUT: per workgroup, shader cycles and 100 MHz wall-clock
 *           ticks spent in the loop (their ratio is the shader clock) */
int skipffn_probe_mfma(int64_t blocks, int64_t iters, int random_operands, float* out, int64_t* clocks,
                       void* stream);

/* Duration in milliseconds, measured with HIP events on `stream`, of the most
 * recent launch of each hot-path kernel class since the last
 * skipffn_profile_begin.  Profiling mode records events around every kernel
 * launch (it never synchronises inside a forward/backward call);
 * skipffn_profile_end synchronises those events and fills host arrays.
 *   names: host array of `cap` const char* (kernel class names, static storage)
 *   ms, launches: host arrays of `cap`;  returns the number of classes. */
int skipffn_profile_begin(void);
int skipffn_profile_end(const char** names, double* ms, int64_t* launches, int cap);

#ifdef __cplusplus
}
#endif
#endif /* SKIPFFN_H */
