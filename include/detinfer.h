/*
 * libdetinfer -- deterministic, batch-invariant transformer decode step for AMD MI355X (gfx950).
 *
 * Every entry point is a pure function of its input bytes and shape arguments: the output bytes
 * never depend on the stream, the launch order, what else runs on the device, the contents of a
 * workspace before the call, or on the batch size (row i of an output is the same whether the call
 * carries 1 row or 256, and whatever the other rows hold).  This is the contract of the paper's
 * section 6.1 (inference as a pure function whose honest re-executions are bit-identical) carried
 * by the three kernel invariants of its section 6.5: a fixed mapping of workgroups to output tiles
 * with no communication between workgroups, canonical stride-halving tree reductions, and no
 * floating-point atomics.
 *
 * Conventions
 *   - Plain C ABI.  All pointers are DEVICE pointers unless a comment says "host".
 *   - The caller owns every buffer.  The library allocates nothing and only enqueues work on the
 *     caller's HIP stream (`stream` is a hipStream_t passed as void*; NULL is the default stream).
 *     No call synchronises; results are ready when the stream reaches them.
 *   - bf16 tensors are arrays of 16-bit patterns (upper half of an IEEE fp32), row-major.
 *   - Workspaces need no initialisation: kernels overwrite whatever they later read.
 *   - Every call returns DET_OK or an error code below and launches nothing on error.  After
 *     DET_EHIP, det_last_hip_error() returns the hipError_t value seen by the calling thread.
 *   - Pointers must be 16-byte aligned (DET_EALIGN otherwise).
 *   - The library keeps no state between calls, with three exceptions that never reach an output byte:
 *     the per-thread last HIP error; the per-device address of the fixed scratch array of
 *     det_attn_decode_static (looked up once); and det_sha256_force_portable(), a process-wide switch
 *     for tests that selects between two implementations of the same hash.
 */
#ifndef DETINFER_H
#define DETINFER_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define DET_OK 0
#define DET_EINVAL 1     /* null pointer, non-positive size, bad enum */
#define DET_ESHAPE 2     /* shape outside what the kernels support (see each call) */
#define DET_EALIGN 3     /* pointer or leading dimension not 16-byte aligned */
#define DET_EWORKSPACE 4 /* workspace smaller than the matching *_workspace_bytes() */
#define DET_EHIP 5       /* a HIP runtime call failed */

#define DET_BF16 0
#define DET_F32 1

/* ---------------------------------------------------------------------------------------------
 * Deterministic GEMM (section 6.5: custom GEMM kernels; invariants 1 and 3).
 *
 *   C[i][j] = sum_k A[i][k] * B[k][j],  bf16 inputs, fp32 accumulation, output rounded once to
 *   bf16 (nearest even) or left in fp32.
 *
 * Each output element has ONE fp32 accumulator that starts at +0 and takes K/32 matrix-core steps
 * in ascending order; step t adds the 32 products of a fixed set of k indices (k in
 * [64*(t/2), 64*(t/2)+64), see det_gemm_pack_b).  There is no split of K across workgroups or
 * waves and there are no atomics.
 *
 * What depends on (N, K) only: the packing, the matrix-core instruction, the K staging and the order
 * of the steps, i.e. everything that enters an element's arithmetic.  What det_gemm_bf16 (and the
 * fused forms below) ALSO choose from M is the tile a launch cuts C into, i.e. which workgroup and wave
 * computes an element: 256 rows x the packing's width by default; rows cut into shorter tiles, in half blocks of 8,
 * when N alone gives fewer than 256 workgroups and M >= 17; 64-column tiles, where they move clearly fewer bytes, from
 * M >= 65 (16-column packings) or, 32-column packings, from M >= 64 in tiles of at most 64 rows and from M >= 161 in any,
 * up to M = 95 and M = 191 only where few of the eight XCDs read each weight; 128-column tiles when ceil(M/256) * N/128 >= 256;
 * 256-column tiles of 128 to 256 rows when M >= 256, K >= 1024, N % 256 == 0 and their rounds of 256 workgroups cost less
 * (det_gemm_tile gives the tile of a launch).  The bytes of a
 * row do not depend on that choice (every tile shape runs the same chain for an element; the tests
 * compare every M in 1..256 with the M = 256 launch and with det_gemm_bf16_fixed_tile), but it IS a
 * launch geometry keyed on the batch size, so it is named here and in det_fingerprint(), and
 * det_gemm_bf16_fixed_tile below is the form without it.
 *
 *   A        [M, K] bf16, row stride lda elements (lda >= K, lda % 8 == 0)
 *   B_packed output of det_gemm_pack_b for the same (N, K)
 *   C        [M, N] bf16 (out_dtype DET_BF16) or fp32 (DET_F32), row stride ldc elements
 *            (ldc >= N, ldc % 4 == 0)
 *   Shapes: M >= 1, N % 16 == 0, K % 64 == 0; DET_ESHAPE otherwise.
 */
int det_gemm_bf16(const void *A, int lda, const void *B_packed, void *C, int ldc, int M, int N,
                  int K, int out_dtype, void *stream);

/* det_gemm_bf16 with ONE tiling per (N, K) that never looks at M (section 6.5, invariant 1 read
 * strictly: a fixed workgroup -> tile mapping whatever the batch): 256-row tiles of the packing's
 * width, M only decides how many 16-row blocks of a tile hold data.  Same arguments, same bytes; slower
 * from about a hundred rows on (the benchmark reports both). */
int det_gemm_bf16_fixed_tile(const void *A, int lda, const void *B_packed, void *C, int ldc, int M, int N,
                             int K, int out_dtype, void *stream);

/* Test hook: rows of the 256-column tiles that det_gemm_bf16 and its fused forms cut a launch of M rows into (128, 160,
 * 192 or 256), 0 where they take another tiling. */
int det_gemm_wide_rows(int M, int N, int K);

/* Test hook: rows of the tiles that det_gemm_bf16 and its fused forms cut a launch of M rows into (0 if the shape is unsupported), and
 * their columns. */
int det_gemm_tile(int M, int N, int K, int *columns);

/* Bytes of the packed form of a [K, N] bf16 matrix (= 2*K*N). 0 if the shape is unsupported. */
size_t det_gemm_packed_b_bytes(int N, int K);

/* One-time, layout-only, bit-preserving repack of a row-major [K, N] bf16 weight matrix into the
 * order the GEMM kernel streams it: each workgroup's column slab becomes one contiguous run, cut
 * into 64-deep K stages already in matrix-core operand order.  B_kn and B_packed must not
 * overlap. */
int det_gemm_pack_b(const void *B_kn, void *B_packed, int N, int K, void *stream);

/* Fused epilogues of the same kernel; each produces exactly the bytes of the unfused sequence.
 *
 * det_gemm_bf16_residual: C = bf16( fp32(bf16(A B)) + fp32(R) ), i.e. det_gemm_bf16 (bf16 out)
 *   followed by det_residual_add.  R [M, N] bf16 with row stride ldr (ldr % 4 == 0); C may be R.
 * det_gemm_pack_gate_up: packs a [K, 2F] bf16 matrix whose columns are F gate columns followed by
 *   F up columns, with gate_j and up_j made neighbours, for det_gemm_swiglu_bf16.  F % 8 == 0.
 * det_gemm_swiglu_bf16: Y[M, F] = det_swiglu( g, u ) with [g | u] = det_gemm_bf16(A, [Wgate | Wup])
 *   rounded to bf16 first.  B_gate_up is the output of det_gemm_pack_gate_up; ldy >= F, ldy % 4 == 0.
 * det_gemm_pack_qkv: packs a [K, (Hq+2Hkv) D] bf16 matrix whose columns are Hq query heads, Hkv key
 *   heads and Hkv value heads of D = 128 columns each, with the columns d and d + D/2 of every head
 *   (a rotation pair of det_rope) made neighbours, for det_gemm_qkv_rope_append.
 * det_gemm_qkv_rope_append: the layer's fused projection.  With qkv = det_gemm_bf16(A, Wqkv) (bf16),
 *   row i at position p = positions[i] (clamped to 0..Lmax-1) and cache slot s = slots[i] (slots NULL:
 *   s = i): qbuf[i] = det_rope(query heads of qkv[i], p); kcache[s][:, p, :] = det_rope(key heads, p);
 *   vcache[s][:, p, :] = value heads.  Exactly the bytes of those three steps; qkv itself is never
 *   stored.  qbuf [M, Hq, D] bf16; caches [S, Hkv, Lmax, D] bf16; rope_cos/sin [Lmax, D/2] fp32,
 *   16-byte aligned; no two rows of one call may name the same (slot, position).  D must be 128.
 */
int det_gemm_bf16_residual(const void *A, int lda, const void *B_packed, const void *R, int ldr,
                           void *C, int ldc, int M, int N, int K, void *stream);
int det_gemm_pack_gate_up(const void *B_kn, void *B_packed, int F, int K, void *stream);
int det_gemm_swiglu_bf16(const void *A, int lda, const void *B_gate_up, void *Y, int ldy, int M,
                         int F, int K, void *stream);
/* The projections that follow an RMSNorm (two in the layer, the output head after the last layer), with the
 * norm in the same call:
 *   det_rmsnorm_gemm_qkv_rope_append(x, ...) = det_gemm_qkv_rope_append(det_rmsnorm(x, w_norm, eps), ...)
 *   det_rmsnorm_gemm_swiglu_bf16(x, ...)     = det_gemm_swiglu_bf16(det_rmsnorm(x, w_norm, eps), ...)
 *   det_rmsnorm_gemm_bf16(x, ...)            = det_gemm_bf16(det_rmsnorm(x, w_norm, eps), ...)
 * byte for byte.  x [M, K] bf16 raw rows with row stride ldx; w_norm [K] bf16; h [M, K] bf16 scratch that
 * the call may or may not write (M <= 4 and K <= 4096: the GEMM's workgroups normalize the rows themselves,
 * one launch instead of two, and h is untouched; otherwise det_rmsnorm into h, then the GEMM, and ldx must
 * be K).  Other arguments and errors as the two GEMM calls. */
int det_rmsnorm_gemm_qkv_rope_append(const void *x, int ldx, const void *w_norm, float eps,
                                     const void *B_qkv, void *h, void *qbuf, void *kcache, void *vcache,
                                     const int32_t *positions, const int32_t *slots,
                                     const float *rope_cos, const float *rope_sin, int M, int Hq,
                                     int Hkv, int D, int Lmax, int K, void *stream);
int det_rmsnorm_gemm_swiglu_bf16(const void *x, int ldx, const void *w_norm, float eps,
                                 const void *B_gate_up, void *h, void *Y, int ldy, int M, int F, int K,
                                 void *stream);
int det_rmsnorm_gemm_bf16(const void *x, int ldx, const void *w_norm, float eps, const void *B_packed,
                          void *h, void *C, int ldc, int M, int N, int K, int out_dtype, void *stream);
int det_gemm_pack_qkv(const void *B_kn, void *B_packed, int Hq, int Hkv, int D, int K, void *stream);
int det_gemm_qkv_rope_append(const void *A, int lda, const void *B_qkv, void *qbuf, void *kcache,
                             void *vcache, const int32_t *positions, const int32_t *slots,
                             const float *rope_cos, const float *rope_sin, int M, int Hq, int Hkv,
                             int D, int Lmax, int K, void *stream);

/* ---------------------------------------------------------------------------------------------
 * RMSNorm (section 6.5, invariant 2: canonical tree reduction; tree of Fig. "kernel_tree").
 *
 *   y[i][e] = bf16( (x[i][e] * r_i) * w[e] ),  r_i = 1 / sqrt( mean_e x[i][e]^2 + eps )
 *
 * Sum of squares: element e belongs to lane (e/8) mod 256; a lane folds its elements in ascending
 * e with fma(x, x, acc) from +0; the 256 lane sums are reduced by six stride-halving levels inside
 * each group of 64 lanes (offsets 32..1) and the four group sums as (q0+q2)+(q1+q3).  mean = ss/H;
 * divide and square root are correctly rounded fp32.
 *
 *   x, y [M, H] bf16 contiguous; w [H] bf16.  H % 8 == 0, H <= 16384.
 */
int det_rmsnorm(const void *x, const void *w, void *y, int M, int H, float eps, void *stream);

/* ---------------------------------------------------------------------------------------------
 * Single-query attention over a KV cache, grouped-query heads (the paper is silent on attention;
 * the reductions follow section 6.5's invariants).
 *
 * For sequence b and query head h (reading KV head h / (Hq/Hkv)), len = seqlens[b]:
 *   s_j = scale * (q . k_j), j < len, contraction on matrix cores with fp32 accumulation;
 *   chunk c = tokens [256c, min(256c+256, len)):  m_c = max s_j;  e_j = det_expf(s_j - m_c);
 *   l_c = tree-sum of e_j (same 256-leaf tree as RMSNorm, leaf = j - 256c);
 *   O_c[d] = sum_j e_j * v_jd on the matrix cores: e_j (fp32) is cut by truncation into three bf16 pieces
 *            with e_j = hi + mid + lo exactly, so every product piece * v is exact in fp32; one fp32
 *            accumulator per (head, d) from +0 takes the chunk's eight 32-token steps in ascending order,
 *            each step the hi, then the mid, then the lo products (tokens at or past len add +0);
 *   combine in ascending c:  m = max m_c;  w_c = det_expf(m_c - m);  L = sum w_c*l_c;
 *   O[d] = sum w_c*O_c[d];  out[d] = bf16(O[d] / L).
 * The number of chunks depends only on that sequence's length.  Cache contents at or past len are
 * never used.  len = 0 gives zeros.
 *
 *   q, out   [B, Hq, D] bf16
 *   kcache, vcache [B, Hkv, Lmax, D] bf16
 *   seqlens  [B] int32, 0 <= seqlens[b] <= Lmax (values above Lmax are clamped to Lmax)
 *   ws       det_attn_decode_workspace_bytes(B, Hq, D, Lmax) bytes.  After the call it holds the chunk
 *            partials, fp32, nc = ceil(Lmax/256): m_c [B, Hq, nc], then l_c [B, Hq, nc], then the
 *            unnormalised chunk outputs o_c [B, Hq, nc, D]; entries of chunks at or past the sequence's
 *            length are not written, and neither is the o_c of a sequence of at most 256 tokens: its
 *            single chunk is finished by the first pass with the operations the combination would
 *            apply to it (det_attn_decode_quant_q8 always takes the second pass).  (Tests read m_c and
 *            l_c there and compare them bit for bit with the reference statistics of the same scores.)
 *   Shapes: D == 128, Hq % Hkv == 0, Hq/Hkv in {1, 2, 4, 8}.
 */
size_t det_attn_decode_workspace_bytes(int B, int Hq, int D, int Lmax);
int det_attn_decode(const void *q, const void *kcache, const void *vcache, const int32_t *seqlens,
                    void *out, void *ws, size_t ws_bytes, int B, int Hq, int Hkv, int D, int Lmax,
                    float scale, void *stream);

/* The same operation on R rows that name their cache slot: row r reads slot slots[r] of caches
 * [S, Hkv, Lmax, D] with length seqlens[r].  Several rows may share a slot (the tokens of one prompt
 * at lengths 1..T: batch-invariant prefill, since each row is exactly the single-token operation).
 * 0 <= slots[r] < S is the caller's responsibility.  Workspace: det_attn_decode_workspace_bytes(R, ...); what it holds
 * after the call is as above for calls of fewer than 256 pairs (next sentence), and unspecified for larger ones, which
 * write the partials of some rows only.
 * From sixteen rows on, eight consecutive rows go to one workgroup, and those of them that name the same
 * slot share each 256-token chunk of K and V (causal prefill: one read of the prompt's cache per eight
 * query tokens instead of one per token); from 256 (KV head, tile of 64 / G rows) pairs on, G = Hq / Hkv, the
 * rows of a tile that name one slot go through all their chunks inside one workgroup, but for rows much longer than the
 * call's others.  Which rows share a workgroup changes no row's arithmetic. */
int det_attn_decode_rows(const void *q, const void *kcache, const void *vcache, const int32_t *seqlens,
                         const int32_t *slots, void *out, void *ws, size_t ws_bytes, int R, int Hq,
                         int Hkv, int D, int Lmax, float scale, void *stream);

/* det_attn_decode for callers that cannot provide or allocate a workspace (code under HIP graph capture,
 * tight serving loops, harnesses that forbid allocation): the chunk partials live in a fixed array of
 * DET_ATTN_STATIC_WS_BYTES inside the library's code object, one copy per device, held until the
 * process ends.  The call allocates nothing (no hipMalloc / hipFree, no allocating library routine); its
 * first call on a device looks up that device's copy of the array (hipGetSymbolAddress), so the device
 * `stream` belongs to must be the current device.  Output bytes are those of det_attn_decode.
 *   Limit: det_attn_decode_workspace_bytes(B, Hq, D, Lmax) <= DET_ATTN_STATIC_WS_BYTES, i.e.
 *   B * Hq * ceil(Lmax/256) <= 64527; DET_EWORKSPACE beyond it (nothing is launched).
 *   All calls on one device share the array, which keeps the previous call's partials; nothing in it
 *   needs clearing (each call overwrites what it later reads), but two calls that overlap in time on
 *   one device (different streams) race on it: serialise them.
 *   Other arguments and errors as det_attn_decode. */
#define DET_ATTN_STATIC_WS_BYTES (32u << 20)
int det_attn_decode_static(const void *q, const void *kcache, const void *vcache, const int32_t *seqlens,
                           void *out, int B, int Hq, int Hkv, int D, int Lmax, float scale, void *stream);

/* Test hook: the softmax statistics of det_attn_decode on caller-provided fp32 scores.  The per-chunk
 * statistics (m_c, e_j, l_c) come from the device routine that the attention of eight rows a workgroup calls;
 * decode and calls of many rows compute them in the same order with code of their own, which the tests hold to those bytes.  The combination over chunks is the same ascending fold, written
 * for one row per workgroup.
 * s, p [R, Lmax] fp32; lens [R]; m_out, l_out [R] fp32.
 * p_j = (w_c * e_j) / L for j < lens[r]; entries at or past lens[r] are not written.
 * lens[r] = 0 gives m = -inf, L = 0.  Lmax <= 262144. */
int det_softmax_f32(const float *s, const int32_t *lens, float *p, float *m_out, float *l_out, int R,
                    int Lmax, void *stream);

/* ---------------------------------------------------------------------------------------------
 * Greedy sampling (section 6.6: deterministic decoding in a canonical iteration order).
 * idx[b] = smallest index attaining the maximum of row b; -0 equals +0; NaN never wins; a row of
 * NaNs gives 0.  logits [B, V] fp32 (DET_F32) or bf16 (DET_BF16); idx [B] int32. */
int det_argmax(const void *logits, int32_t *idx, int B, int V, int dtype, void *stream);

/* Seeded sampling (section 6.6: a fixed-seed PRNG and a canonical iteration order make the token a
 * function of (seed, decode policy)).  Per row:
 *   z_j = logits_j / temperature (NaN counts as -inf);  candidates ordered by (z descending, index
 *   ascending);  the first k = min(top_k, V) kept;  e_i = det_expf(z_i - z_0);  c_i = c_{i-1} + e_i in
 *   rank order (sequential fp32 adds from +0);  n = smallest i+1 with c_i >= top_p * c_{k-1};
 *   u = (splitmix64 output for seed + ((seq_id << 32 | step) + 1) * 0x9E3779B97F4A7C15) >> 40, scaled by
 *   2^-24;  target = u * c_{n-1};  token = candidate of the smallest rank i < n with c_i > target
 *   (rank n-1 if none).  top_k = 1 is det_argmax.
 * The sample depends on (seed, seq_ids[b], steps[b]) and row b's logits only, never on the batch.
 *   logits [B, V] fp32; seq_ids, steps, tokens [B] int32.
 *   temperature > 0, 0 < top_p <= 1 (DET_EINVAL otherwise); 1 <= top_k <= 1024 (DET_ESHAPE). */
int det_sample(const float *logits, int B, int V, float temperature, int top_k, float top_p,
               uint64_t seed, const int32_t *seq_ids, const int32_t *steps, int32_t *tokens,
               void *stream);

/* ---------------------------------------------------------------------------------------------
 * Rules on logits, between the output head and det_argmax, det_sample or det_softmax_f32 (section 6.6: the decode policy is part of what the token is a
 * function of).  Row b, token t, z = logits[b][t]; every step one rounded fp32 operation:
 *   t occurs in the row's history:  z = z > 0 ? z / repetition : z * repetition;
 *   c > 0 of its occurrences are generated ones (index generated_from[b] or behind):  z = (z - frequency * c) - presence;
 *   t has an entry in the row's biases:  z = z + its value (several entries: the last one);
 *   the bit of t in the row's mask is 0:  z = -inf.
 * A token that no rule reaches keeps its bits.  A row whose mask allows nothing is -inf throughout.  Of such a row det_argmax gives token 0 and det_sample, for
 * every seed, the last of its candidates, token min(top_k, V) - 1: both barred, and det_logits_advance takes the transition of whatever token it is given.  A
 * caller who cannot rule such a row out looks at the chosen token's mask.
 * det_logits_rules: device pointers; the part whose first pointer is NULL is left out.
 *   penalties [B, 3] fp32: repetition (> 0), frequency, presence.  history [n_history, ld_history] int32, of which row b has the first history_lens[b] ids
 *   (0..ld_history) of row history_rows[b] (NULL: b; outside 0..n_history-1: none); ids outside 0..V-1 are ignored; generated_from [B] or NULL (0).
 *   bias_begin [B + 1]: row b's entries are bias_begin[b] .. bias_begin[b+1]-1 of bias_tokens, bias_values [n_biases].
 *   masks [n_masks, mask_words]: bit t % 32 of word t / 32; mask_rows [B]: the row's mask (NULL: b; outside 0..n_masks-1: none).
 * logits, out [B, V] fp32 (DET_F32) or bf16 (DET_BF16: computed in fp32, rounded once) with row strides ld >= V in elements; out may be logits (with
 * its stride), else the two may not overlap, nor rows of the one lie between rows of the other.  16-byte aligned (rows need not be).  B <= 65535, V <= 2^30, 32 mask_words >= V;  ld_history and n_biases
 * at most 2^30. */
typedef struct det_logits_rules {
    const float *penalties;
    const int32_t *history;
    const int32_t *history_rows;
    const int32_t *history_lens;
    const int32_t *generated_from;
    const int32_t *bias_begin;
    const int32_t *bias_tokens;
    const float *bias_values;
    const uint32_t *masks;
    const int32_t *mask_rows;
    int32_t ld_history, n_history, n_biases, n_masks, mask_words;
} det_logits_rules;
int det_logits_process(const void *logits, int64_t ld_logits, void *out, int64_t ld_out, int dtype, int B, int V,
                       const det_logits_rules *rules /* host */, void *stream);

/* What the rules need of a step, on the device: history[b][lens_in[b]] = tokens[b] and lens_out[b] = lens_in[b] + 1 (a full row stays as it is;
 * history NULL: neither); states_out[b] = transitions[states_in[b]][class of tokens[b]], the class of a token token_class[token] (NULL: itself), -1 where
 * the state, the token, its class or the next state is none (transitions NULL: left out).  A state is the mask_rows entry of the next step.
 *   history [B, ld_history]; lens, states, tokens [B]; transitions [n_states, n_classes]; token_class [V], all int32.  lens_out may be lens_in, states_out
 *   states_in. */
int det_logits_advance(const int32_t *tokens, int32_t *history, int ld_history, const int32_t *lens_in,
                       int32_t *lens_out, const int32_t *transitions, int n_states, int n_classes,
                       const int32_t *token_class, int V, const int32_t *states_in, int32_t *states_out, int B,
                       void *stream);

/* ---------------------------------------------------------------------------------------------
 * Elementwise steps of the decoder layer, exported so each can be checked bit for bit.
 *
 * det_rope: rotary embedding, rotate-half pairing (i, i + D/2), on nh heads of one token per row.
 *   y_lo = bf16( fma(-x_hi, sin, x_lo*cos) ),  y_hi = bf16( fma(x_lo, sin, x_hi*cos) )
 *   x, y [R, nh, D] bf16 (row stride ldx / ldy elements); pos [R] int32 (< Lmax);
 *   cos_t, sin_t [Lmax, D/2] fp32 built by the caller.  D == 128.
 * det_swiglu: y = bf16( (g / (1 + det_expf(-g))) * u ); g, u, y [R, F] bf16 with row strides.
 * det_residual_add: z = bf16( fp32(x) + fp32(y) ), n elements, n % 8 == 0; z may alias x.
 */
int det_rope(const void *x, int ldx, void *y, int ldy, const int32_t *pos, const float *cos_t,
             const float *sin_t, int R, int nh, int D, int Lmax, void *stream);
int det_swiglu(const void *g, int ldg, const void *u, int ldu, void *y, int ldy, int R, int F,
               void *stream);
int det_residual_add(const void *x, const void *y, void *z, int64_t n, void *stream);

/* out[b][:] = table[tokens[b]][:]  (exact copy).  table [V, H] bf16; tokens [B] int32 in [0, V);
 * out [B, H] bf16.  H % 8 == 0.  Out-of-range ids are clamped into [0, V). */
int det_embed_gather(const void *table, const int32_t *tokens, void *out, int B, int H, int V,
                     void *stream);

/* ---------------------------------------------------------------------------------------------
 * One Llama-style decoder layer on one new token per sequence.
 *
 *   h = rmsnorm(x, w_norm1);  [q|k|v] = h Wqkv;  q, k = rope(q, k) at positions[b];
 *   k, v are written into the caches at row positions[b];
 *   a = attn_decode(q, caches, len = positions[b] + 1);
 *   x = x + a Wo;  h = rmsnorm(x, w_norm2);  [g|u] = h Wgu;  m = swiglu(g, u);  x = x + m Wdown.
 *
 * Every step is the operation documented above (the residual adds and the SwiGLU run as fused GEMM
 * epilogues with the bytes of the unfused steps), so the layer inherits their invariance: row b
 * of x and sequence b's cache rows do not depend on B or on the other sequences.
 */
typedef struct det_layer_cfg {
    int32_t H;      /* hidden size */
    int32_t Hq;     /* query heads */
    int32_t Hkv;    /* KV heads */
    int32_t D;      /* head dim (128) */
    int32_t F;      /* MLP inner size */
    int32_t Lmax;   /* rows per (sequence, KV head) in the caches and in the rope tables */
    float eps;      /* RMSNorm epsilon */
    float scale;    /* attention score scale, normally (float)(1/sqrt(D)) */
} det_layer_cfg;

typedef struct det_layer_weights {
    const void *w_norm1; /* [H] bf16 */
    const void *wqkv;    /* [K=H, N=(Hq+2Hkv)D] (columns: q heads, k heads, v heads) packed by
                          * det_gemm_pack_qkv */
    const void *wo;      /* packed [K=Hq*D, N=H] */
    const void *w_norm2; /* [H] bf16 */
    const void *wgu;     /* [K=H, N=2F] (columns: gate, up) packed by det_gemm_pack_gate_up */
    const void *wdown;   /* packed [K=F, N=H] */
} det_layer_weights;

size_t det_decoder_layer_workspace_bytes(const det_layer_cfg *cfg /* host */, int B);

/* One decoder layer as a pure function of (weights, x, caches, positions): section 6.1's contract (an
 * honest re-execution reproduces the bytes) composed from the operations above, which is what lets a
 * verifier re-run a single layer of a disputed step (section 6.1, layer-granular re-execution).
 *   w, cfg      host structs holding device pointers / sizes
 *   x_inout     [B, H] bf16, updated in place
 *   kcache, vcache [B, Hkv, Lmax, D] bf16, row positions[b] of every KV head of sequence b written
 *   positions   [B] int32, 0 <= positions[b] < Lmax
 *   rope_cos, rope_sin [Lmax, D/2] fp32
 */
int det_decoder_layer(const det_layer_weights *w, const det_layer_cfg *cfg, void *x_inout,
                      void *kcache, void *vcache, const int32_t *positions, const float *rope_cos,
                      const float *rope_sin, void *ws, size_t ws_bytes, int B, void *stream);

/* The layer on R rows that name their cache slot (caches [S, Hkv, Lmax, D]): row r is one token at
 * position positions[r] of the sequence in slot slots[r].  All keys and values of the call are
 * written before any row attends, so the T tokens of a prompt can go through in one call (rows at
 * positions 0..T-1 of one slot): every row's bytes are those of feeding the tokens one call at a
 * time.  No two rows may name the same (slot, position).  Workspace:
 * det_decoder_layer_workspace_bytes(cfg, R). */
int det_decoder_layer_rows(const det_layer_weights *w, const det_layer_cfg *cfg, void *x_inout,
                           void *kcache, void *vcache, const int32_t *positions, const int32_t *slots,
                           const float *rope_cos, const float *rope_sin, void *ws, size_t ws_bytes,
                           int R, void *stream);

/* ---------------------------------------------------------------------------------------------
 * Token bookkeeping of the greedy decode loop, on the device so a step needs no host round trip.
 * For row b at step t:  tok = t < prompt_lens[b] ? prompts[b][t] : last_sampled[b];
 * tokens_out[b] = tok;  history[b][t] = tok;  positions_out[b] = t.
 *   prompts [B, Tp] int32; prompt_lens [B]; last_sampled [B] (the argmax of step t-1);
 *   history [B, Th] int32 with t < Th.
 */
int det_next_token(const int32_t *prompts, int Tp, const int32_t *prompt_lens,
                   const int32_t *last_sampled, int32_t *tokens_out, int32_t *positions_out,
                   int32_t *history, int Th, int t, int B, void *stream);

/* The same bookkeeping after a one-pass prefill, where every sequence sits at its own position (section
 * 6.6's loop with per-sequence step counters): tokens_out[b] = last_sampled[b];
 * positions_out[b] = base_positions[b] + j.  All arrays [B] int32; j >= 0. */
int det_decode_advance(const int32_t *last_sampled, const int32_t *base_positions, int j, int32_t *tokens_out,
                       int32_t *positions_out, int B, void *stream);

/* ---------------------------------------------------------------------------------------------
 * Deterministic block-quantized GEMM (the paper's primary kernel family is the quantized one, section
 * 6.4 and Table 5; it gives no format, so one is defined here).
 *
 *   weights, block = 64 consecutive k of one column:   amax = max|w|; s = bf16(amax / 7);
 *       q = clamp(rint(w / s), -8, 7), 0 if s == 0                      (4-bit code, bf16 scale)
 *   activations, block = 64 consecutive k of one row:  amax = max|a|; d = amax / 127 (fp32);
 *       p = clamp(rint(a / d), -127, 127), 0 if d == 0                  (8-bit code, fp32 scale)
 *   C[i][n] = bf16(acc) (or acc as fp32), acc = 0; for blocks b ascending:
 *       acc = fma( d[i][b] * s[b][n], (float)(sum over the block of p*q, int32), acc )
 *   All of it IEEE fp32 with round-to-nearest-even; the result is a pure function of the operand
 *   bytes and is reproduced bit for bit by a plain CPU implementation.  NaN/Inf inputs and blocks
 *   whose largest magnitude is denormal are unspecified.
 *
 * det_quant_pack_w4: one-time; B_kn is bf16 row-major [K,N]; `packed` (det_qgemm_packed_w_bytes
 * bytes, 16-byte aligned, 4.25 bits per weight) is in the kernel's streaming order.  N % 16 == 0,
 * K % 64 == 0, else DET_ESHAPE.  det_quant_unpack_w4 is a test hook: codes int8 [K,N] and scales bf16
 * [K/64,N] back out of a packed matrix.
 * det_quant_act_q8: A bf16 [M,K] with row stride lda -> codes (det_quant_act_codes_bytes: int8
 * [M,K]) and scales (det_quant_act_scales_bytes: fp32, block-major with row stride (M+3)&~3, so a
 * test reads scale (i, b) at scales[b * ((M+3)&~3) + i]); both 16-byte aligned.
 * det_qgemm_w4a8: C [M,N] with row stride ldc (ldc % 4 == 0), out_dtype DET_BF16 or DET_F32; codes and
 * scales as written by det_quant_act_q8 for the same M and K.  Device pointers; work is enqueued on
 * `stream`. */
size_t det_qgemm_packed_w_bytes(int N, int K);
int det_quant_pack_w4(const void *B_kn, void *packed, int N, int K, void *stream);
int det_quant_unpack_w4(const void *packed, void *codes, void *scales, int N, int K, void *stream);
size_t det_quant_act_codes_bytes(int M, int K);
size_t det_quant_act_scales_bytes(int M, int K);
int det_quant_act_q8(const void *A, int lda, void *codes, void *scales, int M, int K, void *stream);
int det_qgemm_w4a8(const void *codes, const void *scales, const void *packed_w, void *C, int ldc, int M,
                   int N, int K, int out_dtype, void *stream);

/* Test hook: rows of the tiles that det_qgemm_w4a8 and its fused forms cut a launch of M rows into (0 if the shape is unsupported), and
 * their columns. */
int det_qgemm_tile(int M, int N, int K, int *columns);

/* Fused forms for the quantized decoder layer; each gives the bytes of the unfused sequence.
 * det_quant_pack_w4_gate_up: det_quant_pack_w4 of a [K, 2F] matrix (F gate columns, then F up columns)
 *   with gate_j and up_j made neighbours, for det_qgemm_w4a8_swiglu.  F % 8 == 0.
 * det_qgemm_w4a8_residual: C = det_residual_add(R, det_qgemm_w4a8(...) as bf16); C may be R.  R bf16 [M,N]
 *   with row stride ldr (ldr % 4 == 0).
 * det_qgemm_w4a8_swiglu: Y[M,F] = det_swiglu(g, u), [g | u] = det_qgemm_w4a8 of the [K, 2F] matrix as bf16;
 *   packed_gate_up from det_quant_pack_w4_gate_up; ldy >= F, ldy % 4 == 0.
 * det_rmsnorm_quant_q8: det_quant_act_q8(det_rmsnorm(x, w)) without the bf16 round trip through memory:
 *   codes int8 [M,H] and scales as det_quant_act_q8 writes them for (M, K = H).  H % 64 == 0, H <= 16384. */
int det_quant_pack_w4_gate_up(const void *B_kn, void *packed, int F, int K, void *stream);
int det_qgemm_w4a8_residual(const void *codes, const void *scales, const void *packed_w, const void *R,
                            int ldr, void *C, int ldc, int M, int N, int K, void *stream);
int det_qgemm_w4a8_swiglu(const void *codes, const void *scales, const void *packed_gate_up, void *Y,
                          int ldy, int M, int F, int K, void *stream);
/* det_quant_pack_w4_qkv / det_qgemm_w4a8_qkv_rope_append: the quantized layer's fused projection, as
 *   det_gemm_pack_qkv / det_gemm_qkv_rope_append are the bf16 layer's: the packing makes the columns d
 *   and d + D/2 of every head neighbours (the quantizer's blocks run along K, so codes and scales are
 *   those of det_quant_pack_w4 in another column order), and the GEMM's epilogue rotates the query and
 *   key heads at the row's position and writes query heads to qbuf, key and value heads to the row's
 *   cache slot: the bytes of det_qgemm_w4a8 (bf16 out), det_rope and the append.  D must be 128. */
int det_quant_pack_w4_qkv(const void *B_kn, void *packed, int Hq, int Hkv, int D, int K, void *stream);
int det_qgemm_w4a8_qkv_rope_append(const void *codes, const void *scales, const void *packed_qkv,
                                   void *qbuf, void *kcache, void *vcache, const int32_t *positions,
                                   const int32_t *slots, const float *rope_cos, const float *rope_sin,
                                   int M, int Hq, int Hkv, int D, int Lmax, int K, void *stream);
int det_rmsnorm_quant_q8(const void *x, const void *w, void *codes, void *scales, int M, int H, float eps,
                         void *stream);
/* det_attn_decode_quant_q8: det_quant_act_q8 of the [R, Hq*D] output of det_attn_decode_rows (slots may be
 *   NULL: row r reads cache slot r, as det_attn_decode), written as codes int8 [R, Hq*D] and scales for
 *   (M = R, K = Hq*D); other arguments and errors as det_attn_decode_rows. */
/* det_qgemm_w4a8_swiglu_quant: det_quant_act_q8 of the [M, F] output of det_qgemm_w4a8_swiglu, written as codes_out
 *   int8 [M, F] and scales_out for (M, K = F), without the bf16 round trip.  Only where the kernel's tile
 *   is 128 packed columns wide (then a tile row is exactly one 64-output block):
 *   det_qgemm_w4a8_swiglu_quant_supported(F, K) != 0, else DET_ESHAPE; F % 64 == 0.  codes_out / scales_out
 *   must not be the input codes / scales. */
int det_qgemm_w4a8_swiglu_quant_supported(int F, int K);
int det_qgemm_w4a8_swiglu_quant(const void *codes, const void *scales, const void *packed_gate_up,
                                void *codes_out, void *scales_out, int M, int F, int K, void *stream);
int det_attn_decode_quant_q8(const void *q, const void *kcache, const void *vcache, const int32_t *seqlens,
                             const int32_t *slots, void *codes, void *scales, void *ws, size_t ws_bytes,
                             int R, int Hq, int Hkv, int D, int Lmax, float scale, void *stream);

/* The decoder layer with every projection block-quantized (the engine the paper measures runs
 * quantized models, section 6.4): the steps of det_decoder_layer in the same order, each projection
 * det_qgemm_w4a8 on the det_quant_act_q8 codes of the bf16 activations it would have taken.  Weights:
 * w_norm1, w_norm2 bf16 [H]; wqkv from det_quant_pack_w4_qkv; wo, wdown from det_quant_pack_w4; wgu from
 * det_quant_pack_w4_gate_up.  Other arguments as det_decoder_layer_rows; slots may be NULL (row r is
 * the sequence in cache slot r).  Same invariance: a row's bytes and its cache rows do not depend on
 * R or on the other rows.  Workspace: det_qdecoder_layer_workspace_bytes(cfg, R). */
size_t det_qdecoder_layer_workspace_bytes(const det_layer_cfg *cfg /* host */, int R);
int det_qdecoder_layer(const det_layer_weights *w, const det_layer_cfg *cfg, void *x_inout, void *kcache,
                       void *vcache, const int32_t *positions, const int32_t *slots,
                       const float *rope_cos, const float *rope_sin, void *ws, size_t ws_bytes, int R,
                       void *stream);

/* ---------------------------------------------------------------------------------------------
 * An 8-bit paged KV cache and attention over it (the paper is silent on the cache; the form keeps section 6.1's contract: a
 * token's codes are a function of its own row, never of later tokens, so a prompt in one pass and token by token, and a
 * sequence in whatever pages it lies, give the same bytes).
 *
 * A pool is [n_pages, Hkv] records of DET_KV8_RECORD bytes; a record holds DET_KV8_PAGE = 64 tokens of one KV head of D = 128:
 *     K codes [64][128] int8,  V codes [4][128][16] int8 (token 16 g + i, column d at [g][d][i]),  K scales [64] fp32,  V scales [64] fp32.
 * The scale's block is one token of one KV head:  amax = max|x|;  d = amax / 127 (fp32);  code = clamp(rint(x / d), -127, 127), 0 if
 * d == 0;  value = code * d.  A row with an infinity or NaN has codes 0 and the scale NaN.  Scales are what the append writes: NaN or from 0 to 2^90 (a
 * key beyond that may overflow a score), never negative.  page_table [n_slots, max_pages] int32 names the
 * page of tokens 64 i .. 64 i + 63 of a slot; an entry outside 0..n_pages-1 names none.  Pages may be shared between slots and may be
 * anywhere; what lies in them past a row's length is never used.
 *   Shapes: D == 128, max_pages <= DET_KV8_MAX_PAGES; pool 16-byte aligned. */
#define DET_KV8_PAGE 64
#define DET_KV8_RECORD 16896
#define DET_KV8_MAX_PAGES 131072
/* Bytes of a pool (of one layer); 0 if the shape is unsupported. */
size_t det_kv8_pool_bytes(int n_pages, int Hkv, int D);

/* The rows of a fused projection into the cache.  qkv [R, (Hq + 2 Hkv) D] bf16 with row stride ldqkv (ldqkv % 8 == 0): query heads, key
 * heads, value heads.  qbuf[r] = det_rope(query heads, positions[r]); the key heads, rotated and rounded to bf16 the same way, and the value
 * heads are quantized into position positions[r] of slot slots[r] (slots NULL: slot r).  rope_cos/sin [Lrope, D/2] fp32, 16-byte aligned;
 * the rotation clamps positions to 0..Lrope-1.  A row whose slot, position or page does not exist is written to qbuf only.  No two rows
 * of one call may name the same (slot, position), nor a page that slots share. */
int det_kv8_rope_append(const void *qkv, int ldqkv, void *qbuf, void *pool, const int32_t *page_table, int n_pages,
                        int n_slots, int max_pages, const int32_t *positions, const int32_t *slots, const float *rope_cos,
                        const float *rope_sin, int R, int Hq, int Hkv, int D, int Lrope, void *stream);

/* k, v [R, Hkv, D] bf16: the values (code * d, rounded once) of position positions[r] of slot slots[r] (NULL: slot r); zeros where there
 * is no such page. */
int det_kv8_read(const void *pool, const int32_t *page_table, int n_pages, int n_slots, int max_pages,
                 const int32_t *positions, const int32_t *slots, void *k, void *v, int R, int Hkv, int D, void *stream);

/* Page dst[i] = page src[i] in every layer of pools [n_layers, n_pages, Hkv] that lie one behind the other, i < n.  A page may be
 * the source of several copies; no page may be the destination of two, nor of one and a source.  Pairs that name a page outside
 * 0..n_pages-1 are left out. */
int det_kv8_copy_pages(void *pool, int n_layers, int n_pages, int Hkv, int D, const int32_t *src, const int32_t *dst, int n,
                       void *stream);

/* Attention of R rows over the cache: row r, query head h (KV head h / (Hq/Hkv)), the first len = seqlens[r] tokens (clamped to
 * 0..64 max_pages) of slot slots[r] (NULL: slot r; a slot outside 0..n_slots-1 has no tokens).  Tokens without a page are left out; a row
 * without any token gives zeros.  Several rows may share a slot (a prompt's rows at lengths 1..T, the rows of drafted tokens).
 *   s_j = scale * (q . c_j) d^K_j,   out = bf16( sum_j p_j d^V_j c^V_j ),   p = softmax(s).
 * The order: q's (row, head) as integers n_d = rint(q_d 2^(22-E)), 2^E the power of two above its largest magnitude (E >= -100); n . c_j exact, brought to
 * fp32 from its digits to base 256.  Chunk c = tokens [256 c, 256 c + 256): in units of log2, m_c = ceil(max s_j), e_j = 2^(s_j - m_c) by the
 * hardware's exponential (the last product of s_j in one fma with the difference; rounded before it where |m_c| >= 2^24), l_c their sum in a fixed
 * order; a row whose largest score passes fp32 is NaN; weights e_j d^V_j as integers rint(w 2^(22-E_c)), 2^E_c above the chunk's largest
 * (E_c >= -100: weights times scales below 2^-100 lose bits); their products with the codes exact.  Chunks are folded in ascending order, relative to
 * the largest m so far.  A row's bytes do not depend on R, on the other rows, on the pages it lies in or on the call's max_pages.
 * Up to 895 (tile, KV head) pairs, a tile being 16 / (Hq/Hkv) rows, and wherever slots is NULL, chunks go to workgroups of their own and meet in ws in a
 * second launch; beyond, a tile of rows that name slots walks its chunks in one launch.  Rows that name slots are best given slot by slot.
 *   q, out [R, Hq, D] bf16;  Hq % Hkv == 0, Hq/Hkv <= 16;  scale > 0 and finite;  R <= 65535 if slots is NULL;  ws: det_attn_decode_kv8_workspace_bytes bytes, or
 *   for rows that name slots det_attn_decode_kv8_rows_workspace_bytes: enough for a call of up to R such rows, and no more for thousands of them
 *   than for those 895 pairs (a call in one launch keeps nothing in ws and does not look at ws_bytes). */
size_t det_attn_decode_kv8_workspace_bytes(int R, int Hq, int Hkv, int D, int max_pages);
size_t det_attn_decode_kv8_rows_workspace_bytes(int R, int Hq, int Hkv, int D, int max_pages);
int det_attn_decode_kv8(const void *q, const void *pool, const int32_t *page_table, int n_pages, int n_slots,
                        int max_pages, const int32_t *seqlens, const int32_t *slots, void *out, void *ws, size_t ws_bytes,
                        int R, int Hq, int Hkv, int D, float scale, void *stream);

/* det_attn_decode_kv8 for rows whose first tokens lie in the same pages (continuations of a prompt, a document that all requests begin with): the
 * shared chunks are read once for a group of rows.  Group g: rows group_rows[g] .. group_rows[g+1]-1 (group_rows ascending; rows in no group are read for
 * themselves), which hold their first shared[g] tokens in the same pages; of these the whole chunks of 256 tokens are read through the table of the
 * group's first row, or, where that row has no slot or ends in front of their end, of the first that reaches it (of none: of the longest), whatever
 * the tables of its other rows of more than 256 tokens name there.  A row may be shorter than what its group shares.
 * Output bytes are those of det_attn_decode_kv8 (whose arguments, rules and errors hold; slots NULL or not), whatever the groups.
 *   group_rows [n_groups + 1], shared [n_groups] int32;  0 <= n_groups <= R (n_groups = 0: both may be NULL);  R <= 65535;
 *   DET_ESHAPE also for calls of 2^23 workgroups and more (from R Hkv = 2^22 on);
 *   ws: det_attn_decode_kv8_shared_workspace_bytes bytes. */
size_t det_attn_decode_kv8_shared_workspace_bytes(int R, int Hq, int Hkv, int D, int max_pages);
int det_attn_decode_kv8_shared(const void *q, const void *pool, const int32_t *page_table, int n_pages, int n_slots,
                               int max_pages, const int32_t *seqlens, const int32_t *slots, const int32_t *group_rows,
                               const int32_t *shared, int n_groups, void *out, void *ws, size_t ws_bytes, int R, int Hq,
                               int Hkv, int D, float scale, void *stream);

/* The same, and what weight each page of each slot got:
 *   weights_out[s][i] = weights_in[s][i] + sum over the rows r that name slot s, the heads h and the tokens j of page i (64 i .. 64 i + 63) of p[r][h][j],
 * p the softmax of row r and head h.  fp32, in a fixed order: of each row (ascending) the heads (ascending) into the sum h mod 8, these eight in order, then
 * onto weights_in.  A (row, head) whose softmax is not finite adds nothing.  Output bytes as above.
 *   weights_in, weights_out [n_slots, max_pages] fp32, every entry written; weights_in NULL: zeros; the two may be the same array.  n_slots <= 65535,
 *   and n_slots * ceil(max_pages / 64) + R Hq / 2 below 2^24 (DET_ESHAPE).
 *   ws: det_attn_decode_kv8_weights_workspace_bytes bytes. */
size_t det_attn_decode_kv8_weights_workspace_bytes(int R, int Hq, int Hkv, int D, int max_pages);
int det_attn_decode_kv8_weights(const void *q, const void *pool, const int32_t *page_table, int n_pages, int n_slots,
                                int max_pages, const int32_t *seqlens, const int32_t *slots, const int32_t *group_rows,
                                const int32_t *shared, int n_groups, const float *weights_in, float *weights_out,
                                void *out, void *ws, size_t ws_bytes, int R, int Hq, int Hkv, int D, float scale,
                                void *stream);

/* Which pages the slots give up, by the weights that det_attn_decode_kv8_weights added up.  Slot s has ceil(lengths[s] / 64) pages (at most max_pages;
 * none for a length below 1), of which those that its table names are there.  The first `first` and the last `recent` of them always stay.  Of the others
 * that are there the max(0, pages there - keep[s]) with the smallest weight go, as far as there are so many; of equal weights the first pages go;
 * a NaN is the smallest weight.  dropped[s][i] = 1 where page i goes, else 0 (every entry is written; the table is left as it is).
 *   weights [n_slots, max_pages] fp32; lengths, keep [n_slots] int32 (a negative keep counts 0); dropped [n_slots, max_pages] bytes;  first, recent >= 0. */
int det_kv8_pick_pages(const float *weights, const int32_t *page_table, int n_pages, int n_slots, int max_pages,
                       const int32_t *lengths, const int32_t *keep, int first, int recent, uint8_t *dropped,
                       void *stream);

/* The decoder layers on the 8-bit cache: the steps of det_decoder_layer_rows and det_qdecoder_layer in the same order, with qkv in bf16,
 * det_kv8_rope_append and det_attn_decode_kv8 in place of the fused projection and the attention over a bf16 cache (the quantized layer's attention
 * output goes through det_quant_act_q8).  slots may be NULL: row r is the sequence in slot r.
 * Weights: wqkv from det_gemm_pack_b (det_quant_pack_w4 for the quantized layer), columns query, key and value heads; the others as there.
 * cfg->Lmax: rows of the rope tables.  A row whose position has no page attends to what is there.  Same invariance: a row's bytes do not depend on R,
 * on the other rows or on where the pages lie, and T tokens of a prompt in one call are the T calls of one.
 * Workspace: *_kv8_workspace_bytes, or *_kv8_rows_workspace_bytes where slots is not NULL (enough for up to R rows). */
size_t det_decoder_layer_kv8_workspace_bytes(const det_layer_cfg *cfg /* host */, int R, int max_pages);
size_t det_decoder_layer_kv8_rows_workspace_bytes(const det_layer_cfg *cfg /* host */, int R, int max_pages);
int det_decoder_layer_kv8(const det_layer_weights *w, const det_layer_cfg *cfg, void *x_inout, void *pool,
                          const int32_t *page_table, int n_pages, int n_slots, int max_pages, const int32_t *positions,
                          const int32_t *slots, const float *rope_cos, const float *rope_sin, void *ws,
                          size_t ws_bytes, int R, void *stream);
size_t det_qdecoder_layer_kv8_workspace_bytes(const det_layer_cfg *cfg /* host */, int R, int max_pages);
size_t det_qdecoder_layer_kv8_rows_workspace_bytes(const det_layer_cfg *cfg /* host */, int R, int max_pages);
int det_qdecoder_layer_kv8(const det_layer_weights *w, const det_layer_cfg *cfg, void *x_inout, void *pool,
                           const int32_t *page_table, int n_pages, int n_slots, int max_pages, const int32_t *positions,
                           const int32_t *slots, const float *rope_cos, const float *rope_sin, void *ws,
                           size_t ws_bytes, int R, void *stream);

/* The same layers with det_attn_decode_kv8_shared or det_attn_decode_kv8_weights in the place of det_attn_decode_kv8: step (a host struct of device pointers)
 * says which rows share what, and where the pages' weights are added up, over rows, heads, layers and steps (NULL: nowhere).  step NULL, or without groups
 * and weights: the calls above.  A layer's bytes are the same whatever step says.  R <= 65535 with groups or weights.
 * Workspace: *_kv8_step_workspace_bytes(cfg, R, max_pages, weights), weights != 0 where step has some; without groups and weights that of the calls above. */
typedef struct det_kv8_step {
    const int32_t *group_rows; /* [n_groups + 1] */
    const int32_t *shared;     /* [n_groups] */
    float *weights;            /* [n_slots, max_pages], added to, or NULL */
    int32_t n_groups;
} det_kv8_step;
size_t det_decoder_layer_kv8_step_workspace_bytes(const det_layer_cfg *cfg /* host */, int R, int max_pages, int weights);
int det_decoder_layer_kv8_step(const det_layer_weights *w, const det_layer_cfg *cfg, void *x_inout, void *pool,
                               const int32_t *page_table, int n_pages, int n_slots, int max_pages,
                               const int32_t *positions, const int32_t *slots, const float *rope_cos,
                               const float *rope_sin, const det_kv8_step *step /* host */, void *ws, size_t ws_bytes,
                               int R, void *stream);
size_t det_qdecoder_layer_kv8_step_workspace_bytes(const det_layer_cfg *cfg /* host */, int R, int max_pages, int weights);
int det_qdecoder_layer_kv8_step(const det_layer_weights *w, const det_layer_cfg *cfg, void *x_inout, void *pool,
                                const int32_t *page_table, int n_pages, int n_slots, int max_pages,
                                const int32_t *positions, const int32_t *slots, const float *rope_cos,
                                const float *rope_sin, const det_kv8_step *step /* host */, void *ws, size_t ws_bytes,
                                int R, void *stream);

/* ---------------------------------------------------------------------------------------------
 * Verification of drafted tokens against the target's probabilities, from given random numbers (section 6.6: the tokens are a function of
 * what is given; nothing is drawn here).  For sequence b with n = n_drafts[b] drafts (n_drafts NULL: N; clamped to 0..N):
 *   draft i < n is accepted while all before it were and u[b][i] * q[b][i][x_i] < p[b][i][x_i], x_i = drafts[b][i] (decided exactly; an id
 *   outside 0..V-1 is rejected);  a = the number accepted = accepted[b];
 *   r_j = max(p[b][a][j] - q[b][a][j], 0) if a < n, else p[b][a][j];  where all r_j are 0, r_j = p[b][a][j] (NaN and negative values count 0);
 *   the token = smallest j with r_0 + .. + r_j > u[b][N] * sum r (the last j with r_j > 0 if none, 0 if there is none), fp64 sums.
 *   tokens[b] = x_0 .. x_{a-1}, the token, then -1.
 * q NULL: the drafts were certain (q = 1 at x_i, 0 elsewhere).
 *   p [B, N+1, V], q [B, N, V], u [B, N+1] fp32, u in [0, 1);  drafts [B, N], accepted [B], tokens [B, N+1] int32.  p, q 16-byte aligned.
 *   1 <= N <= 63, B <= 65535, V <= 2^30;  ws: det_verify_drafts_workspace_bytes(B, V) bytes, 16-byte aligned. */
size_t det_verify_drafts_workspace_bytes(int B, int V);
int det_verify_drafts(const float *p, const float *q, const int32_t *drafts, const int32_t *n_drafts, const float *u,
                      int32_t *accepted, int32_t *tokens, void *ws, size_t ws_bytes, int B, int N, int V, void *stream);

/* ---------------------------------------------------------------------------------------------
 * Output commitment (the paper's section 6.7 records SHA256(prompt || logits || tokens) for every
 * execution, and a receipt commits to the output by its hash, section 4.1).  HOST code on HOST
 * pointers: SHA-256 (FIPS 180-4) is a serial chain, so the caller copies what it wants committed
 * to host memory (per step, overlapped with the next step) and feeds it here.
 *
 * det_sha256_init / _update / _final: streaming interface; the context is caller-owned plain data
 * (no allocation); after _final the context is spent and must be re-initialised.  DET_EINVAL for
 * null pointers or a spent context.  det_commit_sha256: the three byte strings hashed in the
 * paper's order in one call; a length may be 0 (its pointer is then ignored).  The digest is the 32
 * bytes in the standard's order (big-endian words).  The bytes hashed are the caller's: this
 * library's convention (tests, decode loop) is int32 little-endian token ids and fp32 little-endian
 * logits, step-major. */
typedef struct det_sha256_ctx {
    uint32_t h[8];
    uint64_t nbytes;
    uint8_t buf[64];
    uint32_t fill;
} det_sha256_ctx;
int det_sha256_init(det_sha256_ctx *ctx);
int det_sha256_update(det_sha256_ctx *ctx, const void *data, size_t bytes);
int det_sha256_final(det_sha256_ctx *ctx, uint8_t digest[32]);
int det_commit_sha256(const void *prompt, size_t prompt_bytes, const void *logits, size_t logits_bytes,
                      const void *tokens, size_t tokens_bytes, uint8_t digest[32]);
/* Test hook: nonzero makes the calls above use the portable compression function even where the
 * CPU has SHA instructions (process-wide). */
int det_sha256_force_portable(int on);

/* Measurement aid (not part of the decode path): `workgroups` workgroups of 256 threads each stream the
 * buffer src (src_bytes, at most 1 GiB, every workgroup the same bytes, so that they come from L2) into
 * their LDS `iters` times 32 KB, path 0 through registers and LDS stores, path 1 with LDS-DMA loads.
 * Moves workgroups * iters * 32768 bytes; the caller times it.  sink: 4 bytes, never written in practice. */
int det_probe_lds_fill(const void *src, size_t src_bytes, int path, int workgroups, int iters, void *sink,
                       void *stream);

/* Build identification: target architecture, ROCm version the library was built with, and the
 * kernel-configuration revision (echoes the paper's `system_fingerprint` response field, section
 * 7.1).  Static storage; host pointer. */
const char *det_fingerprint(void);

/* hipError_t value of the last failed HIP call on the calling thread (0 if none). */
int det_last_hip_error(void);

#ifdef __cplusplus
}
#endif
#endif /* DETINFER_H */
