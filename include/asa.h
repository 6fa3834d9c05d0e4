/*
 * libasa -- Adaptive Block-Sparse Attention (ASA) for AMD MI355X (gfx950).
 *
 * C ABI.  Plain pointers and sizes only.  Every tensor pointer is a DEVICE pointer
 * unless it says HOST.  The caller owns every buffer; the library allocates no device
 * memory, keeps no state between calls and only borrows pointers until the work it
 * enqueued on `hip_stream` has completed.  All calls are asynchronous on that stream
 * (0 / NULL = the default stream); the caller synchronises.
 *
 * Method: "BLADE: Block-Sparse Attention Meets Step Distillation for Efficient Video
 * Generation", Sec. 3.3 (Adaptive Block-Sparse Attention) and appendix "Pseudocode"
 * (Alg. 1 GetMaxPooledAttnMap, Alg. 2 Compute Block Importance Score, Alg. 3 ASA Mask
 * Generation).
 *
 * Layout.  Q, K, V, O, dO, dQ, dK, dV are bf16 tensors [B, H, L, d] with d contiguous.
 * Sequence positions are split into Nb = ceil(L / block) blocks of `block` tokens; the
 * last block may be partial.  A "slab" is one (batch, head) pair, slab index = b*H + h.
 *
 * Errors.  Every entry point returns ASA_OK (0) or a negative asa_status.  Arguments are
 * checked before anything is enqueued, so a failed call writes nothing.  No C++ exception
 * crosses this boundary.
 */
#ifndef ASA_H_
#define ASA_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define ASA_VERSION 100

typedef enum asa_status {
  ASA_OK = 0,
  ASA_ERR_INVALID_ARG = -1, /* null pointer, bad size, bad parameter, misaligned pointer */
  ASA_ERR_UNSUPPORTED = -2, /* (block, d) pair or size the kernels were not built for     */
  ASA_ERR_WORKSPACE = -3,   /* workspace missing or smaller than the *_workspace_bytes     */
  ASA_ERR_HIP = -4,         /* a HIP call failed; see asa_last_hip_error()                 */
  ASA_ERR_TOO_LARGE = -5    /* asa_attn_bwd_noalloc: the problem needs more scratch memory than
                               ASA_NOALLOC_SCRATCH_BYTES                                      */
} asa_status;

/*
 * Problem description shared by all entry points.
 *
 * Supported: d in {64, 128}; block in {64, 128}; 1 <= L; Nb = ceil(L/block) <= 1024;
 * 1 <= k_samples <= 16, or k_samples == block: every token sampled, the exact importance map
 * that Sec. 3.3 Step 1 defines and the sampling approximates (mask generation then costs as
 * much as dense attention scores and takes L <= 16 384).
 */
typedef struct asa_params {
  int32_t B, H, L, d;
  int32_t block;                 /* b of Sec. 3.3: query-block size == key-block size        */
  int32_t k_samples;             /* k of Alg. 2/3: sampled tokens per block (paper: 16)       */
  const int32_t *sample_offsets; /* HOST pointer to k strictly ascending offsets in [0, b),
                                    the same for every block, head, Q and K (the sampling of
                                    Alg. 3 step 3 is drawn by the caller); NULL selects the
                                    strided default u * (b / k).  Read during the call.      */
  float tau;                     /* cumulative-score threshold of Alg. 3 step 9              */
  float r_min, r_max;            /* minimum / maximum retention ratios of Alg. 3 step 9:
                                    m is clamped to [max(1, ceil(r_min*Nb)),
                                    max(that, floor(r_max*Nb))]; 0 <= r_min <= r_max <= 1     */
  int32_t n_prefix_dense;        /* tokens [0, n): every block holding one is always kept as
                                    a row and as a column (CogVideoX text tokens); 0 = none  */
  float scale;                   /* soft-max scale; 0 selects 1/sqrt(d)                      */
  /* Element strides of the B, H and L axes; d has stride 1.  All zero selects the packed
     layout {H*L*d, L*d, d}.  q_stride also applies to dQ, k_stride to dK, v_stride to dV,
     o_stride to dO.  Strides must be multiples of 8 elements (16-byte rows); the L stride
     must be below 2^24 elements (the kernels address the 64 rows of a tile with 32-bit
     byte offsets).  Anything else: ASA_ERR_INVALID_ARG.                                     */
  int64_t q_stride[3], k_stride[3], v_stride[3], o_stride[3];
} asa_params;

int asa_version(void);
const char *asa_error_string(int status); /* static string, never freed                     */
const char *asa_last_hip_error(void);     /* text of the last HIP failure on this thread    */

/* Workspace sizes in bytes for the calls below (256-byte aligned device memory).           */
size_t asa_mask_workspace_bytes(const asa_params *p);
size_t asa_fwd_workspace_bytes(const asa_params *p);
size_t asa_bwd_workspace_bytes(const asa_params *p);

/*
 * Mask generation (Sec. 3.3 Steps 1 and 2.1; Alg. 2 -> Alg. 1 -> Alg. 3 steps 6-11).
 *
 * From every block of Q and K the k sampled tokens are read; for each sampled query the
 * soft-max over ALL sampled keys of its slab is formed (online, Alg. 1) and max-pooled to
 * the block importance map P_imp [Nb, Nb] (fp32).  Each row of P_imp is then ranked by
 * (score descending, block index ascending); with c_r the fp64 running sum of the r best
 * scores and T the row total, m* = #{r : c_r < tau*T}; m = clamp(m*, m_min, m_max); the m
 * best blocks are kept.  Tokens past L take no part.  A NaN score counts as 0.  The
 * always-kept prefix rows/columns are OR-ed in afterwards.  Every row keeps >= 1 block.
 *
 * Outputs (all device):
 *   mask    [B*H, Nb, Nb] uint8, 1 = keep
 *   row_ptr [B*H, Nb+1]   int32, offsets into this slab's part of col_idx
 *   col_idx [B*H, Nb*Nb]  int32, kept key blocks of each row, ascending; entries past
 *                          row_ptr[Nb] of a slab are left untouched
 *   col_ptr, row_idx      the same mask by columns (for the backward pass); both NULL to skip
 *   p_imp   [B*H, Nb, Nb] fp32 importance map, or NULL
 * The workspace (asa_mask_workspace_bytes) is always needed: it holds the probe's per-row
 * block maxima and, when p_imp is NULL, the importance map.
 * P_imp and the mask of a slab are the same bits whatever other slabs are in the call.
 */
int asa_build_mask(const asa_params *p, const void *q, const void *k, uint8_t *mask,
                   int32_t *row_ptr, int32_t *col_idx, int32_t *col_ptr, int32_t *row_idx,
                   float *p_imp, void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * asa_build_mask with seeded random sampling (Alg. 3 step 2, "randomly sample k tokens from
 * each block", made reproducible): the sample_offsets of `p` are ignored; instead every block
 * of every (batch, head) slab draws its own k_samples positions with a counter-based generator.
 * Position j of block blk of slab s = batch * H + head gets the first word of Philox-4x32-10
 * (Salmon et al., SC'11) with counter (j, blk, s, 0) and key (seed low word, seed high word);
 * the k_samples positions with the smallest (word, j) are the sample, used in ascending order
 * for both Q and K.  asa_sample_offsets writes that table alone:
 *   table [B*H, Nb, k_samples] uint8 (DEVICE).
 * Workspace of the seeded build: asa_mask_seeded_workspace_bytes.
 */
size_t asa_mask_seeded_workspace_bytes(const asa_params *p);
int asa_build_mask_seeded(const asa_params *p, uint64_t seed, const void *q, const void *k,
                          uint8_t *mask, int32_t *row_ptr, int32_t *col_idx, int32_t *col_ptr,
                          int32_t *row_idx, float *p_imp, void *workspace, size_t workspace_bytes,
                          void *hip_stream);
int asa_sample_offsets(const asa_params *p, uint64_t seed, uint8_t *table, void *hip_stream);

/*
 * The selection rule alone (Alg. 3 steps 6-11) on caller-supplied scores
 * [B*H, Nb, Nb] fp32 -> mask [B*H, Nb, Nb] uint8 (prefix rows/columns included).
 */
int asa_mask_from_scores(const asa_params *p, const float *scores, uint8_t *mask,
                         void *hip_stream);

/* Index lists of a caller-supplied mask; same layouts as asa_build_mask.                   */
int asa_csr_from_mask(const asa_params *p, const uint8_t *mask, int32_t *row_ptr,
                      int32_t *col_idx, int32_t *col_ptr, int32_t *row_idx, void *hip_stream);

/*
 * Block-sparse attention forward (Sec. 3.3 Step 2.2, standard ASA).  Query block i attends
 * to the key blocks col_idx[row_ptr[i] .. row_ptr[i+1]) of its slab and to nothing else:
 *   S = scale * Q_i K_j^T (keys >= L excluded),  LSE = log sum exp S,  O = exp(S - LSE) V.
 * o    [B, H, L, d] bf16 (o_stride); rows >= L do not exist and nothing is written there
 * o_lo [B, H, L, d] bf16 (o_stride), optional (NULL to skip): the part of the fp32 result
 *      that rounding to bf16 dropped, o_lo = bf16(O_fp32 - o).  Saved for the backward pass,
 *      whose Delta = rowsum(dO * O) cancels against dO V^T in sharply peaked rows and needs
 *      more than the 8 significant bits of o there.
 * lse  [B*H, L] fp32, natural logarithm; a row with an empty list gets O = 0, LSE = -inf
 * bf16 products accumulate in fp32; probabilities are rounded to bf16 before P V.
 * Runs of a call repeat bit for bit.  Which kernel a call takes depends on its size (B, H, L) and
 * on the rule's parameters, and kernels add in different orders: the last bits of o and lse of a
 * slab may differ between calls that hold different numbers of slabs.  (The gradients of
 * asa_attn_bwd do not, for the same o and lse.)
 * row_ptr = col_idx = NULL selects the dense specialisation (every key block, no index
 * lists read): the dense attention of the first two sampling steps (Sec. 4.3) and the
 * in-house dense baseline of the kernel-speedup ratio (Table 2); exactly one of them NULL is
 * ASA_ERR_INVALID_ARG.
 */
int asa_attn_fwd(const asa_params *p, const void *q, const void *k, const void *v,
                 const int32_t *row_ptr, const int32_t *col_idx, void *o, void *o_lo, float *lse,
                 void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Block-sparse attention backward with the mask held constant (the mask restricts
 * attention "during both training and inference", Sec. 3.3 Step 2.1).  With
 * P = exp(S - LSE), Delta = rowsum(dO * O), dS = P * (dO V^T - Delta):
 *   dV = P^T dO,  dK = scale * dS^T Q,  dQ = scale * dS K     over the kept tiles only.
 * o, o_lo, lse are the forward's outputs; col_ptr/row_idx is the mask by columns.
 * o_lo may be NULL (the plain call): Delta is then not taken from o at all but formed as
 * sum_c P_c (dO V_c^T) over the kept tiles in fp32, by one more walk over the row lists before
 * the gradient kernels (two tile products; about a quarter more time at the Wan2.1 shape).
 * With o_lo, Delta = rowsum(dO * (o + o_lo)) costs one pass over three tensors.  Both meet the
 * same tolerance; Delta from the bf16 o alone would not where keys and queries are large.
 * dq, dk, dv [B, H, L, d] bf16 (q/k/v strides); every row < L is written.  dq may take the place
 * of q (the same strides), of d_o (if o has q's strides) or of o / o_lo, dk and dv that of o / o_lo
 * (if the strides agree); any other overlap of an output with an input or another output is undefined.
 * All four index-list pointers NULL selects the dense specialisation (see asa_attn_fwd);
 * some but not all NULL is ASA_ERR_INVALID_ARG.
 */
int asa_attn_bwd(const asa_params *p, const void *q, const void *k, const void *v, const void *o,
                 const void *o_lo, const void *d_o, const float *lse, const int32_t *row_ptr,
                 const int32_t *col_idx, const int32_t *col_ptr, const int32_t *row_idx, void *dq,
                 void *dk, void *dv, void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * asa_attn_bwd for callers that cannot allocate device memory or hand over a workspace: code
 * under HIP graph capture, tight serving / training loops, harnesses that forbid hipMalloc.
 * Same arguments, results and kernels as asa_attn_bwd, minus the workspace: the scratch memory
 * of the call (the backward's row statistics and the order of its dK / dV workgroups) lives in
 * a device array of ASA_NOALLOC_SCRATCH_BYTES that is part of the library (every GPU the library
 * is used on holds one copy until the process ends).  The call allocates and frees nothing.
 *   - The device that is current at the call must be the device of `hip_stream` and of the
 *     tensors; its array's address is looked up once per device, at the first call there.
 *   - asa_bwd_workspace_bytes(p) > ASA_NOALLOC_SCRATCH_BYTES: ASA_ERR_TOO_LARGE, nothing is
 *     enqueued (the need is 12 bytes per padded token row of all slabs plus 4 bytes per block
 *     row: 8 MiB cover B * H * L up to about 690 000 tokens; the Wan2.1 layer needs 4.7 MiB).
 *   - All calls on one GPU share that GPU's array: two calls whose work overlaps in time on
 *     one GPU (different streams, or several host threads) race; calls on one stream do not.
 *     The array keeps the previous call's contents; no call depends on them.
 */
#define ASA_NOALLOC_SCRATCH_BYTES (8u << 20)
int asa_attn_bwd_noalloc(const asa_params *p, const void *q, const void *k, const void *v,
                         const void *o, const void *o_lo, const void *d_o, const float *lse,
                         const int32_t *row_ptr, const int32_t *col_idx, const int32_t *col_ptr,
                         const int32_t *row_idx, void *dq, void *dk, void *dv, void *hip_stream);

/*
 * ASA with global tokens, ASA_G (Sec. 3.3, "ASA with Global Tokens"): K and V are extended by
 * mean-pooled copies of themselves, K_aug = Concat(K, MeanPool_n(K)) and likewise V.  A query
 * sees the original keys through the block mask exactly as in asa_attn_fwd and, in addition,
 * EVERY pooled key, with ln(n) added to its pre-soft-max score.
 *
 * The pooled part is kept in tensors of its own:
 *   kg, vg [B, H, G, d] bf16, contiguous, G = asa_global_token_count(p, n) = ceil(L/n) rounded
 *   up to a multiple of `block`.  Row w < ceil(L/n) is the mean of tokens [w n, min(L, (w+1) n))
 *   formed in fp32 and rounded to bf16 (the tensor type); rows past ceil(L/n) are zero and are
 *   never attended.  The bias is ln(n) for every window, the short last one included.
 * asa_global_tokens writes kg and vg from k and v.  n: 1 <= n <= L; ceil(L/block) +
 * G/block may not exceed 1024 (ASA_ERR_UNSUPPORTED).
 */
size_t asa_global_token_count(const asa_params *p, int n);   /* 0 on invalid arguments */
int asa_global_tokens(const asa_params *p, int n, const void *k, const void *v, void *kg,
                      void *vg, void *hip_stream);

/*
 * Forward of ASA_G: as asa_attn_fwd with the pooled keys / values kg, vg of window n appended
 * (NULL index lists: dense over the original keys, plus the pooled ones).  LSE covers both
 * parts.  Workspace: asa_fwd_g_workspace_bytes.  ASA_ERR_UNSUPPORTED here: a (batch, head) slab
 * of K spanning 4 GiB or more, and K rows that are not contiguous (k_stride[2] != d).
 */
size_t asa_fwd_g_workspace_bytes(const asa_params *p, int n);
int asa_attn_fwd_g(const asa_params *p, int n, const void *q, const void *k, const void *v,
                   const void *kg, const void *vg, const int32_t *row_ptr, const int32_t *col_idx,
                   void *o, void *o_lo, float *lse, void *workspace, size_t workspace_bytes,
                   void *hip_stream);

/*
 * Backward of ASA_G with the mask held constant.  o, o_lo, lse are asa_attn_fwd_g's outputs.
 * dq, dk, dv [B, H, L, d] bf16 hold the complete gradients: dk and dv include what flows back
 * through the pooling, the gradient of pooled token w divided by the number of tokens of its
 * window, added in fp32 before the one rounding to bf16.  Workspace: asa_bwd_g_workspace_bytes.
 */
size_t asa_bwd_g_workspace_bytes(const asa_params *p, int n);
int asa_attn_bwd_g(const asa_params *p, int n, const void *q, const void *k, const void *v,
                   const void *kg, const void *vg, const void *o, const void *o_lo, const void *d_o,
                   const float *lse, const int32_t *row_ptr, const int32_t *col_idx,
                   const int32_t *col_ptr, const int32_t *row_idx, void *dq, void *dk, void *dv,
                   void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Token rearrangement along a Gilbert (generalised Hilbert) curve (Sec. 3.3 "Preprocessing and
 * Importance Estimation"; Alg. 3 step 1): before the sequence is cut into blocks, the tokens of
 * the T x Y x X video grid are put into the order in which a space-filling curve visits them, so
 * that a block holds tokens that are neighbours in the video.  The paper names the curve and does
 * not define it; this library's curve visits every cell once, moves one cell along one axis per
 * step for every grid (its major axis is the longest axis of even length, the longest axis if
 * all are odd), and is the classical Hilbert curve on a 2^k square.
 *
 * asa_gilbert_order -- HOST function, no GPU work.  order, inverse: HOST arrays of
 * n_prefix + T*Y*X int32 (inverse may be NULL).  Position i of the rearranged sequence holds the
 * token that raster order (t major, then y, then x; after n_prefix leading tokens, which keep
 * their places) holds at order[i]; inverse[order[i]] = i.  At most 2^30 tokens.
 *
 * asa_reorder_tokens -- dst[t][b, h, i, :] = src[t][b, h, index[i], :] for t < n_tensors <= 3
 * tensors [B, H, L, d] bf16 in one launch (Q, K, V with index = order before the attention
 * calls; O, dQ, dK, dV with index = inverse after them).  index: DEVICE [L] int32; an entry
 * outside [0, L) gives a zero row.  src, dst: HOST arrays of n_tensors device pointers, read
 * during the call; a tensor cannot be its own destination.  src_stride / dst_stride: element
 * strides {B, H, L} of all sources / all destinations, NULL = packed (the strides in `p` are not
 * used).  Of `p` only B, H, L, d have a meaning here.
 */
int asa_gilbert_order(int32_t T, int32_t Y, int32_t X, int32_t n_prefix, int32_t *order,
                      int32_t *inverse);
int asa_reorder_tokens(const asa_params *p, int32_t n_tensors, const void *const *src,
                       void *const *dst, const int64_t *src_stride, const int64_t *dst_stride,
                       const int32_t *index, void *hip_stream);

/*
 * Norm of queries and keys for each head and their rotation by position, in one pass: what stands
 * between the projections of an attention layer and asa_build_mask / asa_attn_fwd.  For every
 * row x of d channels (one token of one head):
 *   ASA_NORM_RMS    y = x r,            r = 1 / sqrt(mean(x^2) + eps)
 *   ASA_NORM_LAYER  y = (x - mean(x)) r, r = 1 / sqrt(var(x) + eps)
 *   z = weight * y + bias
 *   channel pairs t < rot_dim / 2 of z:  (a, b) -> (a c - b s, a s + b c),
 *     c = cos_table[row][t], s = sin_table[row][t],  row = first_row + start[b] + l
 *     ASA_ROPE_ADJACENT  a, b = channels 2 t, 2 t + 1
 *     ASA_ROPE_HALVES    a, b = channels t, t + rot_dim / 2
 * A row outside [0, table_rows) turns nothing (first_row = -n: n text tokens in front of the video).
 * Everything is fp32 until the one rounding of the result to bf16, the sums of squares too: a row whose largest |x| is beyond
 * 2^60 or, with eps = 0, below 2^-50 is out of range.  A norm over the channels of all heads together (one weight of
 * heads * d: Wan2.1's) is not one of these.
 */
#define ASA_NORM_RMS 0
#define ASA_NORM_LAYER 1
#define ASA_ROPE_ADJACENT 0
#define ASA_ROPE_HALVES 1
typedef struct asa_qk_norm {
  int32_t H_kv;              /* heads of K; 0 = as many as Q                                    */
  int32_t kind;              /* ASA_NORM_RMS, ASA_NORM_LAYER                                     */
  float eps;                 /* finite, >= 0                                                    */
  int32_t rot_dim;           /* channels turned: a multiple of 16, 0 .. d (0: norm alone)       */
  int32_t pairing;           /* ASA_ROPE_ADJACENT, ASA_ROPE_HALVES                               */
  int32_t table_rows;        /* rows of the tables (>= 1 unless rot_dim is 0)                    */
  int32_t first_row;         /* table row of token 0                                             */
  const int32_t *start;      /* DEVICE [B], added to first_row for each sequence; NULL = zeros   */
  const float *cos_table, *sin_table;   /* DEVICE [table_rows, rot_dim / 2] fp32                 */
  const float *q_weight, *k_weight;     /* DEVICE [d] fp32; NULL = ones                          */
  const float *q_bias, *k_bias;         /* DEVICE [d] fp32, ASA_NORM_LAYER only; NULL = zeros    */
  int64_t q_out_stride[3], k_out_stride[3];  /* of q_out / dq_out and k_out / dk_out, as in
                                asa_params; all zero = packed [B, H, L, d], [B, H_kv, L, d]      */
  int64_t dq_stride[3], dk_stride[3];        /* backward: of dq and dk; all zero = q_stride, k_stride */
} asa_qk_norm;

/*
 * q [B, H, L, d], k [B, H_kv, L, d] bf16 with p's q_stride and k_stride (slices of one projection
 * [B, L, heads * d], say) -> q_out, k_out bf16.  k = k_out = NULL: queries alone (strides of keys then
 * have no say).  Of `p` only B, H, L, d, q_stride and k_stride have a meaning.  L <= 131 072.  A tensor
 * may be its own output where the strides agree; any other overlap is undefined.  Here and in the calls
 * below the rows of a tensor that is written must lie apart (a stride of 0, for one:
 * ASA_ERR_INVALID_ARG); tensors that are only read may repeat rows.  A call whose launch would have
 * 2^32 threads or more (256 for 16 tokens of 4 heads at d 128; below, for a block of the cache or for
 * 128 rows of queries) is ASA_ERR_UNSUPPORTED.
 */
int asa_qk_norm_rope(const asa_params *p, const asa_qk_norm *n, const void *q, const void *k,
                     void *q_out, void *k_out, void *hip_stream);

/*
 * Its backward: from q, k (the forward's inputs; nothing else is kept) and the gradients dq_out,
 * dk_out of the outputs (q_out_stride, k_out_stride)
 *   dq, dk             bf16, dq_stride and dk_stride (the rows of q and k may then repeat)
 *   dq_weight, dk_weight, dq_bias, dk_bias  [d] fp32, sums over batch, heads and tokens; each may be NULL
 * Sums are formed in a fixed order: runs of a call repeat bit for bit.  dq may take the place of
 * q or of dq_out (the same strides), dk that of k or dk_out.  k = dk_out = dk = NULL: queries alone.
 * The biases' gradients belong to ASA_NORM_LAYER.  The workspace's size depends on B, H, H_kv, L and d
 * alone (0 where the strides of q or k are none that a tensor may have).
 */
size_t asa_qk_norm_rope_bwd_workspace_bytes(const asa_params *p, const asa_qk_norm *n);
int asa_qk_norm_rope_bwd(const asa_params *p, const asa_qk_norm *n, const void *q, const void *k,
                         const void *dq_out, const void *dk_out, void *dq, void *dk,
                         float *dq_weight, float *dk_weight, float *dq_bias, float *dk_bias,
                         void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Keys and values kept in 8 bits: e4m3 (4 significant bits, largest value 448, no infinity) with one fp32
 * scale for each block of `block` tokens and key head; a code stands for code value * scale.
 * Generation that goes on from what was generated (chunk after chunk, token after token) writes
 * each new token once and attends to all that the cache holds.
 *
 * Memory.  Blocks of one (sequence, key head) lie one behind the other; a block is block * d bytes, in
 * groups of 32 tokens, each in the order in which the matrix cores take it:
 *   k  [B, H_kv, max_blocks, block/32, d/16, 32, 16]     token t of the group, channel 16 c + x at [c][t][x]
 *   v  [B, H_kv, max_blocks, block/32, d/32, 2, 32, 16]  token 8 m + 4 h + j, channel 32 c + x at
 *                                                        [c][h][x][4 m + j]  (m, j < 4; h < 2)
 *   k_scale, v_scale  [B, H_kv, max_blocks] fp32, finite, >= 0
 * Token l of a sequence is token l % block of block l / block.  A sequence that begins behind positions
 * that were never written needs codes and scales there that mean something: code 0 and 2^-100, say.
 */
typedef struct asa_kv_cache {
  int32_t H_kv;              /* key heads                                                        */
  int32_t max_blocks;        /* room of every sequence in blocks, 1 .. 65 536                    */
  void *k, *v;               /* DEVICE, 16-byte aligned                                          */
  float *k_scale, *v_scale;  /* DEVICE                                                           */
} asa_kv_cache;

/*
 * Writes p->L new tokens of each sequence, k and v [B, H_kv, L, d] bf16 (k_stride, v_stride; one of
 * them may be NULL: the other tensor alone), to positions start[b] .. start[b] + count[b] - 1.
 * start, count: DEVICE [B] int32; NULL = 0, p->L.  Of `p`: B, L, d, block, k_stride, v_stride.
 * A sequence then ends there: tokens before start[b] are kept, and what lay behind is no longer
 * part of it (its bytes are left as they were).
 *   - A block's scale is the least power of two 2^e, -100 <= e <= 120, with |x| <= 448 * 2^e for
 *     its finite values, and a code is x / scale rounded to nearest, ties to even: the powers of two
 *     cost e4m3 no precision and make scaling exact.
 *   - A block that holds tokens before start[b] keeps its scale if that is enough for the new ones;
 *     otherwise it gets the larger one and the codes held are rounded again to it.
 *   - NaN and infinities are stored as NaN, and have no part in the scale.
 *   - Tokens past max_blocks * block are not written; start[b] < 0 writes nothing of that sequence;
 *     count[b] counts as clamped to [0, L].
 *   - Blocks that no new token goes to are not touched.
 */
int asa_cache_write(const asa_params *p, const asa_kv_cache *c, const void *k, const void *v,
                    const int32_t *start, const int32_t *count, void *hip_stream);

/*
 * Reads tokens start[b] .. start[b] + count[b] - 1 of each sequence back into rows 0 .. count[b] - 1 of
 * k and v [B, H_kv, L, d] bf16 (k_stride, v_stride; one may be NULL): code value * scale, exact up to
 * bf16's range for the scales that asa_cache_write makes.  Rows from count[b] on, and rows of positions
 * outside [0, max_blocks * block), are left as they were.  start, count as above.
 */
int asa_cache_read(const asa_params *p, const asa_kv_cache *c, void *k, void *v,
                   const int32_t *start, const int32_t *count, void *hip_stream);

/*
 * Attention over the cache: q [B, H, L, d] bf16 (q_stride), H a multiple of H_kv; query head h reads
 * key head h / (H / H_kv).  A query sees the tokens [0, length[b]) of its sequence that lie in the
 * blocks its list keeps:
 *   S = scale * q K^T,  LSE = log sum exp S,  O = exp(S - LSE) V,   K, V = code value * scale.
 * length   DEVICE [B] int32, counts as clamped to [0, max_blocks * block]
 * row_ptr  [B*H_kv, ceil(L/block) + 1] int32, col_idx [B*H_kv, ceil(L/block) * max_blocks] int32: lists as
 *          asa_build_mask makes them, one for each block of queries and KEY head, of distinct blocks in any order;
 *          entries that are negative or at or past the sequence's last block are skipped.  Both NULL: every block.
 *          asa_build_mask's own fit where L tokens are all that is held, max_blocks = ceil(L/block) and H_kv = H; for
 *          a chunk on a longer cache, or shared key heads, the caller makes them.
 * o        [B, H, L, d] bf16 (o_stride); lse [B*H, L] fp32.  A row that sees nothing gets O = 0, LSE = -inf.
 * A scale of V below 2^-100 counts as 2^-100 (in a block of scale s keys of less than 2^-126 / s of the weight of the row's
 * heaviest count as nothing: 2^-26 at 2^-100); |V| beyond 2^96 or |q| beyond 2^112 may overflow the fp32 sums.
 * Codes are widened to bf16 (exact), products accumulate in fp32; probabilities, times the block's
 * scale of V, are rounded to bf16 before the second product.  What the cache holds at and past length[b]
 * has no influence, whatever the bytes are.  Runs of a call repeat bit for bit; the last bits of o and lse may
 * differ between calls of other sizes, of another max_blocks, or with lists instead of none (the keys of a row are
 * added up in parts whose number depends on these).  In calls of the same sizes they are the same whatever other rows hold.
 * L = 1 is a token-by-token step.  ceil(L/block) * max_blocks < 2^31.
 */
size_t asa_attn_cache_workspace_bytes(const asa_params *p, const asa_kv_cache *c);
int asa_attn_cache(const asa_params *p, const asa_kv_cache *c, const int32_t *length, const void *q,
                   const int32_t *row_ptr, const int32_t *col_idx, void *o, float *lse,
                   void *workspace, size_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* ASA_H_ */
