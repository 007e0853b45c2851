/*
 * jet.h -- C ABI of libjet: the block-scaled FP8 linear layer of Jet-RL's
 * unified precision flow, and the attention operators beside it, for AMD MI355X (gfx950).
 *
 * One linear layer Y = X W^T (Jet-RL, Sec. 2.2) runs three GEMMs -- FProp,
 * DGrad, WGrad -- on FP8 E4M3 operands (Sec. 2.1: Delta_max = 448) quantized
 * with 1x128 groups for activations and gradients and 128x128 blocks for
 * weights (Sec. 4.2).  Rollout (decode-shaped, small M) and training forward
 * call the SAME entry point and obtain bit-identical rows (Sec. 4.1: the
 * inference graph is a subgraph of the training forward graph).  That is not so of
 * the attention: its passes agree within their roundings.
 *
 * Conventions for every call
 *   - M = tokens, N = output features, K = input features (the paper's N, D, C).
 *   - Every pointer is a DEVICE pointer to a dense row-major array owned by the
 *     caller; the library allocates nothing, keeps no pointer after the call
 *     returns, and does not synchronise.  Required pointers must be 16-byte
 *     aligned.  Outputs must not alias inputs.
 *   - bf16 arrays are passed as void* (2 bytes per element); FP8 arrays are
 *     uint8_t E4M3 codes; scales are IEEE binary32.
 *   - `stream` is a hipStream_t passed as void* (NULL = the default stream);
 *     work is enqueued asynchronously on it.
 *   - Errors are return codes only.  All argument checks happen on the host
 *     before anything is launched; on error nothing is written.
 *   - Sizes: every dimension at most 2^30; the reduction length of a GEMM (K for
 *     FProp, N for DGrad, M for WGrad) below 2^24; the row count of a tensor that
 *     is quantized in 128x128 tiles (jet_quant_weight, jet_silu_mul_bwd_quant, and
 *     jet_quant_act whenever the colT pair is requested) at most 65535 * 128; the K of
 *     jet_silu_mul_bwd_quant, half a row of its output, below 2^29.  Otherwise:
 *     JET_ERR_SHAPE.
 *   - JET_ERR_LAUNCH reports the status of this call's own launch only: an error
 *     left pending by the caller's earlier HIP calls is discarded first.
 *   - Inputs must be finite (NaN / Inf: no fault, result unspecified).
 *   - Same inputs give the same bytes on every call; kernel selection depends
 *     on shapes only and does not change any output bit (but for the order of sums
 *     in the attention operators, which may depend on the sizes of a call).
 *
 * Quantizer (Sec. 2.1):  S = max|X| / 448 over the group (binary32 division;
 * S = 1 for an all-zero group),  code = E4M3( X / S ) rounded to nearest, ties
 * to even, saturating at +-448, sign of zero kept.
 *
 * GEMM element (Sec. 2.2 on Sec. 4.2 operands), R = reduction length:
 *   acc = 0;  for g = 0 .. R/128-1 ascending:
 *       p   = sum over the 128 products of group g  (FP8 matrix-core sum)
 *       s   = sa[i,g] * sb[.,g]                     (binary32 product)
 *       acc = fma(p, s, acc)                        (binary32)
 *   out = bf16(acc), round to nearest even.
 * The chain is the same for every M, so a token row does not depend on the
 * call it is computed in.
 * Accuracy of p: the matrix core does not add the 128 exact products in
 * binary32.  Within each block of 8 consecutive products it cuts every product
 * toward zero to a multiple of 2^(E-13), E being the largest exponent sum of the
 * block, and adds the blocks at 24 bits or more.  For quantized operands p is
 * within 2^-13 of the sum of |products| of the exact group sum (2^-17 on
 * average).  The result therefore equals the exact-product binary32 chain within
 * 2 bf16 ulp except where the group sums cancel: an element much smaller than
 * the sum of its |terms| carries the cut of the large products as an absolute
 * error.  The tests hold every output bit against a CPU model of these steps.
 */
#ifndef JET_H
#define JET_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* The entry points below are the only symbols the library exports. */
#define JET_API __attribute__((visibility("default")))

typedef enum {
    JET_OK = 0,
    JET_ERR_NULL = 1,   /* a required pointer is NULL */
    JET_ERR_SHAPE = 2,  /* a size is < 1 or breaks a divisibility rule */
    JET_ERR_ALIGN = 3,  /* a pointer is not 16-byte aligned */
    JET_ERR_ARG = 4,    /* bad enum value or inconsistent optional arguments */
    JET_ERR_LAUNCH = 5  /* the HIP runtime refused the launch */
} jet_status;

/* Source format of jet_quant_act. */
typedef enum {
    JET_SRC_BF16 = 0,    /* x is bf16 [M,K] */
    JET_SRC_FP8_ROW = 1  /* x is E4M3 [M,K] with x_scales f32 [M,K/128]; the element
                            value is decode(code) * scale (one binary32 multiply):
                            the FP8-saved activation of Sec. 4.1 */
} jet_src;

/*
 * 1x128 per-group quantization of activations and gradients (Sec. 4.2).
 * One pass over x emits either or both of
 *   row  : groups of 128 consecutive k of one row m
 *          q_row  u8 [M,K],  s_row  f32 [M,K/128]
 *   colT : groups of 128 consecutive m of one column k, stored transposed
 *          q_colT u8 [K,M],  s_colT f32 [K,M/128]      needs M % 128 == 0
 * K % 128 == 0 is required in every mode (the tensors of a layer are consumed by
 * GEMMs whose reduction or output axis K is; the kernels work on 128-wide tiles).
 * (the 128x1 operand of WGrad; both at once is the fused quantization of dY
 * for DGrad and WGrad).  A pair is skipped when both its pointers are NULL;
 * giving only one pointer of a pair is JET_ERR_NULL; skipping both pairs is
 * JET_ERR_ARG.  x_scales is required for JET_SRC_FP8_ROW (else ignored).
 */
JET_API jet_status jet_quant_act(const void* x, const float* x_scales, jet_src src,
                         int64_t M, int64_t K,
                         uint8_t* q_row, float* s_row,
                         uint8_t* q_colT, float* s_colT,
                         void* stream);

/*
 * 128x128 per-block quantization of weights (Sec. 4.2).  w bf16 [N,K] ->
 * q u8 [N,K], s f32 [N/128,K/128].  Optional transposed copy for DGrad:
 * qT u8 [K,N], sT f32 [K/128,N/128] with the same codes and scales (the scheme
 * is symmetric under transpose).  qT and sT are given together or both NULL.
 * Needs N % 128 == 0 and K % 128 == 0.
 */
JET_API jet_status jet_quant_weight(const void* w, int64_t N, int64_t K,
                            uint8_t* q, float* s, uint8_t* qT, float* sT,
                            void* stream);

/*
 * FProp (Sec. 2.2):  y bf16 [M,N] = X W^T  from (qx,sx) = row quantization of
 * X [M,K] and (qw,sw) = block quantization of W [N,K].  Any M >= 1 (decode and
 * training shapes alike); N % 128 == 0, K % 128 == 0.
 */
JET_API jet_status jet_fp8_linear_fwd(const uint8_t* qx, const float* sx,
                              const uint8_t* qw, const float* sw,
                              void* y, int64_t M, int64_t N, int64_t K,
                              void* stream);

/*
 * DGrad (Sec. 2.2):  dx bf16 [M,K] = dY W  from (qdy,sdy) = row quantization
 * of dY [M,N] (groups along N) and (qwT,swT) = the transposed copy written by
 * jet_quant_weight ([K,N], [K/128,N/128]).  Any M >= 1; N, K multiples of 128.
 */
JET_API jet_status jet_fp8_linear_dgrad(const uint8_t* qdy, const float* sdy,
                                const uint8_t* qwT, const float* swT,
                                void* dx, int64_t M, int64_t N, int64_t K,
                                void* stream);

/*
 * WGrad (Sec. 2.2):  dw bf16 [N,K] = dY^T X  from the column-transposed
 * quantizations (qdyT,sdyT) [N,M],[N,M/128] and (qxT,sxT) [K,M],[K,M/128],
 * both grouped along the token axis.  M, N, K multiples of 128.
 */
JET_API jet_status jet_fp8_linear_wgrad(const uint8_t* qdyT, const float* sdyT,
                                const uint8_t* qxT, const float* sxT,
                                void* dw, int64_t M, int64_t N, int64_t K,
                                void* stream);

/*
 * Fused producers (Sec. 4.2: the quantization of an activation is fused with
 * the operator in front of the GEMM; Sec. 4.3 names RMSNorm and the activation
 * function).  The operator is evaluated with bf16 module semantics and its
 * result h goes straight to the 1x128 row quantizer: q_row u8 [M,K], s_row f32
 * [M,K/128] are bit-identical to jet_quant_act on a stored bf16 h, which is
 * never written.  K % 128 == 0; any M >= 1.
 *
 * RMSNorm:  h[m,k] = bf16( gamma[k] * bf16( x[m,k] * r[m] ) ),
 *           r[m] = 1 / sqrt( mean_k x[m,k]^2 + eps ).
 * x bf16 [M,K], gamma bf16 [K], eps >= 0 finite (else JET_ERR_ARG).  The mean
 * is formed in binary64 and rounded once to binary32; the rest is binary32.
 * K <= 32768 (a row is held in the registers of one workgroup).  A row of
 * zeros with eps == 0 has no defined result.
 */
JET_API jet_status jet_rmsnorm_quant(const void* x, const void* gamma, float eps,
                             int64_t M, int64_t K,
                             uint8_t* q_row, float* s_row, void* stream);

/*
 * SiLU(gate) * up:  a = bf16( g / (1 + e^-g) ), the real function rounded once;
 *                   h = bf16( a * u ), a binary32 product.
 * gate, up: bf16 [M,K] with a common row stride ld >= K in elements, ld % 8 ==
 * 0 (ld = K for two dense tensors, ld = 2K for the two halves of a fused
 * gate/up projection output).
 */
JET_API jet_status jet_silu_mul_quant(const void* gate, const void* up, int64_t ld,
                              int64_t M, int64_t K,
                              uint8_t* q_row, float* s_row, void* stream);

/*
 * Backward of the operator above, h = bf16( bf16(silu(g)) * u ), for an MLP block whose
 * saved GEMM inputs are FP8 (Sec. 4.1: activations saved for the backward GEMMs are the FP8
 * tensors; the gradients that travel between operators stay bf16).  With a = bf16(silu(g)):
 *     dup   = bf16( dh * a ),   da = bf16( dh * u ),
 *     dgate = bf16( da * silu'(g) ),  silu'(g) = s (1 + g (1 - s)),  s = 1 / (1 + e^-g),
 * each the real value rounded once.  gate, up: bf16 [M,K], row stride ld; dh: bf16 [M,K]
 * dense; dgate, dup: bf16 [M,K], row stride ld_out (ld_out = 2K writes the two halves of one
 * [M,2K] gradient, ready for jet_quant_act with both output pairs).  K % 128 == 0,
 * ld >= K, ld_out >= K, ld % 8 == 0, ld_out % 8 == 0.  Outputs must not alias inputs.
 */
JET_API jet_status jet_silu_mul_bwd(const void* gate, const void* up, int64_t ld, const void* dh,
                                    int64_t M, int64_t K, void* dgate, void* dup, int64_t ld_out,
                                    void* stream);

/*
 * The same, with the row and column quantization of dgu = [dgate | dup] formed in the same pass: dgu bf16 [M,2K] and
 * (q_row, s_row) u8 [M,2K], f32 [M,2K/128], (q_colT, s_colT) u8 [2K,M], f32 [2K,M/128] are
 * bit-identical to jet_silu_mul_bwd followed by jet_quant_act with both pairs.  All outputs are required; M, K
 * multiples of 128, ld as above.  From version 102 on.
 */
JET_API jet_status jet_silu_mul_bwd_quant(const void* gate, const void* up, int64_t ld,
                                const void* dh, int64_t M, int64_t K, void* dgu,
                                uint8_t* q_row, float* s_row, uint8_t* q_colT, float* s_colT,
                                void* stream);

/*
 * Operators of the attention block, between the q/k/v projection and the output projection (from version 103 on).
 *
 * Heads have dim = 64 or 128 channels; n_q query heads share n_kv key/value heads, n_q % n_kv == 0, the group of a
 * key/value head g being the query heads g n_q/n_kv .. (g+1) n_q/n_kv - 1.  Row strides ld* count elements, are multiples of 8 and
 * at most 2^24; the heads of a row lie dim apart.  Tokens times the heads of a row are at most 2^29, n_q / n_kv at most 512.
 *
 * qk_norm_rope: qkv bf16 [T, ld] holds the n_q query, n_kv key and n_kv value heads of every token.
 *     n = x / sqrt(mean x^2 + eps) * gamma             (gamma_q, gamma_k bf16 [dim]; both NULL: n = x)
 *     y_i = n_i cos - n_{i+dim/2} sin,  y_{i+dim/2} = n_{i+dim/2} cos + n_i sin,   i < dim/2,
 * in binary32, rounded to bf16 once: q [T, n_q, dim], k [T, n_kv, dim], both dense.  table f32 [table_rows, dim] holds the dim/2
 * cosines of a position, then its sines; a position outside the table gives NaN.  With a cache, slots int64 [T] says where
 * the token's key and value go too: slot s is row s % page of page s / page; any other value keeps the token out.  No two
 * tokens of a call have the same slot.  Into a cache in E4M3 a head goes as the row quantizer has it: S = max|x| / 448
 * (1 for zeros) of the bf16 values, codes of x / S.
 */
typedef struct {
    void *k, *v;               /* [n_pages, n_kv, page, dim]: bf16, or E4M3 codes where the scales are given */
    float *k_scale, *v_scale;  /* [n_pages, n_kv, page], both or neither */
    int64_t n_pages, n_kv;
    int64_t page;              /* tokens of a page, a multiple of 16, at most 2^16 */
    int64_t dim;
} jet_kv_cache;

JET_API jet_status jet_qk_norm_rope(const void* qkv, int64_t ld, int64_t T, int64_t n_q, int64_t n_kv, int64_t dim,
                            const float* table, int64_t table_rows, const int32_t* positions,
                            const void* gamma_q, const void* gamma_k, float eps, void* q, void* k,
                            const jet_kv_cache* cache, const int64_t* slots, void* stream);

/*
 * Its gradient.  dq [T, n_q, dim], dk [T, n_kv, dim] dense; dx bf16 [T, ld_dx] gets the gradients of the query and key heads in
 * columns 0 .. (n_q + n_kv) dim - 1; dgamma_q, dgamma_k f32 [dim], with the gammas or not at all.  qkv may be
 * NULL without norm.  workspace: jet_qk_norm_rope_bwd_workspace bytes (sums of the workgroups; none without norm).
 */
JET_API int64_t jet_qk_norm_rope_bwd_workspace(int64_t T, int64_t n_q, int64_t n_kv, int64_t dim);
JET_API jet_status jet_qk_norm_rope_bwd(const void* dq, const void* dk, const void* qkv, int64_t ld, int64_t T, int64_t n_q,
                                int64_t n_kv, int64_t dim, const float* table, int64_t table_rows, const int32_t* positions,
                                const void* gamma_q, const void* gamma_k, float eps, void* dx, int64_t ld_dx,
                                float* dgamma_q, float* dgamma_k, void* workspace, void* stream);

/*
 * Attention of packed sequences.  Sequence s has the rows cu_q[s] .. cu_q[s+1] - 1 of q [Tq, ldq] and cu_k[s] .. of k, v
 * [Tk, ldk / ldv]; cu_q, cu_k int32 [n_seqs + 1] on the device, ascending from 0.  Lengths may be zero.
 *     s_ij = scale q_i k_j,  lse_i = ln sum_j e^s_ij,  o_i = sum_j e^(s_ij - lse_i) v_j       (scale > 0)
 * over all keys of the sequence, or with `causal` those whose distance to the sequence's end is at least the row's: the last
 * row sees the last key, a longer k is what came before q.  A row that sees no key has o = 0, lse = -inf and no
 * gradients; so has one in no sequence.  o bf16 [Tq, n_q, dim] dense, lse f32 [n_q, Tq].  Sums and logarithms are binary32; the
 * probabilities enter the second product in bf16.  Keys of other sequences have no influence, whatever they hold.  In a sequence a
 * product runs over whole tiles, with probabilities of 0 for what is not seen: a value that is not finite may reach the results of rows up to 94
 * positions in front of it, which do not see it; in the gradients, a key dq of rows up to 62 positions in front of it, a query
 * or output gradient dk and dv of keys up to 62 positions behind it.  The order of the sums depends on Tq, Tk, n_seqs and the heads,
 * and on a row's place in its sequence; 32 rows of a sequence renew the reference of their exponentials together, so that the last bits
 * of a row also depend on the scores of its neighbours.  Limits beside those above: n_seqs <= 2^20, (Tq n_q / n_kv / 64 + n_seqs + 2) n_kv <= 2^23.
 */
JET_API jet_status jet_attention_fwd(const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv,
                             const int32_t* cu_q, const int32_t* cu_k, int64_t n_seqs, int64_t Tq, int64_t Tk,
                             int64_t n_q, int64_t n_kv, int64_t dim, float scale, int causal, void* o, float* lse, void* stream);

/*
 * Its gradients from what the forward call read and wrote and the gradient dout of o (dense like it): dq, dk, dv bf16 with row
 * strides of their own, so that dv may be a slice of the projection's gradient.  Gradients of a shared head are summed over its
 * group in binary32; probabilities and score gradients enter the products in bf16.  sum_j p_ij dp_ij is not left at what the rounded
 * o gives: it is corrected to binary32, in dq where that makes more than half a step of bf16 of sum_j |ds_ij| (by which the
 * time depends on the values).  So lse has to be the forward call's for these keys: that of a larger softmax, of which they are a
 * part, whose probabilities here sum to less than 1, does not give its gradients.  No atomic sums: same inputs, same bytes.
 * Limit beside those of the forward call: (Tk / 16 + 8 (n_seqs + 2)) n_kv <= 2^23.
 * workspace: 8 bytes for each row and query head, and where the rows of a tile of keys may be dealt to several workgroups, binary32
 * sums of dk and dv for each of them, up to eight times Tk n_kv 2 dim 4 bytes.  The host does not see how long the sequences are:
 * with several of them the sums are sized as if one could have nearly all rows, whether or not any tile is split (64
 * sequences of 1024 tokens, 32 and 8 heads of 128: 4.3 GB, of which they use the first 17 MB; one sequence of 8192: 0.14 GB).
 */
JET_API int64_t jet_attention_bwd_workspace(int64_t n_seqs, int64_t Tq, int64_t Tk, int64_t n_q, int64_t n_kv, int64_t dim);
JET_API jet_status jet_attention_bwd(const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv,
                             const void* o, const float* lse, const void* dout,
                             const int32_t* cu_q, const int32_t* cu_k, int64_t n_seqs, int64_t Tq, int64_t Tk,
                             int64_t n_q, int64_t n_kv, int64_t dim, float scale, int causal,
                             void* dq, int64_t ld_dq, void* dk, int64_t ld_dk, void* dv, int64_t ld_dv,
                             void* workspace, void* stream);

/*
 * Attention of one query token per sequence, q [B, ldq] with n_q heads, over the first lengths[b] rows of the cache pages
 * pages[b][0], pages[b][1], ... (int32 [B, max_pages]; lengths int32 [B]).  o bf16 [B, n_q, dim]: zero where the length is not
 * positive, NaN where a page that is needed lies outside the cache or the length beyond max_pages * page (<= 2^30).  What the
 * cache holds behind a length has no influence.  workspace: jet_attention_decode_workspace bytes (may be none).
 * Limit: 2^23 workgroups, one for each sequence, key/value head, 16 query heads of its group, and 2048 keys of the row of pages.
 */
JET_API int64_t jet_attention_decode_workspace(const jet_kv_cache* cache, int64_t B, int64_t n_q, int64_t max_pages);
JET_API jet_status jet_attention_decode(const void* q, int64_t ldq, int64_t n_q, const jet_kv_cache* cache, const int32_t* pages,
                                int64_t max_pages, const int32_t* lengths, int64_t B, float scale, void* o,
                                void* workspace, void* stream);

/*
 * Operators of a training step around the blocks (from version 104 on).
 *
 * Embedding: w [V, H], bf16 or f32, holds the rows of the ids first .. first + V - 1 (a shard of a larger table, or first = 0);
 *     y_t = bf16( scale w[ids_t - first] ),   zeros for any other id.
 * ids int64 or int32 [T]; y bf16 [T, H].  H % 8 == 0, H <= 2^20, V < 2^31, T <= 2^22, T H <= 2^36, |first| <= 2^62,
 * scale finite.
 */
typedef enum { JET_BF16 = 0, JET_F32 = 1 } jet_type;
typedef enum { JET_I64 = 0, JET_I32 = 1 } jet_ids;

JET_API jet_status jet_embedding_fwd(const void* ids, jet_ids ids_type, int64_t T, const void* w, jet_type w_type, int64_t V, int64_t H,
                             int64_t first, float scale, void* y, void* stream);

/*
 * Its gradient with respect to the table, from dy bf16 [T, H]:
 *     dw_v = scale sum of dy_t over the tokens t with ids_t - first = v,
 * a binary32 sum, rounded once to dw's type, bf16 or f32 [V, H].  add == 0: all of dw is written, zeros where no token is; else the
 * sums are added to what it holds (in binary32), and rows without a token are not touched.  No atomic sums: same inputs, same bytes; the
 * order of a sum depends on T, H and the ids.  workspace: jet_embedding_bwd_workspace bytes (may be none).
 */
JET_API int64_t jet_embedding_bwd_workspace(int64_t T, int64_t H);
JET_API jet_status jet_embedding_bwd(const void* ids, jet_ids ids_type, int64_t T, const void* dy, int64_t V, int64_t H, int64_t first,
                             float scale, void* dw, jet_type dw_type, int add, void* workspace, void* stream);

/*
 * Layer norm of the rows of x bf16 [M, K], or of sum = bf16( x + residual ) where residual and sum (bf16 [M, K]) are given, with
 * gamma, beta bf16 [K] (beta may be NULL: 0):
 *     y = bf16( (x - mean) / sqrt( var + eps ) * gamma + beta ),   var = mean (x - mean)^2.
 * Either y bf16 [M, K], or the pair (q_row, s_row) that jet_quant_act makes of it, bit for bit (K % 128 == 0), the other one NULL.
 * Sums are binary32, with a mean that is corrected by the mean of the differences from it; a row gets the same bytes in every call.
 * K % 8 == 0, K <= 32768, M <= 2^23, M K <= 2^34.  Squares and sums of a row are binary32: the result is that of the formula where var + eps lies in
 * 2^-111 .. 2^126 and the sum of the row's magnitudes below 2^127.  A row of equal values with eps == 0 has no defined result.
 */
JET_API jet_status jet_layernorm_fwd(const void* x, const void* residual, const void* gamma, const void* beta, float eps, int64_t M,
                             int64_t K, void* sum, void* y, uint8_t* q_row, float* s_row, void* stream);

/*
 * Gradients of a norm of the rows of x from dy bf16 [M, K]; x is what the norm was taken of (with a residual, the sum).
 *     JET_NORM_LAYER:  n = (x - mean) r,  r = 1 / sqrt( var + eps ),           dx = r (g - mean(g) - n mean(g n)) + dres
 *     JET_NORM_RMS:    n = x r,           r = 1 / sqrt( mean(x^2) + eps ),     dx = r (g - n mean(g n)) + dres
 * with g = dy gamma and dres bf16 [M, K] the gradient that reaches x beside the norm (NULL: none);
 *     dgamma = sum over the rows of dy n,   dbeta = sum over the rows of dy     (f32 [K]; dbeta with JET_NORM_LAYER only).
 * dx is rounded once.  The gradient of jet_rmsnorm_quant's operator is JET_NORM_RMS (its roundings taken for the identity).  Sums
 * over a row are binary32, with a mean that is corrected by the mean of the differences from it (so that r is not, to the bit, what
 * jet_rmsnorm_quant takes, whose sum is binary64); those over the rows are binary32 in each workgroup and binary64 between them.  Their order
 * depends on M and K, dx on the row and K alone.  Ranges as in jet_layernorm_fwd, mean(x^2) in place of var for JET_NORM_RMS.  With eps == 0 a row of equal values
 * (RMS: of zeros) has no defined result, nor have the sums then.  M and K as in jet_layernorm_fwd.  workspace: jet_norm_bwd_workspace bytes.
 */
typedef enum { JET_NORM_LAYER = 0, JET_NORM_RMS = 1 } jet_norm;
JET_API int64_t jet_norm_bwd_workspace(jet_norm kind, int64_t M, int64_t K);
JET_API jet_status jet_norm_bwd(jet_norm kind, const void* dy, const void* x, const void* gamma, const void* dres, float eps, int64_t M,
                        int64_t K, void* dx, float* dgamma, float* dbeta, void* workspace, void* stream);

/*
 * The norm over all elements of n tensors, norm f32 [1] = sqrt( sum of squares ) (binary64 sums, rounded once), and the tensors scaled
 * down to max_norm >= 0 (infinity: never):
 *     x <- x * (max_norm / norm)   where norm > max_norm and norm is finite; else x stays as it is.
 * The factor is rounded to binary32, or where it is below 2^-126 taken in binary64.  As everywhere here, the addresses of all tensors are multiples of 16
 * (JET_ERR_ALIGN): a view into a flat buffer has to begin at one.
 * `tensors` is an array on the HOST, read during the call; n = 0 elements are fine, and data may then be NULL.  jet_clip_grads
 * writes to `out` (n tensors of the same sizes and types) or, where that is NULL, in place.  given (f32 [1]): the norm to go by, for
 * instance over all shards; it is not formed then.  norm may be NULL in jet_clip_grads.  No two tensors that are written overlap,
 * nor does one that is written overlap another that is read (JET_ERR_ARG); given and norm count as such.  workspace: jet_grad_norm_workspace bytes, not
 * needed with `given`.  At most 2^16 tensors, of at most 2^40 elements.
 */
typedef struct {
    void* data;
    int64_t n;        /* elements */
    jet_type type;
} jet_tensor;
JET_API int64_t jet_grad_norm_workspace(int64_t n);
JET_API jet_status jet_grad_norm(const jet_tensor* tensors, int64_t n, float* norm, void* workspace, void* stream);
JET_API jet_status jet_clip_grads(const jet_tensor* tensors, const jet_tensor* out, int64_t n, float max_norm, const float* given,
                          float* norm, void* workspace, void* stream);

/* Text for a status code (static storage). */
JET_API const char* jet_status_str(jet_status st);

/* Library version: major * 10000 + minor * 100 + patch. */
JET_API int jet_version(void);

#ifdef __cplusplus
}
#endif
#endif /* JET_H */
