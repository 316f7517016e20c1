/*
 * jf_ops.h -- single operators of libjf on caller-owned device buffers, outside any context.
 *
 * jf_op_gemm* run one kernel of the forward pass of Jacobi Forcing's Jacobi iteration (arXiv
 * 2512.14681, Sec. 2.1 Eq. 3: one pass over all in-flight rows). jf_op_kv8_* keep and read a paged
 * cache held in 8 bits, and jf_op_token_logprobs* score given tokens and give the gradient of that
 * score: a draft's or trajectory's tokens over a long context, and the loss of training on them.
 * jf_op_policy_loss is such a loss with its gradient, and jf_op_packed_attention* attention of a batch of
 * whole texts, without a cache, with its backward pass.
 * Same conventions as jf.h: plain pointers, the caller owns all memory, work is ordered on
 * `cuda_stream` (NULL = legacy default stream) and the call does not synchronise; arguments are
 * validated on the host before any launch. `err_word`: device int that receives a device error code
 * (first writer wins); the caller zeroes it before its first use and reads it after synchronising.
 */
#ifndef JF_OPS_H
#define JF_OPS_H

#include <stddef.h>
#include <stdint.h>

#include "jf.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Device workspace bytes jf_op_gemm needs for this shape (split-K partial tiles and tile
 * tickets). k_splits <= 0 selects the split the forward pass uses for this weight shape. */
jf_status jf_op_gemm_workspace_bytes(int N, int K, int M, int k_splits, size_t* out_bytes);

/* Projection Y[m, n] = sum_k X[m, k] * W[n, k] (fp32 accumulate), the weight-streaming GEMM of
 * every projection of the forward pass.
 * dtype JF_BF16: W [N][K] and X [M][K] bf16 (device, 16-byte aligned, K % 8 == 0), tcgen05
 *   tensor cores fed by TMA; JF_F32: W, X fp32, CUDA cores.
 * Y: device fp32 [M][N]. workspace: device, jf_op_gemm_workspace_bytes() bytes, zero-filled before
 * its first use and after a call that left an error code. Calls of different shapes may then share it
 * on a stream: tickets are zero again after a call, and partial tiles that a call of another shape left
 * where this one's tickets are count as zero. err_word: device int that receives a device error code
 * (0 = none); the caller reads it after synchronising. */
jf_status jf_op_gemm(int dtype, const void* W, const void* X, float* Y, int N, int K, int M, int k_splits,
                     void* workspace, size_t workspace_bytes, int* err_word, void* cuda_stream);

/* Size of the fixed device scratch of jf_op_gemm_noalloc (8 MiB). */
#define JF_OP_GEMM_NOALLOC_SCRATCH_BYTES (8u << 20)

/* jf_op_gemm without a workspace, for callers that cannot allocate device memory: code running
 * inside a device-memory allocator's own hooks, or a process whose device memory is entirely
 * reserved by another pool, cannot obtain the workspace jf_op_gemm asks for. (The paper has no
 * counterpart; this is a library facility.)
 * dtype is bf16 only: W [N][K], X [M][K] bf16 (device, 16-byte aligned, K % 8 == 0), Y fp32 [M][N].
 * The split-K scratch is one static device array of JF_OP_GEMM_NOALLOC_SCRATCH_BYTES that every GPU
 * loading libjf holds until the process exits; a shape whose jf_op_gemm_workspace_bytes() exceeds
 * it is refused with JF_ECAPACITY before any launch. The call allocates nothing (no cudaMalloc,
 * no cudaFree, no allocating library routine). Its first call on a device looks up the array's
 * device address (cudaGetSymbolAddress) and sets that device's kernel attributes, so make that
 * first call before any stream capture. Under CUDA's lazy module loading (the default) that first
 * look-up may also be what loads libjf's device code onto the device and reserves the array there:
 * make the first call at start-up, before another pool takes the device memory, or run with
 * CUDA_MODULE_LOADING=EAGER so that the array is reserved when the library is loaded. All calls share the array: calls that may overlap on the GPU (other streams,
 * other threads) race on it and must be serialised by the caller; each call re-zeroes the tickets
 * it uses before its kernel runs. err_word and cuda_stream as in jf_op_gemm. */
jf_status jf_op_gemm_noalloc(const void* W, const void* X, float* Y, int N, int K, int M, int k_splits,
                             int* err_word, void* cuda_stream);

/* A paged key/value cache held in 8 bits. A page holds 16 consecutive tokens of one sequence for every
 * KV head; a block is one head of one page and has one scale. It stands for x = c * 2^e: c is an e4m3
 * value (sign, 4 exponent bits with bias 7, 3 mantissa bits; largest 448) and e the block's exponent,
 * -120 <= e <= 119. A power of two as the scale costs no precision (c is a floating-point number) and
 * folds into a product exactly.
 *   k, v: [n_pages][n_kv_heads][16][head_dim] codes, 16-byte aligned (as a tensor of e4m3 values);
 *   k_exp, v_exp: [n_pages][n_kv_heads] exponents;
 *   page_table: [n_seqs][pages_per_seq]: page of tokens 16 i .. 16 i + 15 of a sequence at entry i
 *     (entries past a sequence's last token are not read).
 * head_dim 64 or 128; n_seqs <= 1024; n_kv_heads <= 32767. All pointers DEVICE, all memory the caller's. Slots that no token
 * was appended to may hold anything. */
typedef struct {
  void *k, *v;
  int8_t *k_exp, *v_exp;
  const int32_t* page_table;
  int n_seqs, n_pages, pages_per_seq, n_kv_heads, head_dim;
} jf_kv8_cache;

/* The new rows of a batch: rows row_start[b] .. row_start[b+1]-1 are the tokens of sequence b at its
 * slots len[b], len[b]+1, ... (b may have none). row_start [n_seqs + 1] ascending from 0 to n_rows and
 * len [n_seqs] are DEVICE arrays, read when the kernels run (a captured graph follows them); n_rows and
 * max_rows (every sequence's row count or more: it chooses the attention's form; where row_start has changed
 * since, the numbers are the same up to rounding) are host numbers. A sequence whose rows lie outside its
 * page table, and pages outside the pool, are reported through err_word (as JF_EDEVICE's bounds code 4) and
 * left out. */
typedef struct {
  const int32_t *row_start, *len;
  int n_rows, max_rows;
} jf_kv8_rows;

/* Append the rows' keys and values, rotated on the way, and rotate their queries.
 * dtype (JF_BF16 or JF_F32): type of q, k, v: [n_rows] rows of n_heads (q) or n_kv_heads (k, v) heads of
 * head_dim features, rows ld_* elements apart (so that the three may be parts of one projection's rows).
 * rope: device fp32 [rope_len][head_dim / 2][2] (cos, sin), 8-byte aligned: keys and queries are rotated
 * (pairs i, i + head_dim / 2, in fp32, products and sum each rounded once); NULL: they are not. positions:
 * device int32 [n_rows], the row's entry in rope; NULL: its slot (a recycled candidate's rows lie behind
 * the draft in the cache, but start over in position). q_out: [n_rows][n_heads][head_dim] of out_dtype; q,
 * q_out NULL: no queries.
 * A block that holds tokens before slot len[b] keeps them: its exponent becomes max(its own, what the new
 * rows need) and, where it grew, its codes are rounded again. Other blocks take what the new rows need:
 * the smallest e with |x| <= 448 * 2^e for all of them. Codes are rounded to nearest, ties to even. Tokens
 * at or behind slot len[b] are replaced, so rejected drafts need no clearing: the next append starts at the
 * accepted length. The cache never holds a NaN: a new NaN is held as 0, an infinity as +-448 * 2^e of the
 * finite ones' e, and err_word receives the code 7. Values beyond 448 * 2^119 are held as that.
 * err_word: see the head of this file. */
jf_status jf_op_kv8_append(const jf_kv8_cache* cache, const jf_kv8_rows* rows, int dtype, const void* q, long long ld_q,
                           const void* k, long long ld_k, const void* v, long long ld_v, int n_heads,
                           const int32_t* positions, const float* rope, int rope_len, int out_dtype, void* q_out,
                           int* err_word, void* cuda_stream);

/* The values that the cache stands for at the rows' slots: k_out, v_out [n_rows][n_kv_heads][head_dim] of
 * out_dtype (either may be NULL). Exact in both types (bf16: what lies below its subnormal range rounds). */
jf_status jf_op_kv8_read(const jf_kv8_cache* cache, const jf_kv8_rows* rows, int out_dtype, void* k_out, void* v_out,
                         int* err_word, void* cuda_stream);

/* Device workspace bytes of jf_op_kv8_attention on the current device (it does not depend on the lengths;
 * no initialisation needed; calls that may overlap on the GPU need one each). */
jf_status jf_op_kv8_attention_workspace_bytes(const jf_kv8_cache* cache, const jf_kv8_rows* rows, int dtype, int n_heads,
                                              size_t* out_bytes);

/* Attention of the rows, whose keys and values have been appended, over the cache: out = softmax(scale *
 * q k^T) v for each of n_heads query heads (a multiple of n_kv_heads; head h reads KV head
 * h / (n_heads / n_kv_heads)), over the keys that the row sees. dtype: type of q and out. q: rows ld_q
 * elements apart (rotated: jf_op_kv8_append's q_out); out: [n_rows][n_heads][head_dim], 16-byte aligned.
 * mask NULL: row i of a sequence sees slots 0 .. len + i. Else mask is [n_rows][mask_words] 32-bit words,
 * 32 * mask_words >= max_rows: the row sees slots 0 .. len - 1, and slot len + j if bit j % 32 of word j / 32
 * is set (a tree of drafts and candidates); a word that the mask does not have counts as 0. lse (optional):
 * fp32 [n_rows][n_heads], the natural logarithm of the sum of exponentials. A row that sees nothing gets out 0
 * and lse -infinity; a NaN in a row's query reaches that row's outputs only.
 * Softmax statistics and sums are fp32. JF_BF16: products of fp16 operands (codes exactly; queries scaled
 * by a power of two per row, exact above 2^-29 of the row's largest; probabilities rounded to 11 bits).
 * JF_F32: queries and probabilities as two fp16 terms. In both, a key whose weight is below 2^-25 of the
 * row's largest may add nothing to out (lse counts it). Results do not depend on the order in which CTAs
 * run; they depend in rounding on the batch, whose work is split evenly over the GPU. */
jf_status jf_op_kv8_attention(const jf_kv8_cache* cache, const jf_kv8_rows* rows, int dtype, const void* q, long long ld_q,
                              int n_heads, float scale, const uint32_t* mask, int mask_words, void* out, float* lse,
                              void* workspace, size_t workspace_bytes, int* err_word, void* cuda_stream);

/* Log probabilities of given tokens. logits: [rows] of `vocab` values of dtype (JF_F32 or JF_BF16), rows ld
 * elements apart, any alignment of the type; z = logit * scale (0 < scale <= 1e30: an inverse temperature).
 * targets: device int32 [rows]; a negative one asks for nothing (logprob 0).
 * Outputs, device fp32 [rows], each optional: logprob = z[target] - lse; lse = log sum exp z; entropy =
 * -sum p log p; row_stats [rows][2] = (largest logit, log sum exp (z - its largest)), what the gradient needs:
 * lse in two parts, which keep their precision where every logit is near the type's lowest value.
 * top_ids, top_logprobs (both or neither): [rows][n_top] (n_top <= 64), the n_top largest logits in falling
 * order, ties to the lowest index, and their log probabilities.
 * A logit of -infinity is a token that cannot occur: it adds nothing, and the top list leaves it out; list
 * entries that remain read 0x7fffffff and -infinity. A row without a token that can occur has lse, logprob and
 * row_stats -infinity and entropy 0. A NaN or +infinity among a row's logits makes lse, entropy and every log
 * probability of the row NaN; NaN is listed nowhere. A target >= vocab: logprob NaN and err_word 4. */
#define JF_LOGPROBS_MAX_TOP 64
jf_status jf_op_token_logprobs_workspace_bytes(int rows, int vocab, int n_top, size_t* out_bytes);
jf_status jf_op_token_logprobs(int dtype, const void* logits, long long ld, int rows, int vocab, float scale,
                               const int32_t* targets, float* logprob, float* entropy, float* lse, float* row_stats,
                               int n_top, int32_t* top_ids, float* top_logprobs, void* workspace,
                               size_t workspace_bytes, int* err_word, void* cuda_stream);

/* Gradient of sum over rows of grad_logprob * logprob + grad_entropy * entropy (either may be NULL: 0) with
 * respect to the logits: scale * (grad_logprob * (1{i = target} - p_i) - grad_entropy * p_i * (log p_i +
 * entropy)). row_stats, entropy: jf_op_token_logprobs' outputs for the same logits, scale and targets (entropy
 * may be NULL without grad_entropy). grad_logits: [rows] of vocab values of the logits' dtype, rows ld_grad
 * elements apart; it may be logits itself (with ld_grad = ld). A negative target has no share of
 * grad_logprob. A logit of -infinity (p_i = 0) has gradient 0, or, where it is the target, scale * grad_logprob;
 * a row without a token that can occur has gradient 0. */
jf_status jf_op_token_logprobs_grad(int dtype, const void* logits, long long ld, int rows, int vocab, float scale,
                                    const int32_t* targets, const float* row_stats, const float* entropy,
                                    const float* grad_logprob, const float* grad_entropy, void* grad_logits,
                                    long long ld_grad, int* err_word, void* cuda_stream);

/* The clipped policy loss of given tokens, and its gradient. Logits, scale (here 1e-28 <= scale <= 1e30: below, masked
 * logits could not be told from the others) and targets as in jf_op_token_logprobs; with lp the target's log probability,
 * x = lp - old_logprob, ratio = e^x, A = advantage, d = ref_logprob - lp, H the row's entropy,
 *   loss = weight * (-min(ratio * A, min(max(ratio, 1 - below), 1 + above) * A) + kl * (e^d - 1 - d) - entropy * H).
 * The gradient is that of the sum of all losses by the logits; where both sides of a min or max are equal, the ratio's own.
 * old_logprob NULL: ratio 1, with the gradient of lp; ref_logprob NULL: kl must be 0; weight NULL: 1. All device fp32 [rows].
 * Outputs, device fp32 [rows], each optional: loss, logprob (lp), entropy (H), ratio, kl (e^d - 1 - d). grad_logits
 * (optional): [rows] of vocab values of the logits' dtype, rows ld_grad elements apart; it may be logits itself (with
 * ld_grad = ld), but not overlap them otherwise. rows <= 2^30.
 * A negative target leaves its row out: loss, logprob, ratio, kl and gradient 0 (entropy is the row's). A weight of 0 makes
 * loss and gradient 0 whatever the other terms are, and an advantage of 0 the first term. A target that cannot occur
 * (a logit of -infinity) has ratio 0 and, with a ref_logprob, an infinite kl; a kl beyond the range of fp32 (d above 88) is infinite
 * and has no gradient. Rows without a token that can occur, NaN
 * among the logits and targets >= vocab: as in jf_op_token_logprobs (the loss of the last is NaN, its gradient 0). A ratio
 * beyond the range of fp32 is infinite, as loss and gradient then are where A is negative; a logit whose token has probability 0 (in
 * fp32, below 2^-126 of the row's most likely one) has gradient 0 all the same, unless it is the target. A NaN in what a
 * row's loss is made of (old_logprob, advantage, weight, ref_logprob with kl, lp) makes loss and gradient NaN, the latter at tokens that can
 * occur; NaN among the logits makes the gradient NaN also where the loss does not depend on lp (no old_logprob).
 * workspace: device, 16-byte aligned, no initialisation needed; calls that may overlap on the GPU need one each. (0 bytes but for
 * rows longer than a cluster's shared memory, 230,400 fp32 or 460,800 bf16 values.) */
typedef struct {
  float below, above; /* how far the ratio counts on either side of 1: 0 <= below <= 1, 0 <= above */
  float kl, entropy;  /* factors of the two other terms */
} jf_policy_terms;
jf_status jf_op_policy_loss_workspace_bytes(int dtype, int rows, int vocab, size_t* out_bytes);
jf_status jf_op_policy_loss(const jf_policy_terms* terms, int dtype, const void* logits, long long ld, int rows, int vocab,
                            float scale, const int32_t* targets, const float* old_logprob, const float* ref_logprob,
                            const float* advantage, const float* weight, float* loss, float* logprob, float* entropy,
                            float* ratio, float* kl, void* grad_logits, long long ld_grad, void* workspace,
                            size_t workspace_bytes, int* err_word, void* cuda_stream);

/* A batch of texts that lie one behind the other in the rows of a call: text b has rows row_start[b] .. row_start[b+1]-1
 * (it may have none). row_start [n_seqs + 1] is a DEVICE array, ascending within 0 .. n_rows, read when the kernels run (a
 * captured graph follows it); n_rows and max_rows (no text is longer) are host numbers. Texts that are not so are reported
 * through err_word (as JF_EDEVICE's bounds code 4), and the call then computes nothing. Rows before the first text and
 * behind the last belong to none: their outputs and gradients are 0, their lse -infinity, and what they hold is used
 * nowhere. n_seqs <= 1024. */
typedef struct {
  const int32_t* row_start;
  int n_seqs, n_rows, max_rows;
} jf_packed;

/* Device workspace bytes of the two calls below on the current device (backward: 0 or 1; no initialisation needed; calls
 * that may overlap on the GPU need one each). */
jf_status jf_op_packed_attention_workspace_bytes(const jf_packed* texts, int dtype, int n_heads, int n_kv_heads, int head_dim,
                                                 int backward, size_t* out_bytes);

/* Causal attention of packed texts without a cache (prompts, trajectories, a training batch): out = softmax(scale * q k^T) v
 * for each of n_heads query heads (head h reads KV head h / (n_heads / n_kv_heads), at most 128 heads each), row i of a text
 * over its rows 0 .. i. dtype (JF_BF16 or JF_F32): type of everything but lse; head_dim 64 or 128. q, k, v: rows of n_heads
 * or n_kv_heads heads, ld_* elements apart, so that the three may be parts of one projection's rows; bf16 rows are read by tensor copies where
 * their addresses and ld_* are multiples of 16 bytes, by slower kernels otherwise. out: [n_rows][n_heads][head_dim], 16-byte aligned; lse (optional
 * here): fp32 [n_rows][n_heads], the natural logarithm of the sum of exponentials. Outputs may not overlap inputs or one another. |scale| <= 1e30. n_rows *
 * n_heads <= 2^30; more is refused (JF_EUNSUPPORTED), as are texts so long that the tiles of all scores pass 2^30.
 * Softmax statistics and sums are fp32; JF_BF16 rounds the probabilities (relative to a row's running maximum) to bf16
 * before their product with v. A NaN or an infinity in a text reaches rows of that text only. Results do not depend on the
 * order in which CTAs run; they depend in rounding on the batch, whose work is split evenly over the GPU. */
jf_status jf_op_packed_attention(const jf_packed* texts, int dtype, const void* q, long long ld_q, const void* k,
                                 long long ld_k, const void* v, long long ld_v, int n_heads, int n_kv_heads, int head_dim,
                                 float scale, void* out, float* lse, void* workspace, size_t workspace_bytes, int* err_word,
                                 void* cuda_stream);

/* Its backward pass: the gradients dq, dk, dv of a loss by q, k, v from that by out, d_out (rows ld_do elements apart), for
 * the same texts, q, k, v and scale and that call's out and lse. dq, dk, dv: rows ld_* elements apart (so that they may be
 * parts of one buffer's rows); they may not overlap the inputs or one another. dk and dv of a KV head are sums over its query heads. No
 * atomics: the order of every sum is fixed. JF_BF16 rounds probabilities and the scores' gradients to bf16 before their products
 * (the latter to two terms for dq in a text's first quarter and its first 512 rows, whose gradients are the largest), and takes the
 * product of d_out and out, which the scores' gradients contain, from out as given for dq of a text's rows with more than 128 keys, exactly
 * otherwise. For bf16 rows that tensor copies cannot read none of these is rounded. */
jf_status jf_op_packed_attention_grad(const jf_packed* texts, int dtype, const void* q, long long ld_q, const void* k,
                                      long long ld_k, const void* v, long long ld_v, int n_heads, int n_kv_heads, int head_dim,
                                      float scale, const void* out, const float* lse, const void* d_out, long long ld_do,
                                      void* dq, long long ld_dq, void* dk, long long ld_dk, void* dv, long long ld_dv,
                                      void* workspace, size_t workspace_bytes, int* err_word, void* cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* JF_OPS_H */
