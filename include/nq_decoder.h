/*
 * nq_decoder.h -- C ABI of the operators between the binary layers of a decoder (nq_binlr.h) on one MI355X (gfx950): what one
 * step of decoding does with the outputs of the q, k, v layers and with the logits.
 *
 *     nq_rope_*    norm of every query and key head, rotary positions, store of keys and values into a paged cache; and the
 *                  backward of norm and rotation
 *     nq_attn_*    attention of new tokens -- one, a tree of drafted ones, a chunk of a prompt -- over the paged cache
 *     nq_sample    next tokens from logits: temperature, top-k, top-p, min-p, from given uniform numbers
 *     nq_kv_*      the paged cache itself: its description, copies of pages, compaction of accepted drafts
 *
 * The streaming layers cost the same for one token and for eight, so a step that verifies several drafted tokens is nearly as
 * cheap as one that adds a single token; these operators are written for such steps.
 *
 * Conventions are those of nq_binlr.h (status codes, nq_last_error_string(), streams; nothing here synchronises or allocates device
 * memory except nq_rope_create).  All tensors are device memory of the current device, owned by the caller.  Element types are
 * NQ_F32, NQ_F16, NQ_BF16.  Strides are in elements; a stride between tokens may be any value of at least a token's length, so that
 * q, k and v may be columns of one wider tensor.  Query, key and value pointers need the alignment of an element only.  Every call
 * may be captured in a HIP graph.  Integers in device memory cannot be refused by the host: where one is out of range the kernels
 * stay inside the caller's buffers as stated with each argument.
 */
#ifndef NQ_DECODER_H
#define NQ_DECODER_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct nq_kv_s*   nq_kv;     /* the description of one layer's paged cache */
typedef struct nq_rope_s* nq_rope;   /* head layout, frequencies and types of norm and rotation */
typedef struct nq_attn_s* nq_attn;   /* attention over one nq_kv */

#define NQ_MAX_HEAD_DIM 256

/* ---- the paged cache of one layer ----
 * k, v: device, NQ_F16 or NQ_BF16, 16-byte aligned.  Element d of the key of head h in slot s of page p is
 * k[p page_stride + s slot_stride + h head_stride + d], the values' likewise in v.  A sequence's token i is in slot
 * i % page_size of page table[i / page_size].  page_size: a power of two, 16 to 1024; head_dim: a multiple of 8, 8 to
 * NQ_MAX_HEAD_DIM; strides: multiples of 8 elements that keep the elements apart (each at least the extent of the next smaller
 * one), a page spanning less than 2 GiB.  0, 0, 0 stands for [n_pages][kv_heads][page_size][head_dim].  Host only; the memory stays the caller's
 * and has to outlive the calls that use it. */
int nq_kv_create(nq_kv* out, void* k, void* v, int dtype, int kv_heads, int head_dim, int page_size, int64_t n_pages,
                 int64_t page_stride, int64_t slot_stride, int64_t head_stride);
int nq_kv_destroy(nq_kv kv);

/* Copies whole pages, keys and values, in all of the n caches (the layers of a model: same shape, strides and type): page src[i] to
 * page dst[i], i < n_pairs.  What a fork of a sequence does with its last, partly filled page.
 * kvs: host array of n handles; src, dst: device int32.  No page may be a dst twice, nor both a src and a dst (the results are then
 * unspecified).  A pair with a page outside the cache is left out.  Asynchronous on `stream`. */
int nq_kv_copy_pages(const nq_kv* kvs, int n, const int32_t* src, const int32_t* dst, int n_pairs, void* stream);

/* Moves the accepted drafts of n_seqs sequences together, keys and values, in all of the n caches (same shape, strides and type): slot
 * ctx_len[s] + path[s path_stride + j] to slot ctx_len[s] + j for j < path_len[s], as if everything were read before anything is
 * written.  path must rise strictly from j to j + 1 and path_len <= path_stride.  page_table: device int32 [n_seqs][table_stride]; sequences must not share the pages
 * written.  A move whose slot is beyond the table, or whose page is outside the cache, is left out.  Asynchronous on `stream`. */
int nq_kv_compact(const nq_kv* kvs, int n, const int32_t* ctx_len, const int32_t* page_table, int64_t table_stride, const int32_t* path,
                  int64_t path_stride, const int32_t* path_len, int n_seqs, void* stream);

/* ---- norm and rotary positions ----
 * For every head x of q and of k, in 32 bits, rounded once at the end:
 *     n = x / sqrt(mean(x^2) + eps) (.) (w + weight_offset)          w NULL: n = x
 *     (y_a, y_b) = magnitude (n_a cos t - n_b sin t, n_a sin t + n_b cos t),   t = position * inv_freq[i]
 * for the rot_dim / 2 pairs (a, b) = (i, i + rot_dim / 2) (NQ_ROPE_HALF) or (2i, 2i + 1) (NQ_ROPE_INTERLEAVED); elements from rot_dim
 * on are n.  t is formed and reduced by 2 pi in binary64: far positions of long contexts lose nothing. */
#define NQ_ROPE_HALF        0
#define NQ_ROPE_INTERLEAVED 1

/* Frequencies for contexts longer than a model was trained on.  Host only.  Writes rot_dim / 2 values to inv_freq and the magnitude that
 * goes with them.  With f_i = base^(-2 i / rot_dim):
 *   NQ_ROPE_PLAIN    f_i                                                                  (factor etc. are not looked at)
 *   NQ_ROPE_LINEAR   f_i / factor
 *   NQ_ROPE_BASE     f_i of the base  base * factor^(rot_dim / (rot_dim - 2))             (rot_dim > 2)
 *   NQ_ROPE_YARN     f_i (1 - g_i) / factor + f_i g_i; g_i falls on a straight line in i from 1 to 0 between the pairs that turn
 *                    `high` and `low` times (rounded down and up, kept within 0 .. rot_dim - 1) over trained_len positions;
 *                    magnitude 0.1 ln(factor) + 1
 *   NQ_ROPE_BANDED   f_i where trained_len f_i / 2 pi > high, f_i / factor where it is < low, between them
 *                    f_i ((1 - g) / factor + g), g = (trained_len f_i / 2 pi - low) / (high - low)
 * factor >= 1, base > 1, trained_len >= 1, 0 < low < high. */
#define NQ_ROPE_PLAIN  0
#define NQ_ROPE_LINEAR 1
#define NQ_ROPE_BASE   2
#define NQ_ROPE_YARN   3
#define NQ_ROPE_BANDED 4
int nq_rope_freqs(int kind, int rot_dim, double base, double factor, double trained_len, double low, double high, double* inv_freq, double* magnitude);

/* inv_freq: host, rot_dim / 2 finite values, copied to the current device.  head_dim as in nq_kv_create; rot_dim: even, 0 to head_dim;
 * q_heads a multiple of kv_heads.  in_dtype: q, k, v and their gradients; out_dtype: the results and the upstream gradients. */
int nq_rope_create(nq_rope* out, int q_heads, int kv_heads, int head_dim, int rot_dim, int layout, const double* inv_freq, double magnitude,
                   double eps, double weight_offset, int in_dtype, int out_dtype);
int nq_rope_destroy(nq_rope r);

/* q: [n_tokens][q_heads * head_dim], k: [n_tokens][kv_heads * head_dim]; q_out, k_out alike.  q_weight, k_weight: float [head_dim]
 * or NULL (that tensor is not normalised).  positions: int32 [n_tokens].  An output may be its input (same pointer, stride and type).
 * n_tokens 0 does nothing. */
int nq_rope_forward(nq_rope r, const void* q, int64_t q_stride, const void* k, int64_t k_stride, const float* q_weight, const float* k_weight,
                    const int32_t* positions, int n_tokens, void* q_out, int64_t q_out_stride, void* k_out, int64_t k_out_stride, void* stream);

/* The same with the keys' results and the values (converted to the cache's type) stored in the cache, whose type is the handle's
 * out_dtype: token t in slot slots[t] % page_size of page slots[t] / page_size.  A token whose slot is negative or beyond the cache is not stored (its
 * query is still written).  slots: int64 [n_tokens], no slot twice. */
int nq_rope_cache(nq_rope r, nq_kv kv, const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                  const float* q_weight, const float* k_weight, const int32_t* positions, const int64_t* slots, int n_tokens, void* q_out,
                  int64_t q_out_stride, void* stream);

/* Gradients: dq, dk (in_dtype) from the upstream dq_out, dk_out (out_dtype) and the inputs of the forward; dq_weight, dk_weight: float
 * [head_dim], fully overwritten, both sums over all tokens and heads in a fixed order (NULL where the weight is NULL, or not wanted).
 * dq may be dq_out and dk dk_out where types and strides agree.  workspace: 16-byte aligned, at least
 * nq_rope_backward_workspace_bytes(r, n_tokens).  n_tokens 0 clears the weights' gradients. */
int nq_rope_backward_workspace_bytes(nq_rope r, int n_tokens, size_t* bytes);
int nq_rope_backward(nq_rope r, const void* q, int64_t q_stride, const void* k, int64_t k_stride, const float* q_weight, const float* k_weight,
                     const int32_t* positions, int n_tokens, const void* dq_out, int64_t dq_out_stride, const void* dk_out,
                     int64_t dk_out_stride, void* dq, int64_t dq_stride, void* dk, int64_t dk_stride, float* dq_weight, float* dk_weight,
                     void* workspace, size_t workspace_bytes, void* stream);

/* ---- attention of new tokens over the cache ----
 * New token t (0 .. n_s - 1) of sequence s sees the ctx_len[s] cached tokens and those of the sequence's new tokens j that its row of
 * `tree` names (bit j % 32 of word j / 32, the packed format of nq_pack_signs; bits past the row are 0), or all j <= t where tree is NULL.
 * Keys and values of the new tokens are in the cache already, at ctx_len[s] + j.  Query head h reads key head h / (q_heads / kv_heads).
 *     a = scale q . k,   a = cap tanh(a / cap) where cap > 0,    out = sum p v / sum p,  p = exp(a - max a),   lse = ln sum exp a
 * over the visible keys.  A row that sees nothing gives zeros and lse = -inf.  What it does not see never reaches a row, whatever it holds
 * (NaN, infinities, memory that was never written).  Scores, statistics and sums are held in 32 bits; the probabilities are rounded to the
 * cache's type for the product with v, in parts that add up: to 16 bits and more for 16-bit results, 22 and more for NQ_F32 ones.  Only calls with
 * more than 64 rows (new tokens times q_heads / kv_heads) to a sequence on average, whose results are of the cache's type or NQ_BF16, have a single part,
 * 8 bits of an NQ_BF16 cache, 11 of an NQ_F16 one: the results are then about as far from binary64 again as their own rounding leaves them (2-norm: 2.3e-3 instead of 1.7e-3
 * for NQ_BF16).  Who wants those finer asks for NQ_F32 results. */

/* out_dtype: of the results; q has the cache's type.  Copies what it needs of kv (which may be destroyed).  q_heads a multiple of the cache's kv_heads.
 * scale finite, cap 0 or above; scale, cap and scale / cap have to be numbers of fp32 (about 1e-38 to 2e38).  Host only. */
int nq_attn_create(nq_attn* out, nq_kv kv, int q_heads, double scale, double cap, int out_dtype);
int nq_attn_destroy(nq_attn a);
/* Workspace of a call with n_seqs sequences and n_tokens new tokens in all; it serves every call with fewer of either as well. */
int nq_attn_workspace_bytes(nq_attn a, int n_seqs, int n_tokens, size_t* bytes);
/* q: [n_tokens][q_heads * head_dim] of the cache's type;  out: [n_tokens][q_heads * head_dim] of out_dtype;  lse: float [n_tokens][q_heads] or
 * NULL.  new_begin: int32 [n_seqs + 1], sequence s has the new tokens new_begin[s] .. new_begin[s + 1] - 1 (rising from 0 to n_tokens; values
 * beyond are cut, and where it does not rise rows may be left unwritten).  ctx_len: int32 [n_seqs].  page_table: int32 [n_seqs][table_stride]; tokens beyond the table are not seen, a page outside the cache is
 * read as one inside it.  tree: [n_tokens][tree_words] or NULL.  workspace: 16-byte aligned.  n_tokens 0 does nothing. */
int nq_attn_forward(nq_attn a, const void* q, int64_t q_stride, const int32_t* new_begin, const int32_t* ctx_len, const int32_t* page_table,
                    int64_t table_stride, const uint32_t* tree, int tree_words, int n_seqs, int n_tokens, void* out, int64_t out_stride, float* lse,
                    void* workspace, size_t workspace_bytes, void* stream);

/* ---- next tokens from logits ----
 * For every row of logits, in the order of falling logits (equal ones: lowest index first), with z = (x - max x) / temperature and the weights
 * w = round(2^31 exp(z)), whole numbers whose sums are exact in any order:
 *     keep the first top_k tokens                                    (top_k <= 0: all)
 *     of these, tokens as long as the weights before them sum to less than top_p times the weight of all of them      (top_p >= 1: all)
 *     of these, tokens with exp(z) >= min_p                           (the first token is always kept)
 *     take the first token at which the sum of kept weights, its own included, exceeds floor(uniform * their total)
 * temperature 0 takes the first token.  logprob: ln of the token's probability under the kept distribution.  A row whose largest logit is NaN or
 * -inf, or that holds a NaN, or whose temperature is negative or NaN gives token -1 and logprob NaN; +inf logits share the row among them.
 * logits: [n_rows][vocab] of dtype with row_stride elements between rows; temperature, top_p, min_p, uniform: float [n_rows]; top_k: int32
 * [n_rows]; temperature, top_k, top_p and min_p may be NULL (1, 0, 1, 0).  uniform in [0, 1).  tokens: int32 [n_rows]; logprobs: float [n_rows] or
 * NULL.  vocab <= 2^20.  workspace: 16-byte aligned, nq_sample_workspace_bytes(n_rows, vocab), which serves every call of fewer rows or tokens as well.
 * n_rows 0 does nothing. */
#define NQ_MAX_VOCAB (1 << 20)
int nq_sample_workspace_bytes(int n_rows, int64_t vocab, size_t* bytes);
int nq_sample(const void* logits, int dtype, int n_rows, int64_t vocab, int64_t row_stride, const float* temperature, const int32_t* top_k,
              const float* top_p, const float* min_p, const float* uniform, int32_t* tokens, float* logprobs, void* workspace, size_t workspace_bytes,
              void* stream);

#ifdef __cplusplus
}
#endif
#endif
