/*
 * klpm_kv.h -- the KV cache behind the radix tree: C ABI of the operators that fill it, read it and shorten it (sm_100a).
 *
 * klpm.h schedules prompts against a tree of cached prefixes; what the tree keeps of a prompt stands for keys and values on
 * the GPU.  The calls here are the ones an engine makes around the scheduler in each step:
 *
 *   rt_prefix_slots (klpm.h)   where the cached tokens of a matched prompt are: a page table with pages of one token
 *   kv_rope_append             rotary positions on new tokens' queries and keys; keys and values into the cache
 *   kv_decode                  attention of one new token per sequence over the cache, optionally with the attention weight that
 *                              every cached token received
 *   kv_evict                   a sequence shortened to the tokens with the largest accumulated weight
 *
 * Conventions are those of klpm.h: d_* pointers are the caller's device memory, work is enqueued on `stream` (a cudaStream_t; NULL =
 * the default stream) of the CURRENT device, entry points do not wait, allocate nothing, keep nothing between calls, and may be
 * captured into a graph.  Argument errors found on the host return RT_ERR_INVALID (RT_ERR_TOO_LARGE for sizes) and enqueue
 * nothing.  Calls on different streams may overlap on the GPU unless one writes what the other uses; a workspace belongs to one
 * call at a time (two captured graphs that may run at the same time need a workspace each).
 *
 * Sums, softmax statistics and rotations are held in 32-bit floating point (rotation angles in 64) and rounded once, when stored; kv_decode
 * rounds probabilities, and bf16 queries next to an 8-bit cache, on the way (see there).
 */
#ifndef KLPM_KV_H_
#define KLPM_KV_H_

#include <stdint.h>
#include "klpm.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { KV_F32 = 0, KV_BF16 = 1, KV_F16 = 2, KV_E4M3 = 3 };

#define KV_MAX_HEAD_DIM 256
#define KV_MAX_PAGE_SIZE 65536

/* A paged cache: element d of head h of the token at place t of page p is k[p * k_stride[0] + t * k_stride[1] + h * k_stride[2] + d]
 * (strides in elements; heads before tokens in memory or after, as the strides say).  A token's slot is p * page_size + t.
 *   dtype      KV_BF16, KV_F16 or KV_E4M3; an 8-bit element stands for its value times k_scale (v_scale).  The scales of the 16-bit
 *              types are 1.
 *   page_size  a power of two, at most KV_MAX_PAGE_SIZE
 *   head_dim   a multiple of 16 bytes, at most KV_MAX_HEAD_DIM elements
 * Bases and strides are multiples of 16 bytes.  n_pages * page_size is at most 2^31 - 1 (of one sequence's table, max_pages *
 * page_size at most 2^30).  A stride of a dimension with more than one
 * entry is at least head_dim; rows do not overlap. */
typedef struct {
    void* k;
    void* v;
    int32_t dtype;
    int32_t n_pages, page_size, n_heads, head_dim;
    float k_scale, v_scale;
    int64_t k_stride[3], v_stride[3];
} kv_cache;

/* Rows of heads outside the cache: element d of head h of row r is data[r * stride[0] + h * stride[1] + d] (strides in elements;
 * the number of rows is the call's).  Any alignment that the type itself needs.  Rows that are written (out, q_out, and likewise those of
 * d_weight in kv_decode and d_new_weight) lie apart from one another: RT_ERR_INVALID where their strides let two share memory. */
typedef struct {
    void* data;
    int32_t dtype;     /* KV_F32, KV_BF16 or KV_F16 */
    int32_t n_heads;
    int64_t stride[2];
} kv_rows;

/* Rotary positions.  The first rot_dim (even, 2 <= rot_dim <= head_dim) elements of a head are rotated, the rest is copied.  Pair i is
 * (2i, 2i+1) if interleaved, else (i, i + rot_dim/2); at position p it is turned by p * d_turns[i] whole turns (d_turns: double[rot_dim/2],
 * see kv_rope_table) and multiplied by factor. */
typedef struct {
    const double* d_turns;
    int32_t rot_dim;
    int32_t interleaved;
    float factor;
} kv_rope;

enum { KV_ROPE_PLAIN = 0, KV_ROPE_LINEAR = 1, KV_ROPE_NTK = 2, KV_ROPE_YARN = 3 };

/* Fill d_turns (double[rot_dim/2]) with theta^(-2i/rot_dim) / (2 pi), scaled for contexts `scale` (>= 1) times as long as the
 * original_len tokens the frequencies were made for:
 *   KV_ROPE_LINEAR  positions divided by scale
 *   KV_ROPE_NTK     theta * scale^(rot_dim / (rot_dim - 2)): the slowest pair is slowed by scale, the fastest not at all
 *   KV_ROPE_YARN    pairs that turn more than beta_fast times within original_len are kept, those that turn less than beta_slow times
 *                   are divided by scale, linear in the number of turns in between (YaRN, arXiv 2309.00071); *factor becomes 0.1 ln(scale) + 1.
 *                   Programs that ramp over the pair's number instead (between the two pairs' numbers, often rounded) have other frequencies:
 *                   a model made with those needs a d_turns of its own, which the caller may fill as it likes
 * *factor (host, nullable) is 1 otherwise. */
rt_status kv_rope_table(double* d_turns, int32_t rot_dim, double theta, int32_t scaling, double scale, double original_len,
                        double beta_fast, double beta_slow, float* factor, void* stream);

/* For i < n: rotate head rows q[i] (nullable) into q_out[i] and k[i] by d_positions[i] (rope NULL: no rotation, d_positions may be
 * NULL), and store k[i], v[i] at slot d_slots[i] of the cache (divided by the scale and rounded to the nearest; 8-bit values saturate at
 * +-448, NaN stays NaN).  q, q_out, k and v have one dtype; it is the cache's, or the cache's is KV_E4M3, or it is KV_F32.
 * q_out may be q itself; otherwise they must not overlap, nor may the cache's k and v.  A slot outside [0, n_pages * page_size) (a padded row) is not stored; its
 * query is rotated all the same.  No slot may occur twice in a call (each element of such a slot is one of the two rows'). */
rt_status kv_rope_append(const kv_cache* cache, const kv_rope* rope, const int32_t* d_positions, const int32_t* d_slots, int32_t n,
                         const kv_rows* q, const kv_rows* q_out, const kv_rows* k, const kv_rows* v, void* stream);

/* Bytes of workspace that kv_decode needs for these sizes (negative: an rt_status). */
int64_t kv_decode_workspace(const kv_cache* cache, int32_t n_seqs, int32_t n_q_heads, int32_t max_pages, int32_t with_weight);

/* Attention of one new token for each of n_seqs sequences: for query head h of sequence b, over the tokens t of the sequence,
 *   s_t = scale * q[b,h] . k_t,  out[b,h] = sum_t softmax(s)_t v_t,  d_lse[b,h] = ln sum_t exp(s_t)
 * with keys and values of cache head h / (n_q_heads / cache->n_heads).  Token t of sequence b is at place t % page_size of page
 * d_page_table[b * table_stride + t / page_size], t < d_lengths[b] (clamped to [0, max_pages * page_size]); with window > 0 only
 * the last `window` tokens are attended to.  A page number outside [0, n_pages) is a page that is not there: its tokens are masked.
 * Masked tokens are not read.  A sequence with nothing to attend to gets out 0 and lse -inf.
 * Several sequences may name the same page.
 *   d_lse     nullable, float[n_seqs, n_q_heads]
 *   d_weight  nullable: d_weight[b * weight_stride[0] + g * weight_stride[1] + t] += the sum over the query heads of cache head g of
 *             their softmax weights of token t (max_pages * page_size entries per row; those of masked tokens stay as they are)
 *   q, out    one dtype: the cache's, or either 16-bit type if the cache is KV_E4M3.  They must not overlap.
 *   n_seqs    at most 65,535 (so for kv_evict)
 *   d_workspace  kv_decode_workspace bytes, aligned to 256; its contents before and after the call mean nothing.  With d_weight it holds
 *             n_seqs * n_q_heads * max_pages * page_size scores of 4 bytes, whatever d_lengths says (128 sequences, 32 heads, tables for 131,072
 *             tokens: 2.1 GB): tables no wider than the longest sequence save most of it
 * The result is the same for every call with the same arguments (no atomics on floating-point values).
 * Roundings on the way: a probability enters the sum of values as the sum of two 16-bit numbers, off by 2^-16 of it at most next to a bf16 cache, else by
 * 2^-22 of it, or 2^-39 of the row's largest if that is more; a bf16 query next to an 8-bit cache has elements off by 2^-39 of the head's largest at most.
 * Range: q . k before it is scaled (of a bf16 query next to an 8-bit cache: scale * k_scale times its largest element) has to stay within 32-bit floating
 * point.  So do sums of values, which are formed before they are divided by the softmax's sum: the number of tokens times the largest value, times 2^15 for f16 and 8-bit caches.
 * Infinite and NaN keys or values of tokens that are attended to come out as the formula says: an infinite value makes the output infinite however small
 * its probability, and with the other infinity, or if it is NaN, NaN; a token whose score is -inf takes no part, whatever its value.  They cost
 * time, see decode_repair in csrc/klpm_kv.cu: a few times a call's, some hundred times only where a token with a score of -inf has such a value. */
rt_status kv_decode(const kv_cache* cache, const kv_rows* q, const kv_rows* out, int32_t n_seqs, const int32_t* d_page_table,
                    int64_t table_stride, int32_t max_pages, const int32_t* d_lengths, float scale, int32_t window, float* d_lse,
                    float* d_weight, const int64_t* weight_stride, void* d_workspace, int64_t workspace_bytes, void* stream);

/* Shorten sequences to `keep` tokens.  For each sequence b and cache head g, of the tokens that are there (as in kv_decode), at most
 * keep are kept: the first `sinks` and the last `recent` positions of the sequence (sinks + recent <= keep), then those with the
 * largest d_weight[b * weight_stride[0] + g * weight_stride[1] + t], the lowest t among equals (-0 equals 0; NaN ranks below every number).
 * In order of position, kept token j of head g is copied to place j % page_size of page d_new_table[b * new_stride + j / page_size]
 * (new_pages * page_size >= keep), and
 *   d_index       int32[n_seqs, n_heads, keep]: its t; -1 behind the last one
 *   d_new_weight  [b * new_weight_stride[0] + g * new_weight_stride[1] + j]: its weight; 0 behind the last one, up to new_weight_len (>= keep)
 *   d_new_lengths int32[n_seqs]: how many were kept
 * A new page outside [0, n_pages) receives nothing.  No new page may be one that d_page_table names (in any row up to its length), nor occur
 * twice: tokens are copied in no order.  (Pages that other sequences share stay as they are; the caller drops its own old
 * pages.)  d_new_weight must not overlap d_weight. */
rt_status kv_evict(const kv_cache* cache, const float* d_weight, const int64_t* weight_stride, int32_t n_seqs,
                   const int32_t* d_page_table, int64_t table_stride, int32_t max_pages, const int32_t* d_lengths,
                   const int32_t* d_new_table, int64_t new_stride, int32_t new_pages, int32_t keep, int32_t sinks, int32_t recent,
                   int32_t* d_index, float* d_new_weight, const int64_t* new_weight_stride, int32_t new_weight_len,
                   int32_t* d_new_lengths, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* KLPM_KV_H_ */
