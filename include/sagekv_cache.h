/* sagekv_cache.h - operators on the FULL cache, the one that the eviction pass of sagekv.h reads.
 *
 * Around the eviction pass a program rotates queries and keys by their positions, writes the keys and values of
 * prompts and generated tokens into the full cache (between two refreshes too, see sagekv.h), and attends over the
 * full cache where nothing has been evicted yet: short sequences, layers that keep everything, or, with a window given, sink
 * and recent tokens only.  These are the calls for that.  They share the conventions of sagekv.h (device pointers
 * owned by the caller, host descriptors, everything enqueued on `hip_stream`, no allocation and no synchronisation, return codes checked
 * before anything is launched, calls can be recorded into a HIP graph); their names start with sagekvc_.
 *
 * A full cache is either dense, K[p][c][t][j] at p*stride_problem + c*stride_head + t*stride_token + j (elements), or paged as
 * in sagekv_select_paged: the same head and token strides inside a page, a block table per problem; a token's stride is less than 2^24 bytes.  Here a problem is
 * one sequence (or one layer of one), and every problem has its own length.
 */
#ifndef SAGEKV_CACHE_H
#define SAGEKV_CACHE_H

#include "sagekv.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- rotary positions -------------------------------------------------------------------------- */

/* Which two elements of a head form pair j: HALF (j, j + rotary_dim/2), PAIRS (2j, 2j+1). */
typedef enum { SAGEKVC_ROTARY_HALF = 0, SAGEKVC_ROTARY_PAIRS = 1 } sagekvc_rotary_layout;

/* A rotation by positions.  With a = pos * inv_freq[j], pair j = (x, y) becomes
 *     (amplitude * (x cos a - y sin a), amplitude * (y cos a + x sin a));
 * elements from rotary_dim on are copied as they are.  transpose: the sign of a is turned, which is the gradient's
 * rotation (and, with amplitude 1, the inverse).  Angles are formed and reduced in fp64, so that positions of a million and
 * more lose nothing; cosines, sines and products are fp32, rounded once to the element type. */
typedef struct {
  int32_t rotary_dim;       /* even, 2 <= rotary_dim <= head_dim                                 */
  int32_t layout;           /* sagekvc_rotary_layout                                             */
  int32_t transpose;        /* 0 or 1                                                            */
  float amplitude;          /* 1 unless the long-context scaling has one                          */
  const double* inv_freq;   /* DEVICE, [rotary_dim / 2] radians per position                      */
} sagekvc_rotary_map;

/* Frequencies base^(-2j / rotary_dim), optionally stretched for contexts longer than a model was trained on:
 *   LINEAR  every frequency / factor;
 *   PARTS   by the turns a pair makes over the original length, n = original_len * f / (2 pi): f / factor where n < low, f where n > high, between them
 *           mixed in proportion to n (Llama 3.1: factor 8, low 1, high 4, original_len 8192);
 *   YARN    the same two ends (YaRN, arXiv 2309.00071: low = 1, high = 32), mixed in proportion to the pair's index between the (real) indices at which a pair
 *           makes `high` and `low` turns, the first rounded down, the second up, both kept within [0, rotary_dim - 1]; amplitude 0.1 ln(factor) + 1.
 * Host only: inv_freq and amplitude are HOST memory; copy the frequencies to the device. */
typedef enum {
  SAGEKVC_SCALING_NONE = 0, SAGEKVC_SCALING_LINEAR = 1, SAGEKVC_SCALING_PARTS = 2, SAGEKVC_SCALING_YARN = 3
} sagekvc_scaling_kind;
typedef struct {
  int32_t kind;             /* sagekvc_scaling_kind; NONE ignores the rest                          */
  double factor;            /* >= 1                                                               */
  double low, high;         /* PARTS, YARN: turns, 0 < low < high                                   */
  double original_len;      /* PARTS, YARN: > 0                                                     */
} sagekvc_rotary_scaling;
sagekv_status sagekvc_rotary_frequencies(int32_t rotary_dim, double base /* > 1 */, const sagekvc_rotary_scaling* scaling /* null: none */,
                                         double* inv_freq, float* amplitude);

/* Rotates the heads of n_tokens tokens.  Strides in ELEMENTS, multiples of 16 bytes, rows 16-byte aligned as everywhere; a
 * stride of x may be 0.  out may be x itself (with the same strides); otherwise they must not overlap, nor may out's own rows. */
typedef struct {
  int64_t n_tokens;         /* 0 <= n_tokens <= 2^25; 0: nothing is done                            */
  int32_t n_heads;          /* >= 1                                                               */
  int32_t head_dim;         /* 64 or 128                                                          */
  int32_t dtype;            /* sagekv_dtype of x and out                                           */
  int64_t x_stride_token, x_stride_head;
  int64_t out_stride_token, out_stride_head;
} sagekvc_rotary_desc;
/* positions: device int32 [n_tokens], any values. */
sagekv_status sagekvc_rotary(const sagekvc_rotary_desc* desc, const sagekvc_rotary_map* rotary, const void* x,
                             const int32_t* positions, void* out, void* hip_stream);

/* ---- the full cache ----------------------------------------------------------------------------- */
typedef struct {
  int32_t n_problems;       /* sequences; n_problems * n_kv_heads <= 65535                        */
  int32_t n_q_heads, n_kv_heads, head_dim, dtype; /* as in sagekv_select_desc; n_q_heads a multiple of n_kv_heads (up to 64 times) */
  int64_t capacity;         /* tokens a problem has room for, up to 2^30; paged: at most table_pitch * page_size */
  int64_t k_stride_problem; /* elements; *_stride_problem: dense caches only                       */
  int64_t k_stride_head;
  int64_t k_stride_token;
  int64_t v_stride_problem;
  int64_t v_stride_head;
  int64_t v_stride_token;
} sagekvc_desc;

/* New tokens of a call, packed: rows of q, k_new, v_new (often slices of one projection's output) and of q_out. */
typedef struct {
  int64_t n_tokens;         /* 0 <= n_tokens <= 2^25                                              */
  int64_t q_stride_token, q_stride_head;   /* elements, multiples of 16 bytes; inputs' strides may be 0 */
  int64_t k_stride_token, k_stride_head;
  int64_t v_stride_token, v_stride_head;
  int64_t q_out_stride_token, q_out_stride_head;
} sagekvc_tokens;

/* Writes new tokens into the cache, keys rotated on the way, and rotates their queries: what stands between a layer's projections and
 * its attention, for prompts (any number of them, of any lengths, whole or in chunks) and for generated tokens alike.
 *   token_offsets  device int32 [n_problems + 1], not decreasing: rows [token_offsets[p], token_offsets[p+1]) are problem p's new tokens, in
 *                  order; a problem may have none.  Rows from n_tokens on do not exist.  NULL: one new token per problem, n_tokens = n_problems.
 *   seq_lens       device int32 [n_problems]: the problems' lengths WITH their new tokens (as sagekvc_attn takes them next), so
 *                  the i-th of n_p new tokens gets place seq_lens[p] - n_p + i.
 *   positions      device int32 [n_tokens], the rotation's positions; NULL: the places.
 *   rotary         NULL: keys are written, and queries copied, as they are.
 *   q, q_out       both NULL: no queries.  q_out may be q (with the same strides).
 * K[p][c][place] = rotated k_new[t][c], V[p][c][place] = v_new[t][c], q_out[t] = rotated q[t].  Nothing else is touched: rows of no problem (in front of
 * token_offsets[0], from token_offsets[n_problems] on) are left out entirely, and a token whose place lies outside [0, capacity) (an unused
 * slot of a batch with seq_lens 0, a full cache) or in a page whose table entry lies outside [0, n_pages) (a page shared with another
 * problem, say, marked -1) is not stored, while its query is rotated.  Pages written to must be distinct, and the caches must not overlap the inputs. */
sagekv_status sagekvc_write(const sagekvc_desc* desc, const sagekv_paged_kv* pages /* NULL: dense */, const sagekvc_tokens* tokens,
                            const sagekvc_rotary_map* rotary, const void* q, const void* k_new, const void* v_new,
                            const int32_t* token_offsets, const int32_t* seq_lens, const int32_t* positions, void* q_out, void* K, void* V,
                            void* hip_stream);

/* Attention of one new token per problem over the full cache:
 *     out[p][h] = sum_t softmax_t( q[p][h] . K[p][c][t] / sqrt(head_dim) ) V[p][c][t],   c = h / G,   t in [0, len_p),
 * len_p = seq_lens[p] kept within [0, max_len], and, where n_recent > 0, only the tokens t < n_sink and t >= len_p - n_recent (sink and recent
 * window over a cache from which nothing has been evicted).  n_recent = 0 (and n_sink = 0): every token.
 *   q         [n_problems, n_q_heads, head_dim] contiguous;
 *   seq_lens  device int32 [n_problems], read by the launch (one recorded graph serves growing sequences), not to be changed while it runs;
 *   max_len   the longest length any problem may have at the launch, 1 <= max_len <= capacity;
 *   out       [n_problems, n_q_heads, head_dim] fp32, contiguous;
 *   lse       nullable, [n_problems, n_q_heads] fp32: log of the sum of exp(logits), with which two parts of a row can be joined.
 * A problem that attends nothing (length 0) gets out = 0 and lse = -infinity.  What the cache holds in places that are not attended (pages' ends, an
 * evicted middle) does not matter, whatever it is; table entries are kept within [0, n_pages), pages may be shared.  Products are exact, softmax weights and
 * sums fp32 with a bf16 cache; logits and sums fp64 with an fp32 one.
 * workspace: sagekvc_attn_workspace_bytes(desc), any contents; two calls that may run at the same time need one each. */
size_t sagekvc_attn_workspace_bytes(const sagekvc_desc* desc);
sagekv_status sagekvc_attn(const sagekvc_desc* desc, const sagekv_paged_kv* pages /* NULL: dense */, const void* q, const void* K, const void* V,
                           const int32_t* seq_lens, int32_t max_len, int32_t n_sink, int32_t n_recent, float* out, float* lse,
                           void* workspace, size_t workspace_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif
