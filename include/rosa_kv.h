/*
 * rosa_kv.h - operators on prefix caches: caches held in 4 bits, attention over
 * them with its log-sum-exp, the attention weight that cached tokens gather,
 * and the eviction of tokens by it.
 *
 * A prefix cache is what rosa.h's requests bring: per request one K and one V
 * array [L][P][n_kv][head_dim] in the model dtype.  It is what a server of
 * many robots keeps in memory per robot, so it pays to hold it in fewer bits
 * and to drop the tokens (image patches, mostly) that no action token looks at.
 *
 * Cache formats (rosa_kv_format)
 *  ROSA_KV_MODEL: the model dtype, as in rosa.h.
 *  ROSA_KV_FP4:   OCP MX blocks: each 32 consecutive elements along head_dim share
 *    one scale 2^e, and an element is one of
 *    +-{0, 0.5, 1, 1.5, 2, 3, 4, 6} 2^e (e2m1).  K and V are one array each of
 *    rosa_kv_bytes() bytes: the codes of all layers, [L][P][n_kv][head_dim / 2]
 *    bytes (element 2 i in the low four bits of byte i; bit 3 of a code is its
 *    sign), then the scales, [L][P][n_kv][head_dim / 32] bytes (e + 127; 255: the block is
 *    NaN).  17 / 32 byte per element instead of 2 or 4.
 *
 * Same conventions as rosa.h: pure C, noexcept, status returns, asynchronous
 * on the given stream or the handle's, all-or-nothing validation; a HIP
 * failure poisons a handle.  cfg gives L, the heads, head_dim, the dtype and the
 * attention layout, and is validated as by rosa_batch_create.  Device pointers
 * of caches, qkv and o are 16-byte aligned, of fp32 and int32 arrays 4-byte
 * aligned (ROSA_E_INVALID otherwise).  A function leaves the calling thread's
 * current device as it was.  A failure of a call without a handle is detailed by
 * rosa_kv_last_error(NULL).
 */
#ifndef ROSA_KV_H_
#define ROSA_KV_H_

#include "rosa.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum rosa_kv_format {
  ROSA_KV_MODEL = 0,
  ROSA_KV_FP4 = 1
} rosa_kv_format;

/* Bytes of one cache (K or V) of prefix_len tokens in `format`; -1 for a
 * configuration, format or length that is not valid. */
int64_t rosa_kv_bytes(const rosa_model_config *cfg, int32_t format, int32_t prefix_len);

/* ---------------------------------------------------------------- formats */

/* One request's caches, all layers.  DEVICE pointers; all may be NULL when
 * prefix_len is 0. */
typedef struct rosa_kv_job {
  const void *src_k, *src_v;   /* read */
  void       *dst_k, *dst_v;   /* written */
  int32_t     prefix_len;      /* P >= 0 */
  int32_t     reserved;        /* 0 */
} rosa_kv_job;

/* Model dtype (src) -> ROSA_KV_FP4 (dst).  Of a block with largest magnitude a,
 * e is the least integer with a <= 7 2^e, clamped to [-125, 125]; every
 * element becomes the nearest code (ties to the even code), magnitudes
 * above 6 2^e the largest.  A block with a NaN or an infinity becomes NaN (scale byte
 * 255, codes 0).  Of clamped blocks, values under 2^-127 become 0.
 * Deterministic, no memory, one launch per 64 jobs; capturable into a
 * graph.  Sources may be shared between jobs; a destination must not overlap
 * another destination or a source of the call.  n == 0 is a no-op.
 * Errors: ROSA_E_INVALID, ROSA_E_UNSUPPORTED (cfg), ROSA_E_DEVICE. */
rosa_status rosa_kv_quantize(const rosa_model_config *cfg, const rosa_kv_job *jobs, int32_t n, void *hip_stream);

/* ROSA_KV_FP4 (src) -> model dtype (dst): exact (every 4-bit value with scale bytes
 * 2 to 252, all that rosa_kv_quantize writes, is a normal bf16 number or zero). */
rosa_status rosa_kv_expand(const rosa_model_config *cfg, const rosa_kv_job *jobs, int32_t n, void *hip_stream);

/* ---------------------------------------------------------------- eviction */

/* One request's eviction.  Per (layer, KV head) `keep` of the P tokens stay:
 * the first `first` and the last `last` ones, and of the others those
 * with the largest mass (of equal masses the lowest index; a NaN counts less than
 * anything).  The kept tokens stay in order.  DEVICE pointers; they may be NULL
 * where they would hold nothing.
 *   mass:      [L][n_kv][P] fp32 (as rosa_kv_mass leaves it)
 *   kept:      [L][n_kv][keep] int32, written: the kept tokens' indices, ascending
 *   kept_mass: [L][n_kv][keep] fp32, written: their masses (so that a shortened
 *              cache goes on gathering); may be NULL
 *   dst_k, dst_v: caches of `keep` tokens in the same format, written       */
typedef struct rosa_kv_evict_job {
  const void  *src_k, *src_v;
  void        *dst_k, *dst_v;
  const float *mass;
  int32_t     *kept;
  float       *kept_mass;
  int32_t      prefix_len;     /* P >= 0 */
  int32_t      keep;           /* first + last <= keep <= P */
  int32_t      first, last;    /* >= 0 */
} rosa_kv_evict_job;

/* Evict n requests' tokens from caches in `format`.  Deterministic, no memory, two
 * launches per 32 jobs (three of 4-bit caches); capturable.  Nothing that is written may overlap
 * anything else the call reads or writes (so not in place).  Errors as
 * rosa_kv_quantize. */
rosa_status rosa_kv_evict(const rosa_model_config *cfg, int32_t format, const rosa_kv_evict_job *jobs, int32_t n,
                          void *hip_stream);

/* --------------------------------------------------- attention over the caches */

typedef struct rosa_kv rosa_kv;   /* opaque handle: a plan and its workspaces */

/* Create a handle for plans of up to `cap` (max_steps is not used but must be
 * valid).  All work is enqueued on hip_stream (NULL: the default stream).  A handle
 * needs no weights, only workspaces: the plan and the partial results of key
 * ranges split over several work items (2 x 512 slots of 256 rows and head_dim floats at
 * most).  Calls on one handle are ordered by its stream; handles share nothing,
 * so calls (or captured graphs) of different handles may overlap, of one
 * handle not.  Errors as rosa_batch_create; *out is NULL on failure. */
rosa_status rosa_kv_create(const rosa_model_config *cfg, const rosa_capacity *cap, void *hip_stream, rosa_kv **out);

/* Plan the attention of a request set, for every layer: prefix_k / prefix_v /
 * prefix_len / horizon of each request are read (the caches in `format`), the other
 * fields ignored.  mass: NULL, or a HOST array of n DEVICE pointers, each the
 * request's masses [L][n_kv][P] fp32 (NULL where P is 0), apart from each other and from the
 * caches (which requests may share).  The plan is copied to the
 * device on the handle's stream and replaces the last one; the arrays it names
 * must stay valid while calls use it.  Not under graph capture
 * (ROSA_E_INVALID); the calls below may be captured once a plan is there, and the graph
 * replayed until the next plan.  n == 0 is an empty plan.  Errors as
 * rosa_generate_actions for the requests. */
rosa_status rosa_kv_plan(rosa_kv *h, const rosa_request *reqs, int32_t n, int32_t format, float *const *mass);

/* The planned requests' attention at layer `layer`, as rosa_generate_actions
 * computes it at that layer: each action token of request r attends over r's prefix keys
 * and values of that layer (4-bit ones at the values they stand for), then r's own action keys
 * and values (ROSA_ATTN_ALTERNATING: prefix in even layers, action keys in odd ones).
 *   qkv: DEVICE [sum H][(n_q + 2 n_kv) head_dim], model dtype, the fused
 *        projection of the action tokens, rows in the plan's request order
 *   o:   DEVICE [sum H][n_q head_dim], model dtype, written
 *   lse: DEVICE [sum H][n_q] fp32, written: ln sum_j exp(q.k_j / sqrt(head_dim))
 *        over all keys the row attends to; may be NULL
 * o and lse may not overlap each other or what the call reads.
 * In the bf16 mode the softmax weights are rounded to bf16 for the product with the
 * values; statistics and sums are fp32.  Errors: ROSA_E_INVALID (no plan,
 * NULL or misaligned pointers, layer out of range), ROSA_E_DEVICE. */
rosa_status rosa_kv_attention(rosa_kv *h, int32_t layer, const void *qkv, void *o, float *lse);

/* The attention weight every cached token of layer `layer` gathers:
 *   mass[layer][kv head][j] (+)= sum over the action tokens and the KV head's
 *       query heads of exp(q.k_j / sqrt(head_dim) - lse)
 * into the arrays given to rosa_kv_plan; added to what they hold, or with
 * accumulate 0 in its place.  qkv as above, lse as rosa_kv_attention left it for the
 * same layer and qkv.  Sums are fp32 in a fixed order (deterministic).
 * Errors: as rosa_kv_attention; ROSA_E_INVALID where the plan has no masses or the
 * layer does not attend to the prefix. */
rosa_status rosa_kv_mass(rosa_kv *h, int32_t layer, const void *qkv, const float *lse, int32_t accumulate);

/* Wait for the handle's stream, then free everything.  NULL-safe. */
void rosa_kv_destroy(rosa_kv *h);

/* Detail of the last failure on this handle ("" if none); with h == NULL the
 * last failure of a create or of a call without a handle. */
const char *rosa_kv_last_error(const rosa_kv *h);

/* ------------------------------------------------------------------ generation */

/* rosa_generate_steps over prefix caches in `format`, optionally gathering masses:
 * with mass (a HOST array of n DEVICE pointers to [L][n_kv][P] fp32, or NULL; as
 * rosa_kv_plan) every attention launch that reads the prefix adds its tokens'
 * weights, over all steps the call runs.  A caller scores a set's prefixes on its
 * first Euler step, evicts, and runs the remaining steps over shorter
 * caches.  Masses do not change the generated actions beyond rounding (the
 * softmax denominators are then summed before the weights are rounded).
 * Errors as rosa_generate_steps, and ROSA_E_INVALID for a format, a mass pointer or
 * caches that are not 16-byte aligned. */
rosa_status rosa_generate_kv(rosa_batch *b, const rosa_request *reqs, int32_t n_reqs, int32_t max_steps,
                             int32_t format, float *const *mass);

#ifdef __cplusplus
}
#endif

#endif /* ROSA_KV_H_ */
