/*
 * rserve_attend.h -- operators on the KV caches of rserve_prefill.h, for callers that compute their own projections.
 *
 * rs_prefill_* (rserve_prefill.h) run a whole decoder layer of one fixed form.  What comes after a prompt, or beside it, often
 * has another form: the tokens a request generates one at a time, a few drafted tokens checked at once, layers with another
 * rotary form, adapters beside the projections, contexts so long that a token should read a part of them only.  Here are
 * the steps that touch the cache, on the same rs_ctx, rs_kv and rs_kv_pool:
 *
 *   rs_kv_append         rotates the new tokens' queries and keys, and stores keys and values into the caches
 *   rs_attend            attention of the new tokens over everything cached: single tokens, a few, or a chunk
 *   rs_kv_bounds_update  bounds on the keys of every finished 64-token block, 8 bits per element
 *   rs_attend_blocks     attention over the blocks that a cheap score from those bounds selects for each token and KV head
 *
 * They take caches of every kind (contiguous or paged, bfloat16 or 8-bit), may be mixed with rs_prefill_* on the same
 * caches, and follow that header's conventions: device memory belongs to the caller, work is enqueued on the caller's stream,
 * errors are decided on the host before anything is launched or changed, nothing allocates device memory (rs_rotary_create
 * excepted, and HIP's own bookkeeping), no call may be captured into a HIP graph (RS_ESTATE), results do not depend on
 * the order in which workgroups run, one thread at a time per rs_ctx.  Calls that share a cache or a workspace are ordered by their stream;
 * a caller that changes the stream between them orders the two with an event.  A call that finds no host memory returns RS_EHIP and
 * leaves the cached tokens as they are.
 *
 * Rows.  q, k, v, q_out and out hold one row per new token, the tokens of request 0 first: sum of lens rows.  A row of q, q_out and
 * out is [Hq][d], of k and v [Hkv][d], bfloat16, contiguous; ld_* is the distance between rows in elements, so that q, k
 * and v may be column ranges of one projection's output.  Pointers must be 16-byte aligned, ld_* multiples of 8 and no
 * smaller than a row.
 */
#ifndef RSERVE_ATTEND_H
#define RSERVE_ATTEND_H

#include "rserve_prefill.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- rotary positions
 * The first rotary_dim features of a head are turned in pairs, pair j of a token at position n by the angle n f_j:
 *     (a, b) -> magnitude * (a cos - b sin, b cos + a sin),   f_j = theta^(-2j / rotary_dim) before scaling
 * RS_ROTARY_HALVES pairs features j and j + rotary_dim/2, RS_ROTARY_INTERLEAVED features 2j and 2j + 1.  Other features pass
 * through.  Products and sums in fp32 from fp32 cosines and sines (of 64-bit angles), one rounding to bfloat16.
 * Frequency scaling for contexts beyond the one a model was trained on:
 *   RS_ROTARY_LINEAR  f / factor
 *   RS_ROTARY_RAMP    f / factor for the pairs that turn fewer than slow_turns times over original_max_pos positions, f for those
 *                     that turn more than fast_turns times, and between the two a mix that is linear in the pair's number:
 *                     pair(t) = rotary_dim ln(original_max_pos / (2 pi t)) / (2 ln theta), from floor(pair(fast_turns)) to
 *                     ceil(pair(slow_turns)).  magnitude = 0 stands for 0.1 ln(factor) + 1 here.
 *   RS_ROTARY_BANDS   with t = original_max_pos f / (2 pi) turns: f / factor for t <= slow_turns, f for t >= fast_turns,
 *                     between them f (1 - s) / factor + f s, s = (t - slow_turns) / (fast_turns - slow_turns)
 */
typedef enum rs_rotary_layout { RS_ROTARY_HALVES = 0, RS_ROTARY_INTERLEAVED = 1 } rs_rotary_layout;
typedef enum rs_rotary_scaling { RS_ROTARY_UNSCALED = 0, RS_ROTARY_LINEAR = 1, RS_ROTARY_RAMP = 2, RS_ROTARY_BANDS = 3 } rs_rotary_scaling;
typedef struct rs_rotary_cfg {
    int rotary_dim;        /* a multiple of 16, at most head_dim */
    int layout;            /* rs_rotary_layout */
    int max_pos;           /* positions 0 .. max_pos - 1 */
    int scaling;           /* rs_rotary_scaling */
    double theta;          /* > 1 */
    double factor;         /* >= 1 (scaled forms) */
    int original_max_pos;  /* > 0 (RAMP, BANDS) */
    double fast_turns;     /* 0: 32 (RAMP), 4 (BANDS) */
    double slow_turns;     /* 0: 1; below fast_turns */
    double magnitude;      /* 0: 1 (RAMP: see above) */
} rs_rotary_cfg;
typedef struct rs_rotary rs_rotary; /* host handle over a device table of max_pos * rotary_dim / 2 * 8 bytes, which rs_rotary_create allocates */
rs_status rs_rotary_create(rs_ctx* ctx, const rs_rotary_cfg* cfg, rs_rotary** out);
void rs_rotary_destroy(rs_rotary* rotary);
/* cos and sin of pair `pair` at position `pos` as the table holds them (host; what tests compare). */
rs_status rs_rotary_at(const rs_rotary* rotary, int pos, int pair, float* cos_out, float* sin_out);

/* ---- append
 * Request i's lens[i] >= 0 new tokens take cache slots first .. first + lens[i] - 1 of `layer`, and its length becomes first +
 * lens[i].  first = rs_kv_len, or starts[i] if `starts` is given: at most rs_kv_len, later tokens are dropped first (drafted
 * tokens that were not accepted; a paged cache keeps the pages that the new length needs).
 *   rotary     null: q and k are not turned
 *   positions  host array, a rotary position per row in [0, rotary max_pos) (RS_ECAPACITY otherwise); null: the cache slots.
 *              Behind rs_prefill_*_mrope a token's position is not its slot, and has to be given.  One number a row is a token whose three
 *              axes agree, as text's do; tokens whose axes differ are appended by rs_prefill_*_mrope alone.
 *   q, q_out   queries before and after the rotation; q_out may be q (with ld_q_out = ld_q); both null: keys and values only
 * 8-bit caches store codes of the bfloat16 rows, as everywhere.  What the cache holds is the same bits as if the tokens came
 * one by one.  RS_ECAPACITY as in rs_prefill_batch. */
rs_status rs_kv_append(rs_ctx* ctx, const rs_rotary* rotary, int layer, rs_kv* const* kvs, const int* starts, const int* lens, int R,
                       const int* positions, const void* q, long ld_q, const void* k, long ld_k, const void* v, long ld_v,
                       void* q_out, long ld_q_out, void* hip_stream);

/* ---- attention
 * Row t of request i is the query at cache slot rs_kv_len - lens[i] + t (its key and value are cached already) and attends to
 * the slots up to its own:  out = sum_k softmax_k(scale q . key_k) value_k,  per head, query head h on KV head h / (Hq / Hkv).
 * lens[i] <= rs_kv_len (RS_EINVAL).  scale: 0 stands for 1 / sqrt(head_dim), else positive and
 * finite, and so, in fp32, is scale log2(e) times an 8-bit cache's keys' scale (RS_EINVAL).  out may be q, with
 * ld_out = ld_q (RS_EINVAL); rows of out that overlap q in any other way are the caller's error.
 * Scores, softmax statistics and sums are fp32, the softmax's weights enter the second product as bfloat16, the output is
 * rounded once.  What a query does not see does not reach it, infinities and NaN included.
 * Requests of few rows (rows * Hq / Hkv <= 64, or more where little is cached) read 8-bit caches directly; longer ones expand the codes
 * that they see to bfloat16 in the workspace first.  A code is exact there, and the scales enter the softmax's scale and the output, so
 * that either way a key or value is code * scale (rs_prefill_* round that to bfloat16).
 * RS_ATTEND_FEW=n, a TEST-ONLY environment variable read in rs_ctx_create, replaces the size up to which "more rows" are few (0: never).
 *   workspace   256-byte aligned, rs_attend_workspace_bytes:
 *     max_rows, max_requests   of a call
 *     max_visible_fp8          8-bit caches in calls with longer requests: the sum of their cached tokens, else 0
 *     n_blocks                 rs_attend_blocks calls: its n_blocks, else 0 */
size_t rs_attend_workspace_bytes(const rs_ctx* ctx, int max_rows, int max_requests, size_t max_visible_fp8, int n_blocks);
rs_status rs_attend(rs_ctx* ctx, int layer, rs_kv* const* kvs, const int* lens, int R, const void* q, long ld_q, void* out, long ld_out,
                    float scale, void* workspace, size_t workspace_bytes, void* hip_stream);

/* ---- bounds on the keys of finished blocks
 * Of block b (slots 64 b .. 64 b + 63, all filled) and KV head, per feature j the largest and smallest element of the 64 keys,
 * as the cache stores them (8-bit caches: fl32(code * scale)); elements beyond +-2^100 count as +-2^100, NaN as 0.  unit = 2^e
 * with the smallest e >= -100 that keeps the largest magnitude within 127 units;  high_j = ceil(largest / unit), low_j =
 * floor(smallest / unit), int8.  So  sum_j max(q_j high_j, q_j low_j) * unit  bounds q . key from above for every key.
 *   rs_kv_attach_bounds   gives a cache memory for them: codes int8 [n_layers][Hkv][n_blocks][2][d] (high, low; 16-byte aligned),
 *                         units fp32 [n_layers][Hkv][n_blocks], both the caller's.  n_blocks: room, in blocks of 64 tokens.
 *                         codes = units = null takes the memory away.  A cache starts with no block covered.
 *   rs_kv_bounded         blocks of `layer` whose bounds are there (-1 on a bad argument): dropping tokens, rs_kv_import* and
 *                         rs_kv_reset take back those of the blocks they touch
 *   rs_kv_bounds_update   computes the bounds of every request's finished blocks that have none yet, or, with firsts (host
 *                         array), of those from slot firsts[i] on.  RS_ESTATE without memory, RS_ECAPACITY beyond its room. */
rs_status rs_kv_attach_bounds(rs_kv* kv, void* codes_dev, void* units_dev, int n_blocks);
int rs_kv_bounded(const rs_kv* kv, int layer);
rs_status rs_kv_bounds_update(rs_ctx* ctx, int layer, rs_kv* const* kvs, const int* firsts, int R, void* hip_stream);

/* ---- attention over selected blocks
 * As rs_attend, but the query of slot p (block b0 = p / 64) sees, per KV head, the slots up to its own of at most n_blocks
 * blocks: the first n_first and the last n_last up to b0 (n_last >= 1: its own is among them), and of the others those with the best
 * scores, ties to the lower block.  (If these first and last ones are more than n_blocks, the lowest of them.)
 *   score of a block = unit * sum_j (p_j high_j + n_j low_j), exact in whole numbers until the product with unit, where p and n
 *   are the group's queries in 8 bits: the g heads' elements (beyond +-2^100 as +-2^100, NaN as 0) are rounded, ties to even, to
 *   codes of their common unit, chosen as above; positive and negative codes are added up over the heads and divided by
 *   2^ceil(log2 g), halves away from zero.
 * It is, up to that rounding, the sum over the group's heads of the bound on a key's score.  Bounds that are missing are
 * computed first, in the same call (one launch more).
 *   chosen   device int32 [rows][Hkv][n_blocks]: the blocks, ascending, -1 behind the last; null: not wanted
 * 1 <= n_blocks <= 1024, 0 <= n_first, 1 <= n_last. */
rs_status rs_attend_blocks(rs_ctx* ctx, int layer, rs_kv* const* kvs, const int* lens, int R, const void* q, long ld_q, void* out, long ld_out,
                           int n_blocks, int n_first, int n_last, float scale, int* chosen, void* workspace, size_t workspace_bytes,
                           void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* RSERVE_ATTEND_H */
