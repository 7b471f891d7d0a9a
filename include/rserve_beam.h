/*
 * rserve_beam.h -- several requests that continue one prompt, on the caches of rserve_prefill.h.
 *
 * Beam search, several answers to one prompt, requests behind a common prefix: what they have in common is prefilled once, and
 * their caches share its pages.
 *
 *   rs_beam_select   the best continuations of every group of beams, from logits and the beams' scores
 *   rs_kv_fork       caches become what other caches hold: on one pool they share its pages, else the tokens are copied
 *   rs_kv_compact    a cache keeps some of its tokens, and gives back the pages that this empties
 *
 * rs_attend (rserve_attend.h) reads pages that neighbouring requests of a call share once for all of them.
 *
 * Shared pages.  Nobody writes to a page that several caches hold.  A call that appends to a cache whose last block is shared and not
 * full (rs_prefill_*, rs_kv_append) gives it a page of its own first and copies the block's tokens, on its stream; the last holder
 * left keeps the page.  rs_kv_import* take pages of their own for all that is shared.  These pages count in what a call needs (RS_ECAPACITY).
 * Dropping, freeing and resetting caches give a page back to the pool when its last holder leaves it.
 *
 * The conventions of rserve_prefill.h and rserve_attend.h hold: the caller's memory and stream, errors on the host before anything
 * changes, one thread at a time per context and pool, caches of a pool on one stream or ordered by events.  A fork is a host-side change: what is
 * enqueued later, on any cache that shares pages, has to be ordered behind what the sources' pages still wait for.
 */
#ifndef RSERVE_BEAM_H
#define RSERVE_BEAM_H

#include "rserve_prefill.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- selection over beams and vocabulary
 * Rows b of a group (beams of them, group after group) hold the logits x_b of beam b's next token, and scores[b] is what the beam
 * has so far.  With m_b = max_t x_bt and S_b = sum_t exp(x_bt - m_b) the continuation of beam b by token t has
 *     score(b, t) = scores[b] + ((x_bt - m_b) - ln S_b)
 * and a group's n_select continuations with the largest scores come out, best first, equal ones in the order of (b, t):
 *   parents, tokens   device int32 [n_groups][n_select]: b in 0 .. beams - 1, and t
 *   out_scores        device fp32 [n_groups][n_select]
 * Scores are compared and added in 64 bits, out_scores is rounded once; the exponentials are summed in 32 bits, which leaves the logarithm
 * within 2^-17 (3e-8 in practice).
 * A beam whose score is not finite is out: its logits are not read.  A logit of minus infinity, or NaN, is a token that is not
 * allowed; one beyond the largest finite number counts as that number.  Where fewer than n_select continuations are left, the others
 * are -1, -1 and minus infinity.
 *   logits     device, fp32 or bf16 (rs_logits_type), [n_groups * beams][vocab], rows ld_logits elements apart; no alignment but the elements'
 *   scores     device fp32 [n_groups * beams]; may be what out_scores was of a call before, not of this one
 *   workspace  256-byte aligned, rs_beam_workspace_bytes
 * What is written, the workspace among it, overlaps neither logits or scores nor one another (RS_EINVAL).
 * 1 <= beams <= 64, 1 <= n_select <= 64, 1 <= vocab < 2^24, n_groups >= 0, n_groups * beams <= 65535 (RS_EINVAL).  Unlike the calls that look at caches this one stages nothing on
 * the host and may be captured into a HIP graph. */
typedef enum rs_logits_type { RS_LOGITS_F32 = 0, RS_LOGITS_BF16 = 1 } rs_logits_type;
size_t rs_beam_workspace_bytes(const rs_ctx* ctx, int n_groups, int beams, int vocab);
rs_status rs_beam_select(rs_ctx* ctx, const void* logits, int type, long ld_logits, int vocab, int n_groups, int beams, const float* scores,
                         int n_select, int* parents, int* tokens, float* out_scores, void* workspace, size_t workspace_bytes, void* hip_stream);

/* ---- forks
 * dsts[i] drops what it holds and becomes, in every layer, the first n_tokens[i] tokens of srcs[i] (null: all of each layer's; else at
 * most what the shortest layer holds, RS_EINVAL).  All sources are meant as they were before the call, so that caches may change places: the
 * beams' caches go with srcs[i] = caches[parents[i]], dsts = caches.  The caches of a pair have equally many layers and the same kind,
 * 8-bit ones the same scales (RS_EINVAL).  A cache is a destination once (RS_EINVAL).
 * Caches on one pool share its pages, and nothing is launched.  Between all others (contiguous ones, other pools) the tokens are
 * copied: RS_ECAPACITY without room, and a source that has to be copied is no other pair's destination (RS_EINVAL).  Where a launch of
 * these copies fails (RS_EHIP), destinations that are copied into are empty.
 * Bounds (rs_kv_attach_bounds) stay valid for blocks that the destination held already, in the same pages.
 *   rs_kv_shared_pages   pages of `layer` that other caches hold too (-1 on a bad argument; 0 for a contiguous cache) */
rs_status rs_kv_fork(rs_ctx* ctx, rs_kv* const* srcs, rs_kv* const* dsts, const int* n_tokens, int R, void* hip_stream);
int rs_kv_shared_pages(const rs_kv* kv, int layer);

/* ---- compaction
 * Slot j of request i's `layer` becomes what slot keep[j] held, for n_keep[i] slots, and that is its length: tokens that are not
 * needed any more (an image's, or those that no query looks at) leave the cache, and the pages this empties go back to the pool.
 *   keep     device int32, sum of n_keep: request 0's slots first, in any order (attention does not mind), the same one twice if so wished.  The host
 *            does not see them: a slot outside 0 .. rs_kv_len - 1 is the caller's error, and read as the nearest one inside.
 *   n_keep   host, 0 <= n_keep[i] <= max_pos, 0 where the cache is empty (RS_EINVAL)
 * Paged caches only (RS_ESTATE).  The kept tokens move to new pages, which the pool has to have (RS_ECAPACITY), while the old ones, or other
 * caches that share them, stay whole.  Keys keep the rotation they were cached with: a later token's rotary position is then not
 * its slot (rs_kv_append takes positions).  Bounds are taken anew. */
rs_status rs_kv_compact(rs_ctx* ctx, int layer, rs_kv* const* kvs, const int* keep, const int* n_keep, int R, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* RSERVE_BEAM_H */
