// Host side of include/rserve_beam.h: argument checks, the caches' pages, descriptors and launches.
#include "../../include/rserve_beam.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstring>
#include <exception>
#include <tuple>
#include <vector>

#include "beam_select.h"
#include "cache_calls.h"
#include "host_state.h"
#include "kv_move.h"
#include "last_error.h"

namespace {

// ---------------------------------------------------------------- moves
// A layer's tokens on their way from one cache to another, or within one.
struct Move {
    TilePlaces from, to;
    const std::vector<int>*from_pages, *to_pages;   // null: contiguous
    int n, len, keep0;
};
int blocks_of(int tokens) { return (tokens + 63) / 64; }
size_t pages_of(const Move& m) { return (m.from_pages ? blocks_of(m.len) : 0) + (m.to_pages ? blocks_of(m.n) : 0); }

// keep: a compaction's; null: copies, those of one source side by side, the longest last.
rs_status launch_moves(rs_ctx* ctx, bool fp8, const std::vector<Move>& moves, const int* keep, hipStream_t st) {
    const size_t staged_pages = ctx->slot_bytes / 4;
    for (size_t i0 = 0; i0 < moves.size();) {
        size_t i1 = i0, pages = 0;
        while (i1 < moves.size() && (size_t)move_reqs_at((int)(i1 + 1 - i0)) + MOVE_WORDS * (i1 + 1 - i0) <= TABLE_WORDS && pages + pages_of(moves[i1]) <= staged_pages)
            pages += pages_of(moves[i1++]);
        if (i1 == i0) return fail(RS_EINVAL, "internal: descriptor sizing");
        const int n = (int)(i1 - i0);
        const size_t words = (size_t)move_reqs_at(n) + MOVE_WORDS * (size_t)n;
        const bool inside = words + pages <= TABLE_WORDS;   // page numbers beside the requests, or read where they are staged
        InlineTable tab;
        int slot = 0;
        rs_status s;
        RingUse ring(ctx, st);
        if (!inside && (s = ring.acquire(&slot)) != RS_OK) return s;
        uint32_t* const numbers = inside ? tab.w + words : reinterpret_cast<uint32_t*>(ctx->pinned[slot]);
        MoveArgs a{};
        a.n_req = n;
        a.hkv = ctx->cfg.n_kv_heads;
        a.pages = inside ? nullptr : reinterpret_cast<const uint32_t*>(ctx->pinned_dev[slot]);
        a.keep = keep;
        int at = 0, before = 0;
        uint32_t items = 0, first = 0, most = 0;
        const auto side = [&](const TilePlaces& p, const std::vector<int>* list, int blocks) {
            MoveSide m{p.k, p.v, p.head_bytes, p.block_bytes, CONTIGUOUS};
            if (list) {
                m.pages = at;
                for (int b = 0; b < blocks; ++b) numbers[at++] = (uint32_t)(*list)[b];
            }
            return m;
        };
        for (int j = 0; j < n; ++j) {
            const Move& m = moves[i0 + j];
            MoveReq q{};
            q.from = side(m.from, m.from_pages, blocks_of(m.len));
            q.to = side(m.to, m.to_pages, blocks_of(m.n));
            q.n = m.n; q.len = m.len; q.keep0 = m.keep0;
            const bool again = !keep && j > 0 && m.from_pages == moves[i0 + j - 1].from_pages && m.from.k == moves[i0 + j - 1].from.k;
            before = again ? before + 1 : 0;
            if (!again) {
                first = items;
                most = 0;
            }
            q.before = before;
            tab.w[j] = first;
            memcpy(&tab.w[move_reqs_at(n) + MOVE_WORDS * j], &q, sizeof(q));
            most = std::max(most, (uint32_t)blocks_of(m.n));
            items = first + most;
        }
        a.heads = inside ? 1 : a.hkv;
        const unsigned groups = (unsigned)(a.hkv / a.heads);
        with_table(tab, words + (inside ? pages : 0), [&](const auto& table) {
            typedef std::decay_t<decltype(table)> Tab;
            for_kind(ctx, fp8, [&](auto d, auto f8) {
                constexpr int D = decltype(d)::value;
                constexpr bool FP8 = decltype(f8)::value;
                if (keep) hipLaunchKernelGGL((kv_compact_kernel<D, FP8, Tab>), dim3(items, groups + groups * (D / COMPACT_ROWS)), dim3(256), 0, st, a, table);
                else hipLaunchKernelGGL((kv_copy_kernel<D, FP8, Tab>), dim3(items, 2u * a.hkv * CopyPiece<D, FP8>::PIECES), dim3(256), 0, st, a, table);
            });
        });
        RS_HIP(hipGetLastError());
        if (!inside && (s = ring.commit()) != RS_OK) return s;
        i0 = i1;
    }
    return RS_OK;
}

// ---------------------------------------------------------------- selection
struct BeamLayout {
    size_t rows, sums_at, total;
};
BeamLayout beam_layout(int n_groups, int beams, int segments) {
    BeamLayout w;
    w.rows = (size_t)n_groups * beams;
    w.sums_at = align_up(w.rows * segments * sizeof(float), 256);
    w.total = w.sums_at + align_up(w.rows * ((segments + BEAM_WAVES - 1) / BEAM_WAVES) * sizeof(float2), 256);
    return w;
}
rs_status check_beams(int n_groups, int beams, int vocab) {
    if (n_groups < 0) return fail(RS_EINVAL, "n_groups = %d is negative", n_groups);
    if (beams < 1 || beams > BEAM_MAX) return fail(RS_EINVAL, "beams = %d must be 1 .. %d", beams, BEAM_MAX);
    if (vocab < 1 || vocab >= 1 << 24) return fail(RS_EINVAL, "vocab = %d must be at least 1 and below 2^24", vocab);
    if ((long)n_groups * beams > 65535) return fail(RS_EINVAL, "%ld rows: more than 65535", (long)n_groups * beams);
    return RS_OK;
}

template <typename T>
rs_status select_launch(const rs_ctx* ctx, BeamArgs a, int n_groups, char* ws, hipStream_t st) {
    const int rows = n_groups * a.beams;
    a.segments = beam_segments<T>(a.vocab);
    a.maxima = reinterpret_cast<float*>(ws);
    a.sums = reinterpret_cast<float2*>(ws + beam_layout(n_groups, a.beams, a.segments).sums_at);
    const auto scan = [&](auto e) {
        constexpr int E = decltype(e)::value;
        a.stretches = (a.segments + BEAM_WAVES * E - 1) / (BEAM_WAVES * E);
        hipLaunchKernelGGL((beam_scan_kernel<T, E>), dim3(a.stretches, rows), dim3(BEAM_THREADS), 0, st, a);
    };
    // segments of a wavefront: as many as leave every compute unit four workgroups.  us a pass with one / eight / as many: 1 group of 4 beams of
    // 32000 10.1 / 12.1 / 10.2, 24 of 5 of 50001 in bfloat16 14.2 / 16.6 / 14.3, 16 of 8 of 152064 27.2 / 25.0 / 25.0, 32 of 8 39.1 / 35.3 / 35.3
    const long segments = (long)rows * a.segments;
    const auto leaves = [&](int e) { return segments / (BEAM_WAVES * e) >= 4L * ctx->n_cu; };
    if (leaves(8)) scan(std::integral_constant<int, 8>{});
    else if (leaves(4)) scan(std::integral_constant<int, 4>{});
    else if (leaves(2)) scan(std::integral_constant<int, 2>{});
    else scan(std::integral_constant<int, 1>{});
    if (a.beams * a.segments <= 4 * BEAM_THREADS) hipLaunchKernelGGL((beam_pick_kernel<T, 4>), dim3(n_groups), dim3(BEAM_THREADS), 0, st, a);
    else hipLaunchKernelGGL((beam_pick_kernel<T, 20>), dim3(n_groups), dim3(BEAM_THREADS), 0, st, a);
    RS_HIP(hipGetLastError());
    return RS_OK;
}
bool overlap(const void* a, size_t na, const void* b, size_t nb) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x < y + nb && y < x + na;
}

}  // namespace

rs_status launch_page_copies(const rs_ctx* ctx, bool fp8, const std::vector<PageCopy>& copies, hipStream_t st) {
    constexpr size_t MOST = TABLE_WORDS / (sizeof(PageCopy) / 4);
    for (size_t i0 = 0; i0 < copies.size(); i0 += MOST) {
        const size_t n = std::min(MOST, copies.size() - i0), words = n * (sizeof(PageCopy) / 4);
        InlineTable tab;
        memcpy(tab.w, &copies[i0], n * sizeof(PageCopy));
        with_table(tab, words, [&](const auto& table) {
            for_kind(ctx, fp8, [&](auto d, auto f8) {
                hipLaunchKernelGGL((page_copy_kernel<decltype(d)::value, decltype(f8)::value, std::decay_t<decltype(table)>>),
                                   dim3((unsigned)n, 2 * ctx->cfg.n_kv_heads), dim3(256), 0, st, ctx->cfg.n_kv_heads, table);
            });
        });
        RS_HIP(hipGetLastError());
    }
    return RS_OK;
}

extern "C" {

// =============================================================================================== selection
size_t rs_beam_workspace_bytes(const rs_ctx* ctx, int n_groups, int beams, int vocab) {
    if (!ctx || n_groups < 1 || beams < 1 || beams > BEAM_MAX || vocab < 1 || vocab >= 1 << 24 || (long)n_groups * beams > 65535) return 0;
    return beam_layout(n_groups, beams, std::max(beam_segments<float>(vocab), beam_segments<bf16>(vocab))).total;
}

rs_status rs_beam_select(rs_ctx* ctx, const void* logits, int type, long ld_logits, int vocab, int n_groups, int beams, const float* scores,
                         int n_select, int* parents, int* tokens, float* out_scores, void* workspace, size_t workspace_bytes, void* stream) {
    if (!ctx) return fail(RS_EINVAL, "ctx is null");
    rs_status s = check_beams(n_groups, beams, vocab);
    if (s != RS_OK) return s;
    if (type != RS_LOGITS_F32 && type != RS_LOGITS_BF16) return fail(RS_EINVAL, "type %d", type);
    if (n_select < 1 || n_select > BEAM_MAX) return fail(RS_EINVAL, "n_select = %d must be 1 .. %d", n_select, BEAM_MAX);
    if (n_groups == 0) return RS_OK;
    const size_t el = type == RS_LOGITS_F32 ? 4 : 2, rows = (size_t)n_groups * beams, out = (size_t)n_groups * n_select * 4;
    if (!logits || !scores || !parents || !tokens || !out_scores) return fail(RS_EINVAL, "logits / scores / parents / tokens / out_scores is null");
    if (!aligned(logits, el) || !aligned(scores, 4) || !aligned(parents, 4) || !aligned(tokens, 4) || !aligned(out_scores, 4))
        return fail(RS_EINVAL, "logits, scores, parents, tokens and out_scores must be aligned to their elements");
    if (rows > 1 && ld_logits < vocab) return fail(RS_EINVAL, "ld_logits = %ld is smaller than a row (%d)", ld_logits, vocab);
    const size_t need = rs_beam_workspace_bytes(ctx, n_groups, beams, vocab);
    if (!workspace) return fail(RS_EINVAL, "workspace is null");
    if (!aligned(workspace, 256)) return fail(RS_EINVAL, "workspace must be 256-byte aligned");
    if (workspace_bytes < need) return fail(RS_EWORKSPACE, "workspace has %zu bytes, this call needs %zu (rs_beam_workspace_bytes)", workspace_bytes, need);
    // (a workgroup's results would be logits or scores that another has yet to read, or another's results)
    const std::pair<const void*, size_t> written[] = {{parents, out}, {tokens, out}, {out_scores, out}, {workspace, need}};
    for (const auto& x : written) {
        if (overlap(x.first, x.second, scores, rows * 4) || overlap(x.first, x.second, logits, ((rows - 1) * (size_t)ld_logits + vocab) * el))
            return fail(RS_EINVAL, "parents, tokens, out_scores and workspace must not overlap logits or scores");
        for (const auto& y : written)
            if (&x != &y && overlap(x.first, x.second, y.first, y.second))
                return fail(RS_EINVAL, "parents, tokens, out_scores and workspace must not overlap one another");
    }
    if ((s = check_device(ctx)) != RS_OK) return s;
    BeamArgs a{};
    a.logits = logits; a.ld = ld_logits; a.vocab = vocab; a.beams = beams; a.n_select = n_select;
    a.scores = scores;
    a.parents = parents; a.tokens = tokens; a.out_scores = out_scores;
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    return type == RS_LOGITS_F32 ? select_launch<float>(ctx, a, n_groups, (char*)workspace, st) : select_launch<bf16>(ctx, a, n_groups, (char*)workspace, st);
}

// =============================================================================================== forks
int rs_kv_shared_pages(const rs_kv* kv, int layer) {
    if (!kv || layer < 0 || layer >= kv->n_layers) return -1;
    if (!kv->paged()) return 0;
    int n = 0;
    for (int page : kv->pages[layer]) n += kv->pool->shared(page);
    return n;
}

rs_status rs_kv_fork(rs_ctx* ctx, rs_kv* const* srcs, rs_kv* const* dsts, const int* n_tokens, int R, void* stream) try {
    if (!ctx) return fail(RS_EINVAL, "ctx is null");
    if (R < 0) return fail(RS_EINVAL, "R = %d is negative", R);
    if (R > 0 && (!srcs || !dsts)) return fail(RS_EINVAL, "srcs / dsts is null");
    const auto shares = [&](int i) { return srcs[i]->paged() && srcs[i]->pool == dsts[i]->pool; };
    const auto tokens = [&](int i, int layer) { return n_tokens ? n_tokens[i] : srcs[i]->len[layer]; };
    PageNeed need;
    bool moving = false, copying = false;   // a pair that does not share; with tokens
    for (int i = 0; i < R; ++i) {
        const rs_kv *src = srcs[i], *dst = dsts[i];
        if (!src || !dst) return fail(RS_EINVAL, "srcs[%d] / dsts[%d] is null", i, i);
        if (src->ctx != ctx || dst->ctx != ctx) return fail(RS_ESTATE, "srcs[%d] / dsts[%d] belongs to another context", i, i);
        if (src->n_layers != dst->n_layers) return fail(RS_EINVAL, "srcs[%d] has %d layers, dsts[%d] %d", i, src->n_layers, i, dst->n_layers);
        if (src->fp8 != dst->fp8 || src->k_scale != dst->k_scale || src->v_scale != dst->v_scale)
            return fail(RS_EINVAL, "srcs[%d] and dsts[%d] are not of one kind, or their scales differ", i, i);
        if (src->fp8 != srcs[0]->fp8) return fail(RS_EINVAL, "srcs[%d]: the caches of one call must all be bfloat16 or all be 8-bit", i);
        moving |= !shares(i) && src != dst;
        for (int l = 0; l < src->n_layers; ++l) {
            if (n_tokens && (n_tokens[i] < 0 || n_tokens[i] > src->len[l]))
                return fail(RS_EINVAL, "n_tokens[%d] = %d outside [0, %d] of layer %d", i, n_tokens[i], src->len[l], l);
            if (shares(i) || src == dst) continue;
            if (!dst->paged() && tokens(i, l) > dst->cap) return fail(RS_ECAPACITY, "pair %d: %d tokens exceed cache capacity %d", i, tokens(i, l), dst->cap);
            if (dst->paged()) need.add(dst->pool, dst->pages_to_replace(l, tokens(i, l)));
            copying |= tokens(i, l) > 0;
        }
    }
    // a destination is one once; what is copied is neither overwritten before, nor a source of another pair behind it
    if (twice(ctx, dsts, R)) return fail(RS_EINVAL, "the same rs_kv is a destination twice");
    std::vector<const rs_kv*> to, from;
    if (moving) {
        to.assign(dsts, dsts + R);
        from.assign(srcs, srcs + R);
        std::sort(to.begin(), to.end());
        std::sort(from.begin(), from.end());
    }
    for (int i = 0; i < R && moving; ++i) {
        if (shares(i) || srcs[i] == dsts[i]) continue;
        if (std::binary_search(to.begin(), to.end(), srcs[i])) return fail(RS_EINVAL, "srcs[%d] has to be copied, and is another pair's destination", i);
        if (std::binary_search(from.begin(), from.end(), dsts[i])) return fail(RS_EINVAL, "dsts[%d] is copied into, and is another pair's source", i);
    }
    rs_status s = need.check();
    if (s != RS_OK) return s;
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    if (copying) {
        if ((s = check_device(ctx)) != RS_OK) return s;
        if ((s = refuse_capture(st)) != RS_OK) return s;
    }
    // host memory first.  Of a list of pages that is shared only what differs from what the destination holds matters - beams that change places
    // have their prompt in common -, and is kept apart until all sources have been looked at.
    struct Shared { int pair, layer, n, same, first; };   // blocks that stay, place of the others in `others`
    std::vector<Shared> shared;
    std::vector<int> others;
    std::vector<Move> moves;
    for (int i = 0; i < R; ++i)
        for (int l = 0; l < srcs[i]->n_layers; ++l) {
            const int n = tokens(i, l), blocks = blocks_of(n);
            std::vector<int>& held = dsts[i]->pages.empty() ? others : dsts[i]->pages[l];
            if (shares(i)) {
                const std::vector<int>& from = srcs[i]->pages[l];
                const int most = std::min<int>(blocks, (int)held.size());
                const int same = pages_in_common(from.data(), held.data(), most);
                shared.push_back(Shared{i, l, n, same, (int)others.size()});
                others.insert(others.end(), from.begin() + same, from.begin() + blocks);
                if ((int)held.capacity() < blocks) held.reserve(blocks + 8);   // (tokens to come)
            } else if (srcs[i] != dsts[i]) {
                if (dsts[i]->paged()) held.reserve(blocks);
                if (n > 0) moves.push_back(Move{places_of(srcs[i], l), places_of(dsts[i], l), srcs[i]->paged() ? &srcs[i]->pages[l] : nullptr,
                                                dsts[i]->paged() ? &held : nullptr, n, n, 0});
            }
        }
    std::vector<char> stale(shared.size());
    for (size_t j = 0; j < shared.size(); ++j) {
        const rs_kv* const src = srcs[shared[j].pair];
        stale[j] = shared[j].n % 64 != 0 && (shared[j].n < src->len[shared[j].layer] || src->stale_tail[shared[j].layer]);
    }
    // ---- from here on the call is made
    for (const Shared& x : shared)
        for (int b = x.same; b < blocks_of(x.n); ++b) ++srcs[x.pair]->pool->holders[others[x.first + b - x.same]];
    for (size_t j = shared.size(); j-- > 0;) {   // (backwards: what comes back is taken in the same order again)
        const Shared& x = shared[j];
        rs_kv* const dst = dsts[x.pair];
        std::vector<int>& held = dst->pages[x.layer];
        dst->bounded[x.layer] = std::min(dst->bounded[x.layer], std::min(x.same, x.n / 64));
        dst->give_back_pages(x.layer, 64L * x.same);
        held.insert(held.end(), others.begin() + x.first, others.begin() + x.first + (blocks_of(x.n) - x.same));
        dst->len[x.layer] = x.n;
        dst->stale_tail[x.layer] = stale[j];
    }
    for (int i = 0; i < R; ++i) {
        if (shares(i)) continue;
        rs_kv* const dst = dsts[i];
        for (int l = 0; l < dst->n_layers; ++l) {
            const int n = tokens(i, l);
            if (srcs[i] == dst) {   // (contiguous: tokens dropped)
                dst->dropped_from(l, n);
                dst->len[l] = n;
                continue;
            }
            if (dst->paged()) dst->replace_pages(l, n);
            dst->dropped_from(l, 0);
            dst->len[l] = n;
            dst->stale_tail[l] = 0;
        }
    }
    if (moves.empty()) return RS_OK;
    std::sort(moves.begin(), moves.end(), [](const Move& x, const Move& y) {   // by source and length (what lands where does not depend on their order)
        return std::make_tuple((uintptr_t)x.from_pages, x.from.k, x.n) < std::make_tuple((uintptr_t)y.from_pages, y.from.k, y.n);
    });
    if ((s = launch_moves(ctx, srcs[0]->fp8, moves, nullptr, st)) == RS_OK) return RS_OK;
    for (int i = 0; i < R; ++i) {   // nobody knows what has been copied
        if (shares(i) || srcs[i] == dsts[i]) continue;
        for (int l = 0; l < dsts[i]->n_layers; ++l) {
            dsts[i]->len[l] = 0;
            if (dsts[i]->paged()) dsts[i]->give_back_pages(l, 0);
        }
    }
    return s;
} catch (const std::exception& e) {
    return not_allocated(e);
}

// =============================================================================================== compaction
rs_status rs_kv_compact(rs_ctx* ctx, int layer, rs_kv* const* kvs, const int* keep, const int* n_keep, int R, void* stream) try {
    rs_status s = check_call(ctx, layer, kvs, nullptr, false, R, nullptr);
    if (s != RS_OK) return s;
    if (R > 0 && !n_keep) return fail(RS_EINVAL, "n_keep is null");
    PageNeed need;
    long kept = 0;
    for (int i = 0; i < R; ++i) {
        if (!kvs[i]->paged()) return fail(RS_ESTATE, "kvs[%d] is contiguous: it has no pages to give back", i);
        if (n_keep[i] < 0 || n_keep[i] > ctx->cfg.max_pos || (n_keep[i] > 0 && kvs[i]->len[layer] == 0))
            return fail(RS_EINVAL, "n_keep[%d] = %d of %d cached tokens", i, n_keep[i], kvs[i]->len[layer]);
        need.add(kvs[i]->pool, blocks_of(n_keep[i]));
        kept += n_keep[i];
    }
    if (kept > 0x7fffffff) return fail(RS_EINVAL, "%ld tokens to keep: more than 2^31 - 1", kept);
    if (kept > 0 && (!keep || !aligned(keep, 4))) return fail(RS_EINVAL, "keep is null or not 4-byte aligned");
    if ((s = need.check()) != RS_OK) return s;
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    if (kept > 0) {
        if ((s = check_device(ctx)) != RS_OK) return s;
        if ((s = refuse_capture(st)) != RS_OK) return s;
    }
    std::vector<std::vector<int>> pages(R);
    std::vector<Move> moves;
    int keep0 = 0;
    for (int i = 0; i < R; keep0 += n_keep[i], ++i) {
        pages[i].reserve(blocks_of(n_keep[i]) + 8);   // (tokens to come)
        const TilePlaces at = places_of(kvs[i], layer);
        if (n_keep[i] > 0) moves.push_back(Move{at, at, &kvs[i]->pages[layer], &pages[i], n_keep[i], kvs[i]->len[layer], keep0});
    }
    for (int i = 0; i < R; ++i)
        while ((int)pages[i].size() < blocks_of(n_keep[i])) pages[i].push_back(kvs[i]->pool->take());
    s = moves.empty() ? RS_OK : launch_moves(ctx, kvs[0]->fp8, moves, keep, st);
    if (s != RS_OK) {   // the old pages stay
        for (int i = R - 1; i >= 0; --i)
            for (auto it = pages[i].rbegin(); it != pages[i].rend(); ++it) kvs[i]->pool->release(*it);
        return s;
    }
    for (int i = R - 1; i >= 0; --i) {
        rs_kv* const kv = kvs[i];
        kv->dropped_from(layer, 0);
        kv->give_back_pages(layer, 0);
        kv->pages[layer].swap(pages[i]);
        kv->len[layer] = n_keep[i];
        kv->stale_tail[layer] = 0;
    }
    return RS_OK;
} catch (const std::exception& e) {
    return not_allocated(e);
}

}  // extern "C"
