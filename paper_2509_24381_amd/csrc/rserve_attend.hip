// Host side of include/rserve_attend.h: argument checks, descriptors and launches of the operators on KV caches.
#include "../../include/rserve_attend.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <exception>
#include <memory>
#include <vector>

#include "attend_few.h"
#include "attend_selected.h"
#include "attend_shared.h"
#include "attention.h"
#include "block_select.h"
#include "cache_calls.h"
#include "few_plan.h"
#include "host_state.h"
#include "kv_fp8.h"
#include "last_error.h"
#include "rope_append.h"

struct rs_rotary {
    rs_ctx* ctx;
    rs_rotary_cfg cfg;
    std::vector<float2> table;    // [max_pos][rotary_dim / 2]
    float2* table_dev = nullptr;
};

namespace {

// Requests of up to 64 stacked rows go to attend_few_kernel, and so do the others of a call if they have little to read: their row groups times
// KV heads times tiles, all together, up to FEW_TILES; beside requests of few rows, where the chunk kernel's launches come on top of those, up
// to FEW_TILES_BESIDE; with 8-bit caches, which the chunk kernel needs expanded, up to FEW_TILES_FP8.  us a pass, chunk kernel /
// attend_few_kernel, (g) 28 query and 4 KV heads, (h) 64 and 8.  One request: (g) 64 tokens on 2000 (896 row groups x heads x tiles)
// 21.1 / 19.4, 96 on 2000 (1408) 23.0 / 22.0, 96 on 4000 (2772) 25.5 / 26.7, 12 on 20000 (2504) 31.6 / 25.2; (h) 12 on 8000 (2000) 22.1 / 21.5,
// 32 on 6000 (3008) 24.9 / 25.8, 100 on 4000 (6552) 33.0 / 40.4.  Beside 23 single tokens on 3000: (g) 12 on 5000 (632) 51.4 / 36.9, 24 on 20000
// (3756) 65.1 / 52.3; (h) 48 on 4000 (3024) 79.1 / 73.4; beside 30 on 300: (g) 96 on 4000 (2772) 37.5 / 28.8, (h) 64 on 2000 (2048) 38.4 / 28.0,
// 96 on 4000 (6048) 46.2 / 54.8; beside 60 on 4000, (g) 128 on 4000 (3528) 109.8 / 100.0, (h) (8064) 184 / 215.  8 bits: (h) 12 on 16000 (4000)
// 46.9 / 24.6, 100 on 4000 (6552) 41.4 / 37.2; beside 30 on 300, 96 on 4000 (6048) 47.9 / 50.5; beside 60 on 4000, 128 on 4000 (8064) 122.4 / 143.5.
// One product does not tell few rows on long caches from many on short ones, and near its bounds the rule takes the slower side: of the lines above
// 12 on 20000, 8 bits 100 on 4000 and beside 30 on 300, 96 on 4000; farther out, (g) 12 on 64000 68.6 / 43.9, 16 on 20000 32.6 / 26.0, on 64000
// 69.6 / 43.3, 32 on 64000 72.5 / 66.8, where (h) has the chunk kernel ahead: 12 on 64000 73.1 / 74.5, 32 on 20000 41.5 / 49.7, on 64000 99.2 / 127.0.
constexpr int FEW_ROWS = FEW_GROUP;
constexpr long FEW_TILES = 2500, FEW_TILES_BESIDE = 5000, FEW_TILES_FP8 = 6500;
// Where a request has more than 32 rows in a group, wavefronts get 32 rows instead of 16 if the call has this many tiles (times KV heads and
// groups).  us a pass, 16 rows / 32: (h) 16 requests of 5 tokens on up to 8000 (7700) 68.8 / 56.2, 8 bits 47.4 / 39.6; (g) 16 of 8 (3900), 8 bits,
// 32.4 / 29.8; (h) one of 100 on 4000 (6552) 47.5 / 40.4, 64 on 2000 (2048) 23.0 / 21.6, 8 on 8000 (1000) 20.8 / 21.7, (g) 96 on 2000 (1408) 22.0 / 23.8.
constexpr long FEW_PAIRS = 2000;
// Caches that one call reads once are loaded with the streaming hint, unless they are so small that the L2s may still have them from a call
// before.  us with / without it, behind a fill of 1 GB: 8 MB 14.6 / 15.6, 35 MB 19.6 / 26.6, 141 MB 38.3 / 69.5; call after call on the
// same caches: 4 MB 15.7 / 14.6, 8 MB 20.2 / 20.4, 141 MB 53.3 / 54.5.
constexpr size_t FEW_ONCE_BYTES = (size_t)8 << 20;
// Workgroups per compute unit that parts are made for.  Four fit, but two stream as fast as four.  us a pass with 1 / 2 / 3 / 4: 64 requests on up to
// 8000 86.0 / 89.4 / 87.1 / 86.1, 16 on up to 32000, 8 bits, 65.1 / 60.2 / 60.9 / 62.3, 24 of 3 and one of 12 81.6 / 53.7 / 57.4 / 57.7.
constexpr int FEW_PLACES = 2;
// Pages that neighbours share are read once where that leaves this much unread: it costs a longer chain of tiles, and parts that have to be joined.  us a pass,
// each alone / shared, (g) 28 and 4 heads, (h) 64 and 8, prompts x beams on tokens (MB that are read again when each reads alone):
// (g) 1 x 8 on 2000 (28) 11.7 / 15.2, 4 x 4 on 2000 (29) 13.9 / 13.0, 1 x 4 on 8000 (49) 15.1 / 15.7, 16 x 4 on 1000 (53) 20.1 / 21.6, 1 x 16 on 2000 (61)
// 13.8 / 16.7, 1 x 2 on 32000 (66) 25.9 / 22.2, 4 x 8 on 2000 (69) 18.4 / 16.2, 16 x 2 on 4000 (74) 28.4 / 24.9, 1 x 8 on 8000 (115) 19.2 / 18.6, 1 x 16 on 8000
// (246) 25.3 / 19.5, 16 x 4 on 8000 (444) 72.7 / 43.5; (h) 4 x 4 on 2000 (59) 17.1 / 15.5, 1 x 8 on 4000 (114) 18.3 / 17.7, 4 x 16 on 8000 (1190) 105 / 46;
// 8 bits: (g) 4 x 4 on 4000 (29) 14.7 / 15.3, 1 x 8 on 8000 (57) 16.5 / 18.8, 16 x 4 on 8000 (222) 43.7 / 32.7, (h) 4 x 16 on 32000 (2390) 227 / 76.
constexpr size_t SHARED_BYTES = (size_t)60 << 20;
constexpr size_t SLOT_ROWS = 65536;   // rows there is room for in the slots of split key ranges
// Tokens times KV heads up to which a workgroup selects for one token, and several share its blocks; beyond, for four.  us a pass, four / one, 4 KV
// heads: 16 tokens on 8000 20.2 / 19.3, on 60000 34.7 / 27.3; 64 on 16000 29.2 / 28.7, on 60000 42.1 / 40.4; 96 on 16000 34.8 / 35.5; 128 on 60000 47.6 / 51.7.
constexpr size_t SELECT_WIDE_UNITS = 256;
constexpr int SELECTED_IN_PLACE_BLOCKS = 1024, SELECTED_IN_PLACE_UNITS = 32;   // (see rs_attend_blocks)
constexpr size_t SELECT_LDS = (size_t)SELECT_MAX_BLOCKS * 4;

rs_status check_matrix(const char* name, const void* p, long ld, int width) {
    if (!p) return fail(RS_EINVAL, "%s is null", name);
    if (!aligned(p, 16)) return fail(RS_EINVAL, "%s must be 16-byte aligned", name);
    if (ld < width || ld % 8) return fail(RS_EINVAL, "ld of %s = %ld must be a multiple of 8 and at least %d", name, ld, width);
    return RS_OK;
}

// ---------------------------------------------------------------- bounds
rs_status check_bounds(const rs_kv* kv, int layer, int i) {
    if (!kv->bound_codes) return fail(RS_ESTATE, "kvs[%d] has no memory for bounds (rs_kv_attach_bounds)", i);
    if (kv->len[layer] / 64 > kv->bound_blocks)
        return fail(RS_ECAPACITY, "kvs[%d]: %d finished blocks, its bounds have room for %d", i, kv->len[layer] / 64, kv->bound_blocks);
    return RS_OK;
}

// Bounds of blocks first[i] .. of every request, in as many launches as their descriptors need kernel arguments.
rs_status launch_bounds(rs_ctx* ctx, int layer, rs_kv* const* kvs, const int* first, int R, hipStream_t st) {
    const int hkv = ctx->cfg.n_kv_heads;
    InlineTable tab;
    int i = 0, b = R > 0 ? first[0] : 0;
    while (i < R) {
        // requests i .. until the words are used up; the last one perhaps in part
        struct Part { int req, b0, b1; };
        Part parts[TABLE_WORDS / 18];
        int n = 0, words = 0;
        while (i < R && n < TABLE_WORDS / 20) {
            const int done = kvs[i]->len[layer] / 64;
            if (b < done) {
                const int room = TABLE_WORDS - words - 24;   // (a request's 16 words and its share of the padded prefix arrays)
                if (room < 1) break;
                const int take = kvs[i]->paged() ? std::min(done - b, room) : done - b;
                parts[n++] = Part{i, b, b + take};
                words += 18 + (kvs[i]->paged() ? take : 0);
                b += take;
            }
            if (b >= done) {
                ++i;
                b = i < R ? first[i] : 0;
            }
        }
        if (n == 0) continue;
        uint32_t items = 0;
        int page_at = table_reqs_at(n) + 16 * n;
        for (int j = 0; j < n; ++j) {
            const rs_kv* kv = kvs[parts[j].req];
            const TilePlaces p = places_of(kv, layer);
            BoundsReq q{};
            q.k = p.k;
            q.head_bytes = p.head_bytes;
            q.block_bytes = p.block_bytes;
            q.pages = CONTIGUOUS;
            if (kv->paged()) {
                q.pages = page_at - parts[j].b0;
                for (int blk = parts[j].b0; blk < parts[j].b1; ++blk) tab.w[page_at++] = (uint32_t)kv->pages[layer][blk];
            }
            const size_t plane = (size_t)layer * hkv * kv->bound_blocks;
            q.codes = (uint64_t)(uintptr_t)(kv->bound_codes + plane * 2 * ctx->cfg.head_dim);
            q.units = (uint64_t)(uintptr_t)(kv->bound_units + plane);
            q.room = kv->bound_blocks;
            q.first = parts[j].b0;
            q.k_scale = kv->k_scale;
            tab.w[j] = items;
            memcpy(&tab.w[table_reqs_at(n) + 16 * j], &q, sizeof(q));
            items += (uint32_t)(parts[j].b1 - parts[j].b0) * hkv;
        }
        with_table(tab, (size_t)page_at, [&](const auto& table) {
            for_kind(ctx, kvs[0]->fp8, [&](auto d, auto fp8) {
                hipLaunchKernelGGL((key_bounds_kernel<decltype(d)::value, decltype(fp8)::value, std::decay_t<decltype(table)>>), dim3((items + 3) / 4), dim3(256), 0,
                                   st, n, hkv, (int)items, table);
            });
        });
        RS_HIP(hipGetLastError());
    }
    return RS_OK;
}

// ---------------------------------------------------------------- workspace
struct AttendLayout {
    size_t few, reqs, items, pagetab, mitems, fp8, tables;   // descriptors: sizes, and their sum
    size_t slots_at, keys_at, chosen_at, split_at, total;   // offsets behind them
};
AttendLayout attend_layout(const rs_layer_cfg& f, int max_rows, int max_requests, int n_blocks) {
    const size_t rows = std::max(max_rows, 1), reqs = std::max(max_requests, 1), g = f.n_q_heads / f.n_kv_heads;
    const size_t pages = reqs * ((size_t)f.max_pos / 64 + 2), entries = reqs + reqs / 2;   // (two requests that share pages are three)
    AttendLayout w;
    w.few = align_up(4 * (std::max(table_reqs_at((int)reqs) + REQ_WORDS * reqs, table_reqs_at((int)entries) + SHARED_WORDS * entries) + pages), 256);
    w.reqs = align_up(sizeof(ReqDesc) * reqs, 256);
    w.items = align_up(sizeof(AttnItem) * (((rows * g + 32 * ATT_WAVES_SMALL - 1) / (32 * ATT_WAVES_SMALL) + reqs) * f.n_kv_heads + ATT_SPLIT_SLOTS), 256);
    w.pagetab = align_up(4 * pages, 256);
    w.mitems = align_up(sizeof(AttnMergeItem) * ATT_SPLIT_SLOTS, 256);
    w.fp8 = align_up(sizeof(Fp8CacheDesc) * reqs, 256);
    w.tables = w.few + w.reqs + w.items + w.pagetab + w.mitems + w.fp8;
    w.slots_at = w.tables;
    w.keys_at = w.slots_at + align_up(SLOT_ROWS * (f.head_dim + 2) * 4, 256);
    w.chosen_at = w.keys_at + align_up(n_blocks > 0 ? std::min<size_t>(rows * f.n_kv_heads, SELECT_WIDE_UNITS) * align_up(f.max_pos / 64 + 1, 4) * 4 : 0, 256);
    w.split_at = w.chosen_at + align_up(n_blocks > 0 ? rows * f.n_kv_heads * n_blocks * 4 : 0, 256);
    w.total = w.split_at;
    if (n_blocks == 0 && rows * g > FEW_ROWS) w.total += align_up((size_t)ATT_SPLIT_SLOTS * 32 * ATT_WAVES * (f.head_dim + 2) * 4, 256);
    return w;
}
size_t expansion_bytes(const rs_ctx* c, long tokens) { return (size_t)2 * align_up((size_t)tokens, 64) * c->kv_dim * 2; }

// ---------------------------------------------------------------- few rows
// The table of `reqs` at `w` (`words` of room, checked by the caller), their page numbers at `pages`.  LIST: items are rows.
struct FewTable {
    uint32_t items = 0, units = 0;
    bool any_split = false;
};
FewTable write_few_table(const rs_ctx* ctx, int layer, rs_kv* const* kvs, const std::vector<FewRequest>& reqs, bool list, bool shared, uint32_t* w,
                         uint32_t* pages) {
    const int n = (int)reqs.size();
    FewTable t;
    int page_at = 0, slot = 0;
    for (int j = 0; j < n; ++j) {
        const FewRequest& r = reqs[j];
        const rs_kv* kv = kvs[r.kv];
        FewReq q{};
        q.k = places_of(kv, layer).k;
        q.head_tiles = kv->paged() ? 1 : kv->cap / 64;
        q.pages = CONTIGUOUS;
        if (kv->paged()) {
            q.pages = page_at;
            q.pages -= r.tile0;
            for (int b = 0; b < r.tiles; ++b) pages[page_at++] = (uint32_t)kv->pages[layer][r.tile0 + b];
        }
        q.row0 = r.row0; q.T = r.T; q.P = r.with == SEVERAL ? r.tiles * 64 : kv->len[layer] - r.T;   // (all rows see all of what is shared)
        q.parts = r.parts;
        q.once = r.once;
        q.slot0 = list ? 0 : slot;
        q.k_scale = kv->k_scale; q.v_scale = kv->v_scale;
        if (shared) {
            const FewShared sh{(uint16_t)q.row0, (uint16_t)q.T, q.pages, q.P, (uint16_t)q.slot0, (uint16_t)r.with, (uint16_t)r.tile0, (uint16_t)r.tiles,
                               (uint8_t)q.parts, (uint8_t)q.once, (uint8_t)r.together, 0};
            memcpy(&w[table_reqs_at(n) + SHARED_WORDS * j], &sh, sizeof(sh));
        } else {
            memcpy(&w[table_reqs_at(n) + REQ_WORDS * j], &q, sizeof(q));
        }
        w[j] = list ? (uint32_t)r.row0 : t.items;
        w[table_units_at(n) + j] = t.units;
        t.items += (uint32_t)(r.units * r.parts);
        if (r.with != SEVERAL) t.units += (uint32_t)(r.units * r.row_blocks);
        if (r.in_slots()) {
            slot += r.units * r.parts * r.row_blocks;
            t.any_split = true;
        }
    }
    return t;
}
size_t few_table_words(const std::vector<FewRequest>& reqs, bool shared) {
    return table_reqs_at((int)reqs.size()) + (shared ? SHARED_WORDS : REQ_WORDS) * reqs.size();
}
size_t few_table_pages(rs_kv* const* kvs, const std::vector<FewRequest>& reqs) {
    size_t n = 0;
    for (const FewRequest& r : reqs) n += kvs[r.kv]->paged() ? r.tiles : 0;
    return n;
}

// Neighbouring requests whose caches start with the same pages become one more request each time, ahead of them, for what they share.
// A request joins its neighbours while that leaves no fewer tiles unread.  False, and all as it was, where there are too few (SHARED_BYTES).
bool share_pages(const rs_ctx* ctx, int layer, rs_kv* const* kvs, std::vector<FewRequest>& reqs) {
    const auto held = [&](const FewRequest& r) -> const std::vector<int>& { return kvs[r.kv]->pages[layer]; };
    const auto unread = [&](const FewRequest& r) { return (kvs[r.kv]->len[layer] - r.T) / 64; };   // blocks that all its rows see whole
    std::vector<FewRequest> several;
    long unread_tiles = 0;
    const rs_kv* const one = kvs[reqs[0].kv];   // (all are told of in a few bits, and are alike: FewShared)
    if (!one->paged() || reqs.size() > 40000 || ctx->cfg.max_tokens_per_call > 65535 || ctx->cfg.max_pos > 4000000) return false;
    for (const FewRequest& r : reqs)
        if (kvs[r.kv]->pool != one->pool || kvs[r.kv]->k_scale != one->k_scale || kvs[r.kv]->v_scale != one->v_scale) return false;
    for (size_t i = 0, j; i < reqs.size(); i = j) {
        const rs_kv* const kv = kvs[reqs[i].kv];
        int same = unread(reqs[i]), T = reqs[i].T;
        if (same > 0 && !kv->pool->shared(held(reqs[i])[0])) same = 0;
        for (j = i + 1; j < reqs.size() && same > 0; ++j) {
            if (reqs[j].row0 != reqs[j - 1].row0 + reqs[j - 1].T) break;
            const int most = std::min(same, unread(reqs[j]));
            const auto& a = held(reqs[i]);
            const int n = pages_in_common(a.data(), held(reqs[j]).data(), most);
            if ((long)n * (long)(j - i) < (long)same * (long)(j - i - 1) || n == 0) break;
            same = n;
            T += reqs[j].T;
        }
        if (j - i < 2 || same == 0) continue;
        unread_tiles += (long)same * (long)(j - i - 1);
        const long rows = (long)T * ctx->group;
        FewRequest all{reqs[i].kv, reqs[i].row0, T, (int)((rows + FEW_GROUP - 1) / FEW_GROUP) * ctx->cfg.n_kv_heads, same,
                       few_row_blocks((int)std::min<long>(rows, FEW_GROUP)), 1};
        all.with = SEVERAL;
        for (size_t k = i; k < j; ++k) {
            reqs[k].with = (int)several.size();
            reqs[k].tile0 = same;
            reqs[k].tiles -= same;
        }
        several.push_back(all);
    }
    if (several.empty()) return false;
    several.insert(several.end(), reqs.begin(), reqs.end());
    const size_t tile_bytes = (size_t)128 * ctx->kv_dim * (kvs[reqs[0].kv]->fp8 ? 1 : 2);   // of all KV heads
    if ((size_t)unread_tiles * tile_bytes < (ctx->shared_bytes >= 0 ? (size_t)ctx->shared_bytes : SHARED_BYTES) || 2 * fewest_slots(several) > SLOT_ROWS / 16) {   // (or no room for their sums: see share_tiles)
        for (FewRequest& r : reqs) {
            r.tiles += r.tile0;
            r.tile0 = 0;
            r.with = NOBODY;
        }
        return false;
    }
    reqs.swap(several);
    return true;
}

template <bool LIST, class Tab>
rs_status launch_few(const rs_ctx* ctx, bool fp8, bool pairs, bool shared, int together, const FewArgs& a, uint32_t items, uint32_t units, bool split, const Tab& tab, hipStream_t st) {
    for_kind(ctx, fp8, [&](auto d, auto f8) {
        constexpr int D = decltype(d)::value;
        constexpr bool FP8 = decltype(f8)::value;
        const auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(items), dim3(64 * FEW_WAVES), 0, st, a, tab); };
        if constexpr (!LIST && !std::is_same_v<Tab, SmallTable>)
            if (shared) {
                if (together == 1) launch(attend_shared_kernel<D, FP8, true, Tab>);
                else if (together == 2) launch(attend_shared_kernel<D, FP8, false, Tab>);
                else launch(attend_few_kernel<D, FP8, false, 1, Tab, true>);
                hipLaunchKernelGGL((shared_merge_kernel<D, Tab>), dim3(units, D / 32), dim3(256), 0, st, a, tab);
                return;
            }
        if constexpr (LIST) launch(attend_few_kernel<D, FP8, true, 1, Tab>);
        else if (pairs) launch(attend_few_kernel<D, FP8, false, 2, Tab>);
        else launch(attend_few_kernel<D, FP8, false, 1, Tab>);
        if (split) hipLaunchKernelGGL((few_merge_kernel<D, LIST, Tab>), dim3(units, D / 32), dim3(256), 0, st, a, tab);
    });
    RS_HIP(hipGetLastError());
    return RS_OK;
}

float log2e_times(float scale) { return (float)(1.4426950408889634 * (double)scale); }

rs_status check_attend(const rs_ctx* ctx, int layer, rs_kv* const* kvs, const int* lens, int R, const void* q, long ld_q, const void* out, long ld_out,
                       float* scale, long* rows) {
    rs_status s = check_call(ctx, layer, kvs, lens, true, R, rows);
    if (s != RS_OK) return s;
    // (a workgroup's rows of out would be rows of q that another has yet to read)
    if (*rows > 1 && q && q == out && ld_q != ld_out) return fail(RS_EINVAL, "out is q, but their ld differ: %ld, %ld", ld_q, ld_out);
    for (int i = 0; i < R; ++i)
        if (lens[i] > kvs[i]->len[layer]) return fail(RS_EINVAL, "lens[%d] = %d exceeds the %d cached tokens", i, lens[i], kvs[i]->len[layer]);
    if (*scale == 0.0f) *scale = (float)(1.0 / std::sqrt((double)ctx->cfg.head_dim));
    if (!(*scale > 0.0f) || !std::isfinite(*scale)) return fail(RS_EINVAL, "scale = %g must be positive and finite, or 0", *scale);
    // what the kernels multiply by: a masked score, minus infinity, times zero would be NaN, and so would a score of zero times infinity
    for (int i = 0; i < R; ++i) {
        const float factor = log2e_times(*scale) * kvs[i]->k_scale;
        if (!(factor > 0.0f) || !std::isfinite(factor))
            return fail(RS_EINVAL, "scale = %g times log2 e times the keys' scale %g of kvs[%d] is not a positive number in 32 bits", *scale, kvs[i]->k_scale, i);
    }
    if (*rows == 0) return RS_OK;
    if ((s = check_matrix("q", q, ld_q, ctx->q_dim)) != RS_OK) return s;
    return check_matrix("out", out, ld_out, ctx->q_dim);
}
rs_status check_workspace(const void* ws, size_t bytes, size_t need) {
    if (!ws) return fail(RS_EINVAL, "workspace is null");
    if (!aligned(ws, 256)) return fail(RS_EINVAL, "workspace must be 256-byte aligned");
    if (bytes < need) return fail(RS_EWORKSPACE, "workspace has %zu bytes, this call needs %zu (rs_attend_workspace_bytes)", bytes, need);
    return RS_OK;
}

// ---------------------------------------------------------------- chunks
template <int D>
rs_status launch_chunks(const rs_ctx* c, const AttnPlan& plan, const ReqDesc* d_reqs, const AttnItem* d_items, const AttnMergeItem* d_mitems, bool paged,
                        const bf16* q, long ld_q, bf16* out, long ld_out, float scale_log2e, float* split_buf, hipStream_t st) {
    int most_parts = 0;
    for (const AttnMergeItem& m : plan.merges) most_parts = std::max(most_parts, m.n_parts);
    const int n_mitems = (int)plan.merges.size();
    const auto attend = [&](auto may_page, auto waves) {
        constexpr int W = decltype(waves)::value;
        hipLaunchKernelGGL((attn_prefill_pipelined_kernel<D, decltype(may_page)::value, W, true>), dim3((unsigned)plan.items.size()), dim3(64 * W), 0, st, d_reqs,
                           d_items, q, (int)ld_q, out, (int)ld_out, c->group, scale_log2e, split_buf);
        const auto merge = [&](auto max_parts, auto early) {
            hipLaunchKernelGGL((attn_merge_kernel<D, W, decltype(max_parts)::value, decltype(early)::value, true>), dim3(n_mitems, ATT_MERGE_Y), dim3(32 * W), 0, st,
                               d_reqs, d_mitems, (const float*)split_buf, out, (int)ld_out, c->group, scale_log2e);
        };
        if (n_mitems == 0) return;
        if (most_parts <= ATT_FEW_PARTS) merge(std::integral_constant<int, ATT_FEW_PARTS>{}, std::true_type{});
        else if (n_mitems * ATT_MERGE_Y * (W / 2) <= ATT_MERGE_EARLY_WAVES * c->n_cu) merge(std::integral_constant<int, ATT_MAX_PARTS>{}, std::true_type{});
        else merge(std::integral_constant<int, ATT_MAX_PARTS>{}, std::false_type{});
    };
    const auto attend_waves = [&](auto may_page) {
        if (plan.waves == ATT_WAVES) attend(may_page, std::integral_constant<int, ATT_WAVES>{});
        else attend(may_page, std::integral_constant<int, ATT_WAVES_SMALL>{});
    };
    if (paged) attend_waves(std::true_type{});
    else attend_waves(std::false_type{});
    RS_HIP(hipGetLastError());
    return RS_OK;
}

}  // namespace

size_t attend_staging_bytes(const rs_layer_cfg& cfg) { return attend_layout(cfg, cfg.max_tokens_per_call, cfg.max_requests, 0).tables; }

extern "C" {

// =============================================================================================== rotary positions
rs_status rs_rotary_create(rs_ctx* ctx, const rs_rotary_cfg* cfg, rs_rotary** out) try {
    if (!ctx || !cfg || !out) return fail(RS_EINVAL, "ctx / cfg / out is null");
    *out = nullptr;
    rs_rotary_cfg c = *cfg;
    if (c.rotary_dim <= 0 || c.rotary_dim % 16 || c.rotary_dim > ctx->cfg.head_dim)
        return fail(RS_EINVAL, "rotary_dim = %d must be a multiple of 16 and at most head_dim = %d", c.rotary_dim, ctx->cfg.head_dim);
    if (c.layout != RS_ROTARY_HALVES && c.layout != RS_ROTARY_INTERLEAVED) return fail(RS_EINVAL, "layout %d", c.layout);
    if (c.scaling < RS_ROTARY_UNSCALED || c.scaling > RS_ROTARY_BANDS) return fail(RS_EINVAL, "scaling %d", c.scaling);
    if (c.max_pos <= 0) return fail(RS_EINVAL, "max_pos must be positive");
    if (!(c.theta > 1.0) || !std::isfinite(c.theta)) return fail(RS_EINVAL, "theta = %g must be above 1 and finite", c.theta);
    if (!(c.magnitude >= 0.0) || !std::isfinite(c.magnitude)) return fail(RS_EINVAL, "magnitude = %g must be positive and finite, or 0", c.magnitude);
    if (c.scaling != RS_ROTARY_UNSCALED && (!(c.factor >= 1.0) || !std::isfinite(c.factor))) return fail(RS_EINVAL, "factor = %g must be at least 1 and finite", c.factor);
    if (c.scaling == RS_ROTARY_RAMP || c.scaling == RS_ROTARY_BANDS) {
        if (c.original_max_pos <= 0) return fail(RS_EINVAL, "original_max_pos must be positive");
        if (c.fast_turns == 0.0) c.fast_turns = c.scaling == RS_ROTARY_RAMP ? 32.0 : 4.0;
        if (c.slow_turns == 0.0) c.slow_turns = 1.0;
        if (!(c.slow_turns > 0.0) || !(c.fast_turns > c.slow_turns) || !std::isfinite(c.fast_turns))
            return fail(RS_EINVAL, "fast_turns = %g must be above slow_turns = %g, both positive", c.fast_turns, c.slow_turns);
    }
    const int half = c.rotary_dim / 2;
    double magnitude = c.magnitude;
    if (magnitude == 0.0) magnitude = c.scaling == RS_ROTARY_RAMP ? 0.1 * std::log(c.factor) + 1.0 : 1.0;
    std::vector<double> freq(half);
    const double pi2 = 6.283185307179586;
    const auto pair_of = [&](double turns) { return c.rotary_dim * std::log(c.original_max_pos / (turns * pi2)) / (2.0 * std::log(c.theta)); };
    for (int j = 0; j < half; ++j) {
        const double f = std::pow(c.theta, -2.0 * j / c.rotary_dim);
        freq[j] = f;
        if (c.scaling == RS_ROTARY_LINEAR) {
            freq[j] = f / c.factor;
        } else if (c.scaling == RS_ROTARY_RAMP) {
            const double low = std::max(std::floor(pair_of(c.fast_turns)), 0.0), high = std::min(std::ceil(pair_of(c.slow_turns)), c.rotary_dim - 1.0);
            const double share = std::min(std::max((j - low) / std::max(high - low, 1e-3), 0.0), 1.0);
            freq[j] = f / c.factor * share + f * (1.0 - share);
        } else if (c.scaling == RS_ROTARY_BANDS) {
            const double turns = c.original_max_pos * f / pi2;
            const double keep = std::min(std::max((turns - c.slow_turns) / (c.fast_turns - c.slow_turns), 0.0), 1.0);
            freq[j] = f / c.factor * (1.0 - keep) + f * keep;
        }
    }
    std::unique_ptr<rs_rotary, void (*)(rs_rotary*)> r(new rs_rotary(), rs_rotary_destroy);
    r->ctx = ctx;
    r->cfg = c;
    r->table.resize((size_t)c.max_pos * half);
    for (int p = 0; p < c.max_pos; ++p)
        for (int j = 0; j < half; ++j) {
            const double angle = p * freq[j];
            r->table[(size_t)p * half + j] = make_float2((float)(std::cos(angle) * magnitude), (float)(std::sin(angle) * magnitude));
        }
    if (ctx->has_device) {
        hipError_t e = hipMalloc((void**)&r->table_dev, r->table.size() * sizeof(float2));
        if (e == hipSuccess) e = hipMemcpy(r->table_dev, r->table.data(), r->table.size() * sizeof(float2), hipMemcpyHostToDevice);
        if (e != hipSuccess) return fail(RS_EHIP, "rotary table: %s", hipGetErrorString(e));
    }
    *out = r.release();
    return RS_OK;
} catch (const std::exception& e) {
    return not_allocated(e);
}

void rs_rotary_destroy(rs_rotary* r) {
    if (!r) return;
    if (r->table_dev) (void)hipFree(r->table_dev);
    delete r;
}

rs_status rs_rotary_at(const rs_rotary* r, int pos, int pair, float* cos_out, float* sin_out) {
    if (!r || !cos_out || !sin_out) return fail(RS_EINVAL, "null argument");
    if (pos < 0 || pos >= r->cfg.max_pos || pair < 0 || pair >= r->cfg.rotary_dim / 2) return fail(RS_EINVAL, "position %d, pair %d out of range", pos, pair);
    const float2 t = r->table[(size_t)pos * (r->cfg.rotary_dim / 2) + pair];
    *cos_out = t.x;
    *sin_out = t.y;
    return RS_OK;
}

// =============================================================================================== append
rs_status rs_kv_append(rs_ctx* ctx, const rs_rotary* rotary, int layer, rs_kv* const* kvs, const int* starts, const int* lens, int R,
                       const int* positions, const void* q, long ld_q, const void* k, long ld_k, const void* v, long ld_v, void* q_out, long ld_q_out,
                       void* stream) try {
    long rows = 0;
    rs_status s = check_call(ctx, layer, kvs, lens, true, R, &rows);
    if (s != RS_OK) return s;
    const rs_layer_cfg& f = ctx->cfg;
    if (rotary && rotary->ctx != ctx) return fail(RS_ESTATE, "the rotary table belongs to another context");
    PageNeed need;
    bool returning = false;   // pages come back to the pool
    for (int i = 0; i < R; ++i) {
        rs_kv* kv = kvs[i];
        const int first = starts ? starts[i] : kv->len[layer];
        if (first < 0 || first > kv->len[layer]) return fail(RS_EINVAL, "starts[%d] = %d outside [0, %d]", i, first, kv->len[layer]);
        const long after = (long)first + lens[i];
        if (!kv->paged() && after > kv->cap) return fail(RS_ECAPACITY, "request %d: %ld tokens exceed cache capacity %d", i, after, kv->cap);
        if (after > f.max_pos) return fail(RS_ECAPACITY, "request %d: %ld tokens exceed max_pos %d", i, after, f.max_pos);
        if (rotary && !positions && lens[i] > 0 && after > rotary->cfg.max_pos)
            return fail(RS_ECAPACITY, "request %d: positions up to %ld exceed the rotary table's %d", i, after - 1, rotary->cfg.max_pos);
        if (kv->paged()) {
            const int missing = kv->pages_missing(layer, after);
            std::vector<int>& held = kv->pages[layer];
            returning |= (int)held.size() > (first + 63) / 64;
            if (held.capacity() < held.size() + missing) held.reserve(std::max(held.size() + missing, 2 * held.capacity()));
            need.add(kv, layer, first, after);
        }
    }
    if ((s = need.check()) != RS_OK) return s;
    if (rotary && positions)
        for (long i = 0; i < rows; ++i)
            if (positions[i] < 0 || positions[i] >= rotary->cfg.max_pos)
                return fail(RS_ECAPACITY, "rotary position %d of row %ld is outside [0, %d)", positions[i], i, rotary->cfg.max_pos);
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    if (rows > 0) {
        if ((q == nullptr) != (q_out == nullptr)) return fail(RS_EINVAL, "q and q_out must both be given, or neither");
        if (q && (s = check_matrix("q", q, ld_q, ctx->q_dim)) != RS_OK) return s;
        if (q && (s = check_matrix("q_out", q_out, ld_q_out, ctx->q_dim)) != RS_OK) return s;
        if (q && q == q_out && ld_q != ld_q_out) return fail(RS_EINVAL, "q_out is q, but their ld differ");
        if ((s = check_matrix("k", k, ld_k, ctx->kv_dim)) != RS_OK) return s;
        if ((s = check_matrix("v", v, ld_v, ctx->kv_dim)) != RS_OK) return s;
        if ((s = check_device(ctx)) != RS_OK) return s;
        if ((s = refuse_capture(st)) != RS_OK) return s;
    }
    std::vector<AppendItem> items;
    items.reserve((size_t)rows / 64 + 2 * (size_t)R);
    std::vector<std::pair<float, float>> scales;   // per item, of 8-bit caches
    if (R > 0 && kvs[0]->fp8) scales.reserve(items.capacity());
    std::vector<PageCopy> copies;   // of shared pages that are continued
    std::vector<int> copied_from;   // per request: the page, or -1
    if (need.copies()) {
        copies.reserve(R);
        copied_from.assign(R, -1);
    }
    bool apart = false;             // a page that is copied from is written in what a copy reads: the copies are a launch before
    // from here on the call is made: tokens dropped, pages taken, launches
    int row = 0, longest = 0;
    const bool fp8 = R > 0 && kvs[0]->fp8;
    // (before anything is given back: a page that is copied into must not be one that another copy still reads.  Where nothing is, all pages are taken here, in
    // the requests' order.)
    for (int i = 0; i < R && need.copies(); ++i) {
        rs_kv* kv = kvs[i];
        const int first = starts ? starts[i] : kv->len[layer];
        if (lens[i] > 0 && kv->continues_shared(layer, first)) {
            copied_from[i] = kv->pages[layer][first / 64];
            copies.push_back(kv->own_block(layer, first));
            uint8_t& read = kv->pool->read_slots[copied_from[i]];
            read = std::max(read, (uint8_t)(first % 64));
        }
        if (!returning && kv->paged()) kv->take_pages(layer, first + lens[i]);
    }
    for (int i = 0; i < R; ++i) {
        rs_kv* kv = kvs[i];
        const int first = starts ? starts[i] : kv->len[layer], after = first + lens[i];
        kv->dropped_from(layer, first);
        kv->len[layer] = after;
        if (kv->paged()) {
            kv->give_back_pages(layer, first);   // (what is written from a block's start on needs nothing of what the block held)
            kv->take_pages(layer, after);
        }
        if (lens[i] == 0) continue;
        const TilePlaces p = places_of(kv, layer);
        for (int pos = first; pos < after;) {
            const int n = std::min(64 - pos % 64, after - pos);
            const uint64_t off = block_offset(kv, layer, p, pos / 64);
            AppendItem it{};
            it.k_lo = (uint32_t)(p.k + off);
            it.k_hi = (uint32_t)((p.k + off) >> 32);
            it.head_tiles = kv->paged() ? 1 : kv->cap / 64;
            it.row0 = row;
            it.pos0 = pos;
            it.slot = (int8_t)(pos % 64);
            it.n = (int8_t)n;
            if (need.copies() && kv->paged()) {
                const int page = kv->pages[layer][pos / 64];
                apart |= pos % 64 < kv->pool->read_slots[page];
                if (pos == first && copied_from[i] >= 0) it.from = copied_from[i] - page;
            }
            it.zero_tail = (pos % 64 == 0 || kv->stale_tail[layer]) && pos % 64 + n < 64;
            items.push_back(it);
            if (fp8) scales.emplace_back(1.0f / kv->k_scale, 1.0f / kv->v_scale);
            longest = std::max(longest, n);
            pos += n;
            row += n;
        }
        kv->stale_tail[layer] = 0;
    }
    if (rows == 0) return RS_OK;
    for (int i = 0; i < R && need.copies(); ++i)
        if (copied_from[i] >= 0) kvs[i]->pool->read_slots[copied_from[i]] = 0;
    // A launch has failed: nothing is left of the call, nor of the blocks that it went on with in pages of their own.
    const auto without = [&](rs_status failed) {
        for (int i = 0; i < R; ++i) {
            rs_kv* kv = kvs[i];
            if (lens[i] == 0) continue;
            const int first = kv->len[layer] - lens[i], left = need.copies() && copied_from[i] >= 0 ? first / 64 * 64 : first;
            kv->dropped_from(layer, left);
            kv->len[layer] = left;
            if (kv->paged()) kv->give_back_pages(layer, left);
        }
        return failed;
    };
    if (apart && (s = launch_page_copies(ctx, fp8, copies, st)) != RS_OK) return without(s);
    AppendArgs a{};
    a.q = (const bf16*)q; a.k = (const bf16*)k; a.v = (const bf16*)v; a.q_out = (bf16*)q_out;
    a.ld_q = ld_q; a.ld_k = ld_k; a.ld_v = ld_v; a.ld_q_out = ld_q_out;
    a.rd = rotary ? rotary->cfg.rotary_dim : 0;
    a.cs = rotary ? rotary->table_dev : nullptr;
    a.hq = f.n_q_heads; a.hkv = f.n_kv_heads;
    // four tasks per thread (2048 rows, 28 heads, us per launch with 4 / 2 / 1: 10.4 / 11.4 / 12.1)
    a.q_slices = q ? std::max(1, (longest * f.n_q_heads * (f.head_dim / 16) + 1023) / 1024) : 0;
    const bool explicit_positions = rotary && positions;
    InlineTable tab;
    for (size_t i0 = 0; i0 < items.size();) {
        size_t i1 = i0, n_scales = 0;
        int words = 0;
        std::pair<float, float> own[TABLE_WORDS / APPEND_WORDS];   // the launch's scales
        while (i1 < items.size()) {   // (an item takes its words, one for each of its rows if positions are explicit, and two if its scales are new)
            size_t which = n_scales;
            if (fp8) which = std::find(own, own + n_scales, scales[i1]) - own;
            const bool another = fp8 && which == n_scales;
            const int w = APPEND_WORDS + (explicit_positions ? items[i1].n : 0) + (another ? 2 : 0);
            if (words + w > TABLE_WORDS) break;
            if (another) own[n_scales++] = scales[i1];
            items[i1].scales = (uint8_t)(fp8 ? which : 0);
            words += w;
            ++i1;
        }
        memcpy(tab.w, &items[i0], sizeof(AppendItem) * (i1 - i0));
        a.positions = NO_POSITIONS;
        a.scales = words - 2 * (int)n_scales;
        memcpy(&tab.w[a.scales], own, sizeof(own[0]) * n_scales);
        if (explicit_positions) {
            const int at = (int)(APPEND_WORDS * (i1 - i0)), r0 = items[i0].row0, r1 = items[i1 - 1].row0 + items[i1 - 1].n;
            memcpy(&tab.w[at], positions + r0, sizeof(int) * (r1 - r0));
            a.positions = at - r0;
        }
        const dim3 grid((unsigned)(i1 - i0), a.hkv + a.q_slices);
        with_table(tab, (size_t)words, [&](const auto& table) {
            typedef std::decay_t<decltype(table)> Tab;
            for_kind(ctx, fp8, [&](auto d, auto f8) {
                constexpr int D = decltype(d)::value;
                constexpr bool FP8 = decltype(f8)::value;
                const auto go = [&](auto interleaved, auto copying) {
                    hipLaunchKernelGGL((rope_append_kernel<D, FP8, decltype(interleaved)::value, decltype(copying)::value, Tab>), grid, dim3(256), 0, st, a, table);
                };
                const bool interleaved = rotary && rotary->cfg.layout == RS_ROTARY_INTERLEAVED, copying = need.copies() && !apart;
                if (interleaved && copying) go(std::true_type{}, std::true_type{});
                else if (interleaved) go(std::true_type{}, std::false_type{});
                else if (copying) go(std::false_type{}, std::true_type{});
                else go(std::false_type{}, std::false_type{});
            });
        });
        const hipError_t launched = hipGetLastError();
        if (launched != hipSuccess) return without(fail(RS_EHIP, "append: %s", hipGetErrorString(launched)));
        i0 = i1;
    }
    return RS_OK;
} catch (const std::exception& e) {
    return not_allocated(e);
}

// =============================================================================================== attention
size_t rs_attend_workspace_bytes(const rs_ctx* c, int max_rows, int max_requests, size_t max_visible_fp8, int n_blocks) {
    if (!c || max_rows <= 0 || max_requests <= 0 || n_blocks < 0) return 0;
    const size_t base = attend_layout(c->cfg, max_rows, max_requests, n_blocks).total;
    return max_visible_fp8 ? base + expansion_bytes(c, (long)max_visible_fp8 + 63L * max_requests) : base;
}

rs_status rs_attend(rs_ctx* ctx, int layer, rs_kv* const* kvs, const int* lens, int R, const void* q, long ld_q, void* out, long ld_out, float scale,
                    void* workspace, size_t workspace_bytes, void* stream) try {
    long rows = 0;
    rs_status s = check_attend(ctx, layer, kvs, lens, R, q, ld_q, out, ld_out, &scale, &rows);
    if (s != RS_OK) return s;
    if (rows == 0) return RS_OK;
    const rs_layer_cfg& f = ctx->cfg;
    const AttendLayout L = attend_layout(f, (int)rows, R, 0);
    const bool fp8 = kvs[0]->fp8;
    const auto stacked_rows = [&](int i) { return (long)lens[i] * ctx->group; };
    const auto row_groups = [&](int i) { return (stacked_rows(i) + FEW_GROUP - 1) / FEW_GROUP; };
    size_t expansion = 0;
    long tiles = 0;   // of the requests with more rows
    bool beside = false;
    for (int i = 0; i < R; ++i) {
        beside |= lens[i] > 0 && stacked_rows(i) <= FEW_ROWS;
        if (stacked_rows(i) > FEW_ROWS) {
            tiles += row_groups(i) * f.n_kv_heads * ((kvs[i]->len[layer] + 63) / 64);
            if (fp8) expansion += expansion_bytes(ctx, kvs[i]->len[layer]);
        }
    }
    const bool chunks = tiles > (ctx->few_tiles >= 0 ? ctx->few_tiles : fp8 ? FEW_TILES_FP8 : beside ? FEW_TILES_BESIDE : FEW_TILES);
    const auto is_few = [&](int i) { return lens[i] > 0 && (!chunks || stacked_rows(i) <= FEW_ROWS); };
    if (!chunks) expansion = 0;
    if ((s = check_workspace(workspace, workspace_bytes, L.total + expansion)) != RS_OK) return s;
    if (chunks && (ld_q > 0x7fffffff || ld_out > 0x7fffffff)) return fail(RS_EINVAL, "ld beyond 2^31");
    if ((s = check_device(ctx)) != RS_OK) return s;
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    if ((s = refuse_capture(st)) != RS_OK) return s;
    char* const ws = reinterpret_cast<char*>(workspace);
    const float scale_log2e = log2e_times(scale);

    // ---- requests of few rows
    std::vector<FewRequest> few;
    int row = 0;
    for (int i = 0; i < R; ++i) {
        if (is_few(i))
            few.push_back(FewRequest{i, row, lens[i], (int)row_groups(i) * f.n_kv_heads, (kvs[i]->len[layer] + 63) / 64,
                                     few_row_blocks((int)std::min<long>(stacked_rows(i), FEW_GROUP)), 1});
        row += lens[i];
    }
    FewArgs a{};
    FewTable ft;
    InlineTable tab;
    bool shared = false;                 // requests share pages
    int together = 0;                    // (FewShared, of those that have it)
    bool pairs = false;                  // wavefronts have two blocks of 16 rows
    enum { NOTHING, PAGES, ALL } few_staged = NOTHING;   // of the table (see TABLE_WORDS)
    size_t few_words = 0, few_pages = 0, few_bytes = 0;   // few_bytes: of the keys and values they read
    if (!few.empty()) {
        shared = few.size() > 1 && share_pages(ctx, layer, kvs, few);
        if (shared) together = share_tiles(few, ctx->group, f.n_kv_heads, ctx->together_tiles >= 0 ? ctx->together_tiles : TOGETHER_TILES, SLOT_ROWS / 16);
        for (const FewRequest& r : few) few_bytes += (size_t)r.tiles * 128 * ctx->kv_dim * (fp8 ? 1 : 2);
        long all_tiles = 0;
        for (const FewRequest& r : few) {
            pairs |= r.row_blocks > 2;
            all_tiles += (long)r.units * r.tiles;
        }
        pairs = pairs && all_tiles >= FEW_PAIRS && !shared;
        for (FewRequest& r : few) {
            r.once = few_bytes >= FEW_ONCE_BYTES && (r.together ? r.units == f.n_kv_heads : r.row_blocks == 1);
            r.weight = r.together ? 1.0 : pairs ? (r.row_blocks == 1 ? 1.0 : r.row_blocks == 2 ? 1.5 : 2.0) : (r.row_blocks == 1 ? 1.0 : r.row_blocks == 2 ? 2.0 : 3.0);
        }
        if (!plan_few(few, FEW_PLACES * ctx->n_cu, SLOT_ROWS / 16)) return fail(RS_EINVAL, "internal: sums beyond the slots");
        a.n_req = (int)few.size();
        a.hkv = f.n_kv_heads; a.g = ctx->group;
        a.q = (const bf16*)q; a.ld_q = ld_q; a.out = (bf16*)out; a.ld_out = ld_out;
        a.scale_log2e = scale_log2e;
        a.slots = reinterpret_cast<float*>(ws + L.slots_at);
        const rs_kv* const one = kvs[few[0].kv];   // (as all of them, where pages are shared)
        a.k = places_of(one, layer).k;
        a.k_scale = one->k_scale; a.v_scale = one->v_scale;
        few_words = few_table_words(few, shared);
        few_pages = few_table_pages(kvs, few);
        few_staged = few_words + few_pages <= TABLE_WORDS ? NOTHING : few_words <= TABLE_WORDS ? PAGES : ALL;
        if (few_staged == NOTHING) ft = write_few_table(ctx, layer, kvs, few, false, shared, tab.w, tab.w + few_words);
    }
    const bool staged = chunks || few_staged != NOTHING;
    int slot = 0;
    RingUse ring(ctx, st);
    if (staged && (s = ring.acquire(&slot)) != RS_OK) return s;
    char* const stage = staged ? ctx->pinned[slot] : nullptr;
    size_t staged_bytes = 0;
    if (few_staged == ALL) {
        ft = write_few_table(ctx, layer, kvs, few, false, shared, reinterpret_cast<uint32_t*>(stage), reinterpret_cast<uint32_t*>(stage) + few_words);
        a.table = reinterpret_cast<const uint32_t*>(ws);
        staged_bytes = align_up((few_words + few_pages) * 4, 16);
    } else if (few_staged == PAGES) {
        ft = write_few_table(ctx, layer, kvs, few, false, shared, tab.w, reinterpret_cast<uint32_t*>(stage));
        a.pages = reinterpret_cast<const uint32_t*>(ctx->pinned_dev[slot]);
        staged_bytes = align_up(few_pages * 4, 16);
    }
    // ---- chunks
    std::vector<ReqDesc> reqs;
    std::vector<int> pagetab;
    std::vector<Fp8CacheDesc> fp8s;
    std::vector<AttnRequest> att;
    AttnPlan plan;
    int n_xblocks = 0;
    size_t at_reqs = 0, at_items = 0, at_mitems = 0, at_fp8 = 0;   // (packed: what is staged crosses the host link)
    if (chunks) {
        const size_t at_pages = staged_bytes;
        const int* const d_pagetab = reinterpret_cast<const int*>(ws + at_pages);
        size_t expand_at = L.total;
        row = 0;
        for (int i = 0; i < R; row += lens[i], ++i) {
            if (stacked_rows(i) <= FEW_ROWS) continue;
            const rs_kv* kv = kvs[i];
            const int len = kv->len[layer];
            ReqDesc d = kv->view(layer, d_pagetab + pagetab.size());
            d.row0 = row; d.T = lens[i]; d.P = len - lens[i];
            d.k_scale = kv->k_scale; d.v_scale = kv->v_scale;   // (bfloat16 caches: one)
            if (fp8) {
                Fp8CacheDesc fc{};
                if (kv->paged()) {
                    fc.kc = reinterpret_cast<uint8_t*>(kv->pool->base);
                    fc.pages = d.pages;
                    d.pages = nullptr;
                } else {
                    fc.kc = kv->kc_of(layer); fc.vc = kv->vc_of(layer); fc.cap = kv->cap;
                }
                fc.xb0 = n_xblocks; fc.hkv = f.n_kv_heads;
                fc.k_scale = fc.v_scale = 1.0f;   // (a code is a bfloat16 number, code times scale is not)
                fp8s.push_back(fc);
                const size_t plane = expansion_bytes(ctx, len) / 2;
                d.kcache = reinterpret_cast<bf16*>(ws + expand_at);
                d.vtcache = reinterpret_cast<bf16*>(ws + expand_at + plane);
                d.cap = (int)align_up((size_t)len, 64);
                expand_at += 2 * plane;
                n_xblocks += d.cap / 64;
            }
            if (kv->paged()) pagetab.insert(pagetab.end(), kv->pages[layer].begin(), kv->pages[layer].begin() + (len + 63) / 64);
            reqs.push_back(d);
            att.push_back(AttnRequest{lens[i], d.P});
        }
        plan = plan_attention(AttnPlanSettings{ctx->n_cu, ctx->attn_split, ctx->attn_plain_order}, att, ctx->group, f.n_kv_heads);
        at_reqs = align_up(at_pages + sizeof(int) * pagetab.size(), 16);
        at_items = align_up(at_reqs + sizeof(ReqDesc) * reqs.size(), 16);
        at_mitems = align_up(at_items + sizeof(AttnItem) * plan.items.size(), 16);
        at_fp8 = align_up(at_mitems + sizeof(AttnMergeItem) * plan.merges.size(), 16);
        staged_bytes = align_up(at_fp8 + sizeof(Fp8CacheDesc) * fp8s.size(), 16);
        if (staged_bytes > L.tables || staged_bytes > ctx->slot_bytes) return fail(RS_EINVAL, "internal: descriptor sizing");
        memcpy(stage + at_reqs, reqs.data(), sizeof(ReqDesc) * reqs.size());
        memcpy(stage + at_items, plan.items.data(), sizeof(AttnItem) * plan.items.size());
        memcpy(stage + at_pages, pagetab.data(), sizeof(int) * pagetab.size());
        memcpy(stage + at_mitems, plan.merges.data(), sizeof(AttnMergeItem) * plan.merges.size());
        memcpy(stage + at_fp8, fp8s.data(), sizeof(Fp8CacheDesc) * fp8s.size());
    }
    if (chunks || few_staged == ALL) {
        const int chunks16 = (int)(staged_bytes / 16);
        hipLaunchKernelGGL(copy_table_kernel, dim3((chunks16 + 255) / 256), dim3(256), 0, st, reinterpret_cast<const uint4*>(ctx->pinned_dev[slot]),
                           reinterpret_cast<uint4*>(ws), chunks16);
        RS_HIP(hipGetLastError());
        if (a.pages) a.pages = reinterpret_cast<const uint32_t*>(ws);   // (copied too)
    }
    if (!few.empty()) {
        const auto launch = [&](const auto& table) { s = launch_few<false>(ctx, fp8, pairs, shared, together, a, ft.items, ft.units, ft.any_split, table, st); };
        if (few_staged == ALL) launch(NoTable{});
        else if (shared) launch(tab);
        else with_table(tab, few_words + (few_staged == NOTHING ? few_pages : 0), launch);
        if (s != RS_OK) return s;
    }
    if (staged && (s = ring.commit()) != RS_OK) return s;
    if (!chunks) return RS_OK;
    const ReqDesc* const d_reqs = reinterpret_cast<const ReqDesc*>(ws + at_reqs);
    const AttnItem* const d_items = reinterpret_cast<const AttnItem*>(ws + at_items);
    const AttnMergeItem* const d_mitems = reinterpret_cast<const AttnMergeItem*>(ws + at_mitems);
    if (fp8) {
        const Fp8CacheDesc* const d_fp8 = reinterpret_cast<const Fp8CacheDesc*>(ws + at_fp8);
        if (f.head_dim == 128) hipLaunchKernelGGL(kv_expand_fp8_kernel<128>, dim3(n_xblocks, f.n_kv_heads), dim3(256), 0, st, d_reqs, d_fp8, (int)reqs.size());
        else hipLaunchKernelGGL(kv_expand_fp8_kernel<64>, dim3(n_xblocks, f.n_kv_heads), dim3(256), 0, st, d_reqs, d_fp8, (int)reqs.size());
        RS_HIP(hipGetLastError());
    }
    float* const split_buf = reinterpret_cast<float*>(ws + L.split_at);
    const bool paged = !pagetab.empty() && !fp8;
    if (f.head_dim == 128) return launch_chunks<128>(ctx, plan, d_reqs, d_items, d_mitems, paged, (const bf16*)q, ld_q, (bf16*)out, ld_out, scale_log2e, split_buf, st);
    return launch_chunks<64>(ctx, plan, d_reqs, d_items, d_mitems, paged, (const bf16*)q, ld_q, (bf16*)out, ld_out, scale_log2e, split_buf, st);
} catch (const std::exception& e) {
    return not_allocated(e);
}

// =============================================================================================== bounds
rs_status rs_kv_attach_bounds(rs_kv* kv, void* codes, void* units, int n_blocks) {
    if (!kv) return fail(RS_EINVAL, "kv is null");
    if ((codes == nullptr) != (units == nullptr)) return fail(RS_EINVAL, "codes and units must both be given, or neither");
    if (codes && n_blocks <= 0) return fail(RS_EINVAL, "n_blocks = %d must be positive", n_blocks);
    if (codes && (!aligned(codes, 16) || !aligned(units, 4))) return fail(RS_EINVAL, "codes must be 16-byte aligned, units 4-byte");
    kv->bound_codes = reinterpret_cast<int8_t*>(codes);
    kv->bound_units = reinterpret_cast<float*>(units);
    kv->bound_blocks = codes ? n_blocks : 0;
    std::fill(kv->bounded.begin(), kv->bounded.end(), 0);
    return RS_OK;
}

int rs_kv_bounded(const rs_kv* kv, int layer) {
    if (!kv || layer < 0 || layer >= kv->n_layers) return -1;
    return kv->bounded[layer];
}

rs_status rs_kv_bounds_update(rs_ctx* ctx, int layer, rs_kv* const* kvs, const int* firsts, int R, void* stream) try {
    rs_status s = check_call(ctx, layer, kvs, nullptr, false, R, nullptr);
    if (s != RS_OK) return s;
    std::vector<int> first(R);
    bool any = false;
    for (int i = 0; i < R; ++i) {
        if ((s = check_bounds(kvs[i], layer, i)) != RS_OK) return s;
        if (firsts && (firsts[i] < 0 || firsts[i] > kvs[i]->len[layer])) return fail(RS_EINVAL, "firsts[%d] = %d outside [0, %d]", i, firsts[i], kvs[i]->len[layer]);
        first[i] = firsts ? firsts[i] / 64 : kvs[i]->bounded[layer];
        any |= first[i] < kvs[i]->len[layer] / 64;
    }
    if (!any) return RS_OK;
    if ((s = check_device(ctx)) != RS_OK) return s;
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    if ((s = refuse_capture(st)) != RS_OK) return s;
    if ((s = launch_bounds(ctx, layer, kvs, first.data(), R, st)) != RS_OK) return s;
    for (int i = 0; i < R; ++i)   // (with a gap before the first block the blocks after it do not count)
        if (first[i] <= kvs[i]->bounded[layer]) kvs[i]->bounded[layer] = kvs[i]->len[layer] / 64;
    return RS_OK;
} catch (const std::exception& e) {
    return not_allocated(e);
}

// =============================================================================================== attention over selected blocks
rs_status rs_attend_blocks(rs_ctx* ctx, int layer, rs_kv* const* kvs, const int* lens, int R, const void* q, long ld_q, void* out, long ld_out,
                           int n_blocks, int n_first, int n_last, float scale, int* chosen, void* workspace, size_t workspace_bytes, void* stream) try {
    long rows = 0;
    rs_status s = check_attend(ctx, layer, kvs, lens, R, q, ld_q, out, ld_out, &scale, &rows);
    if (s != RS_OK) return s;
    if (n_blocks < 1 || n_blocks > 1024 || n_first < 0 || n_last < 1)
        return fail(RS_EINVAL, "n_blocks = %d must be 1 .. 1024, n_first = %d at least 0, n_last = %d at least 1", n_blocks, n_first, n_last);
    if (ctx->group > FEW_GROUP) return fail(RS_EINVAL, "%d query heads per KV head: more than %d", ctx->group, FEW_GROUP);
    for (int i = 0; i < R; ++i)
        if ((s = check_bounds(kvs[i], layer, i)) != RS_OK) return s;
    if (rows == 0) return RS_OK;
    const rs_layer_cfg& f = ctx->cfg;
    int longest = 0;
    for (int i = 0; i < R; ++i) longest = std::max(longest, lens[i] > 0 ? kvs[i]->len[layer] / 64 + 1 : 0);
    if (longest > SELECT_MAX_BLOCKS) return fail(RS_ECAPACITY, "a cache of %d blocks is longer than the selection can hold (%d)", longest, SELECT_MAX_BLOCKS);
    if (chosen && !aligned(chosen, 4)) return fail(RS_EINVAL, "chosen must be 4-byte aligned");
    const AttendLayout L = attend_layout(f, (int)rows, R, n_blocks);
    if ((s = check_workspace(workspace, workspace_bytes, L.total)) != RS_OK) return s;
    if ((s = check_device(ctx)) != RS_OK) return s;
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    if ((s = refuse_capture(st)) != RS_OK) return s;
    char* const ws = reinterpret_cast<char*>(workspace);
    const bool fp8 = kvs[0]->fp8;
    if (!ctx->select_ready) {   // first use on this context: opt in to the LDS size once
        const auto opt_in = [](auto d, auto table) -> rs_status {
            constexpr int D = decltype(d)::value;
            typedef decltype(table) Tab;
            for (const void* k : {(const void*)block_select_kernel<D, false, SELECT_ALL, Tab>, (const void*)block_select_kernel<D, true, SELECT_ALL, Tab>,
                                  (const void*)block_select_kernel<D, true, SELECT_FROM_SCORES, Tab>})
                RS_HIP(hipFuncSetAttribute(k, hipFuncAttributeMaxDynamicSharedMemorySize, (int)SELECT_LDS));
            return RS_OK;
        };
        const std::integral_constant<int, 64> narrow{};
        const std::integral_constant<int, 128> broad{};
        if ((s = opt_in(narrow, InlineTable{})) != RS_OK || (s = opt_in(narrow, SmallTable{})) != RS_OK || (s = opt_in(broad, InlineTable{})) != RS_OK ||
            (s = opt_in(broad, SmallTable{})) != RS_OK)
            return s;
        ctx->select_ready = true;
    }
    // bounds that are missing
    std::vector<int> first(R);
    bool missing = false;
    for (int i = 0; i < R; ++i) {
        first[i] = kvs[i]->bounded[layer];
        if (lens[i] == 0) first[i] = kvs[i]->len[layer] / 64;
        missing |= first[i] < kvs[i]->len[layer] / 64;
    }
    if (missing) {
        if ((s = launch_bounds(ctx, layer, kvs, first.data(), R, st)) != RS_OK) return s;
        for (int i = 0; i < R; ++i)
            if (lens[i] > 0) kvs[i]->bounded[layer] = kvs[i]->len[layer] / 64;
    }
    std::vector<FewRequest> reqs;
    int row = 0;
    for (int i = 0; i < R; ++i) {
        if (lens[i] > 0) reqs.push_back(FewRequest{i, row, lens[i], lens[i] * f.n_kv_heads, (kvs[i]->len[layer] + 63) / 64, few_row_blocks(ctx->group), 1});
        row += lens[i];
    }
    const int rbn = few_row_blocks(ctx->group), units = (int)rows * f.n_kv_heads;
    // Parts of a list: a block per wavefront where there are places for that, else a power of two, so that wavefronts' shares stay even; one part
    // where a list is short or three quarters of the compute units are busy without.  us a pass with 1 / 2 / 4 / 8 parts, 4 KV heads: lists of 16,
    // one token 17.5 / 18.4 / 17.5 / 17.2, 32 tokens 18.9 / 20.5 / 20.5 / 22.5; of 32, one 21.7 / 20.3 / 18.4 / 17.4, 16 24.2 / 21.1 / 19.5 / 20.1,
    // 32 25.0 / 22.5 / 22.4 / 24.9, 48 25.2 / 26.0 / 26.5 / 30.4, 64 26.9 / 28.9 / 31.0 / 35.8; of 64, 8 36.5 / 25.9 / 22.2 / 20.0, 48 35.4 / 33.9 / 33.2 / 36.4.
    // Lists of 48, one token: 12 parts 17.5, 8 parts 18.4; 24 tokens (96 units): 6 parts 26.3, 4 parts 24.4.
    int parts = 1;
    const int held = std::min(n_blocks, longest), places = FEW_PLACES * ctx->n_cu, apart = std::min((held + FEW_WAVES - 1) / FEW_WAVES, FEW_MAX_PARTS);
    if (held > 4 * FEW_WAVES && 4 * units <= 3 * ctx->n_cu) {
        if (apart * units <= places) parts = apart;
        else while (2 * parts * units <= places && 2 * parts <= apart) parts *= 2;
    }
    if ((size_t)units * parts * rbn > SLOT_ROWS / 16) parts = 1;
    const bool wide = (size_t)units <= SELECT_WIDE_UNITS;
    int halvings = 0;
    for (int x = 1; x < ctx->group; x *= 2) ++halvings;
    const size_t few_words = few_table_words(reqs, false), few_pages = few_table_pages(kvs, reqs), selected_words = few_words + BOUNDS_WORDS * reqs.size();
    const int split = wide ? std::min((longest + SELECT_ROUND - 1) / SELECT_ROUND, std::max(1, 2 * ctx->n_cu / units)) : 1;
    // One kernel selects and attends where the descriptors fit its arguments and the keys of scores its LDS, as long as all its workgroups run at
    // once.  Page numbers are beside the descriptors or in place; a token or two whose scores are a launch of their own and whose pages
    // are many have theirs copied behind the scores instead, for kernels of their own.  us a pass, kernels of their own / one, 4 KV heads: lists of 8
    // on 16000, one token 15.4 / 12.2, 64 tokens 17.5 / 12.7, 128 19.4 / 16.6, 256 27.1 / 27.3, 500 38.6 / 45.1; of 32, one 17.1 / 15.2, 64 27.2 / 22.0,
    // 256 54.0 / 53.2, 500 91.9 / 95.8; on 60000, of 8, one 19.0 / 17.7, 16 21.3 / 18.4, of 32, one 21.5 / 20.5; on 130000, of 32, one 22.3 / 23.2, 4
    // 23.1 / 23.7, 8 25.5 / 24.4, 64 46.8 / 46.3; contiguous, 8 bits, one 22.1 / 21.2, 8 24.9 / 22.3.
    const bool fits = selected_words + few_pages <= TABLE_WORDS;
    const bool selected = units <= FEW_PLACES * ctx->n_cu && longest <= SELECTED_BLOCKS && selected_words <= TABLE_WORDS &&
                          (split == 1 || fits || longest <= SELECTED_IN_PLACE_BLOCKS || units >= SELECTED_IN_PLACE_UNITS);
    const bool in_arguments = selected && fits;
    int slot = 0;
    RingUse ring(ctx, st);
    if (!in_arguments && (s = ring.acquire(&slot)) != RS_OK) return s;
    uint32_t* const stage = in_arguments ? nullptr : reinterpret_cast<uint32_t*>(ctx->pinned[slot]);

    SelectArgs sa{};
    sa.hkv = f.n_kv_heads; sa.g = ctx->group;
    sa.halvings = halvings;
    sa.q = (const bf16*)q; sa.ld_q = ld_q;
    sa.blocks = (int)align_up(longest, 4);
    sa.n_blocks = n_blocks; sa.n_first = n_first; sa.n_last = n_last;
    sa.tokens = wide ? 1 : (int)std::min<size_t>(4, SELECT_LDS / ((size_t)sa.blocks * 4));   // (blocks, at most SELECT_MAX_BLOCKS, which is a multiple of 4 too)
    sa.split = split;
    sa.shared_keys = reinterpret_cast<uint32_t*>(ws + L.keys_at);
    FewArgs a{};
    a.n_req = (int)reqs.size();
    a.hkv = f.n_kv_heads; a.g = ctx->group;
    a.q = (const bf16*)q; a.ld_q = ld_q; a.out = (bf16*)out; a.ld_out = ld_out;
    a.scale_log2e = log2e_times(scale);
    a.slots = reinterpret_cast<float*>(ws + L.slots_at);
    a.n_blocks = n_blocks;
    a.list_parts = parts;

    const auto bounds_at = [&](const FewRequest& r) {
        const rs_kv* kv = kvs[r.kv];
        const size_t plane = (size_t)layer * f.n_kv_heads * kv->bound_blocks;
        return BoundsAt{(uint64_t)(uintptr_t)(kv->bound_codes + plane * 2 * f.head_dim), (uint64_t)(uintptr_t)(kv->bound_units + plane), kv->bound_blocks, 0};
    };
    // the selection's descriptors of n requests from the i0-th on; their groups of tokens
    const auto write_select_table = [&](size_t i0, int n, InlineTable& tab) {
        uint32_t groups = 0;
        for (int j = 0; j < n; ++j) {
            const FewRequest& r = reqs[i0 + j];
            const BoundsAt at = bounds_at(r);
            SelectReq sr{};
            sr.codes = at.codes; sr.units = at.units; sr.room = at.room;
            sr.row0 = r.row0; sr.T = r.T; sr.P = kvs[r.kv]->len[layer] - r.T;
            tab.w[j] = groups;
            memcpy(&tab.w[table_reqs_at(n) + 16 * j], &sr, sizeof(sr));
            groups += (uint32_t)((r.T + sa.tokens - 1) / sa.tokens);
        }
        return groups;
    };
    constexpr int threads = 256;
    if (selected) {
        const int n = a.n_req;
        InlineTable tab;
        write_few_table(ctx, layer, kvs, reqs, true, false, tab.w, in_arguments ? tab.w + selected_words : stage);
        for (int j = 0; j < n; ++j) {
            const BoundsAt at = bounds_at(reqs[j]);
            memcpy(&tab.w[few_words + BOUNDS_WORDS * j], &at, sizeof(at));
        }
        if (!in_arguments) a.pages = reinterpret_cast<const uint32_t*>(ctx->pinned_dev[slot]);
        if (sa.split > 1) {   // scores first, several workgroups per token
            InlineTable select_tab;
            const uint32_t groups = write_select_table(0, n, select_tab) * sa.split;
            sa.n_req = n;
            sa.groups = (int)groups;
            with_table(select_tab, (size_t)table_reqs_at(n) + 16 * n, [&](const auto& table) {
                typedef std::decay_t<decltype(table)> Tab;
                const auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(groups, f.n_kv_heads), dim3(threads), 0, st, sa, table); };
                if (f.head_dim == 128) launch(block_select_kernel<128, true, SELECT_SCORES, Tab>);
                else launch(block_select_kernel<64, true, SELECT_SCORES, Tab>);
            });
            RS_HIP(hipGetLastError());
        }
        SelectedArgs se{halvings, n_first, n_last, sa.blocks, sa.shared_keys, chosen};
        with_table(tab, selected_words + (in_arguments ? few_pages : 0), [&](const auto& table) {
            typedef std::decay_t<decltype(table)> Tab;
            for_kind(ctx, fp8, [&](auto d, auto f8) {
                constexpr int D = decltype(d)::value;
                constexpr bool FP8 = decltype(f8)::value;
                const auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(units * parts), dim3(64 * FEW_WAVES), 0, st, a, se, table); };
                if (sa.split > 1) launch(attend_selected_kernel<D, FP8, true, Tab>);
                else launch(attend_selected_kernel<D, FP8, false, Tab>);
                if (parts > 1) hipLaunchKernelGGL((few_merge_kernel<D, true, Tab>), dim3(units * rbn, D / 32), dim3(256), 0, st, a, table);
            });
        });
        RS_HIP(hipGetLastError());
        return in_arguments ? RS_OK : ring.commit();
    }
    // the attention kernel's table, copied by the first selection launch
    write_few_table(ctx, layer, kvs, reqs, true, false, stage, stage + few_words);
    sa.chosen = chosen ? chosen : reinterpret_cast<int*>(ws + L.chosen_at);
    sa.copy_from = reinterpret_cast<const uint4*>(ctx->pinned_dev[slot]);
    sa.copy_to = reinterpret_cast<uint4*>(ws);
    sa.copy_chunks = (int)(align_up((few_words + few_pages) * 4, 16) / 16);
    constexpr int WINDOW = TABLE_WORDS / 20;   // requests whose descriptors the kernel arguments hold
    for (size_t i0 = 0; i0 < reqs.size(); i0 += WINDOW) {
        const int n = (int)std::min<size_t>(WINDOW, reqs.size() - i0);
        InlineTable tab;
        const uint32_t groups = write_select_table(i0, n, tab);
        sa.n_req = n;
        const unsigned copying = i0 == 0 ? (unsigned)((sa.copy_chunks + threads - 1) / threads) : 0u;
        const size_t lds = (size_t)sa.tokens * sa.blocks * 4;
        const auto select = [&](auto d) {
            constexpr int D = decltype(d)::value;
            with_table(tab, (size_t)table_reqs_at(n) + 16 * n, [&](const auto& table) {
                typedef std::decay_t<decltype(table)> Tab;
                if (sa.split > 1) {
                    sa.groups = (int)groups * sa.split;
                    hipLaunchKernelGGL((block_select_kernel<D, true, SELECT_SCORES, Tab>), dim3(groups * sa.split + copying, f.n_kv_heads), dim3(threads), 0, st, sa, table);
                    hipLaunchKernelGGL((block_select_kernel<D, true, SELECT_FROM_SCORES, Tab>), dim3(groups, f.n_kv_heads), dim3(1024), lds, st, sa, table);
                    return;
                }
                sa.groups = (int)groups;
                if (wide) hipLaunchKernelGGL((block_select_kernel<D, true, SELECT_ALL, Tab>), dim3(groups + copying, f.n_kv_heads), dim3(threads), lds, st, sa, table);
                else hipLaunchKernelGGL((block_select_kernel<D, false, SELECT_ALL, Tab>), dim3(groups + copying, f.n_kv_heads), dim3(threads), lds, st, sa, table);
            });
        };
        if (f.head_dim == 128) select(std::integral_constant<int, 128>{});
        else select(std::integral_constant<int, 64>{});
        RS_HIP(hipGetLastError());
        if (i0 == 0 && (s = ring.commit()) != RS_OK) return s;
    }
    a.table = reinterpret_cast<const uint32_t*>(ws);
    a.chosen = sa.chosen;
    return launch_few<true>(ctx, fp8, false, false, 0, a, (uint32_t)(units * parts), (uint32_t)(units * rbn), parts > 1, NoTable{}, st);
} catch (const std::exception& e) {
    return not_allocated(e);
}

}  // extern "C"
