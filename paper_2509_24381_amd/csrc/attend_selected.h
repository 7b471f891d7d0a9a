// Selection and attention in one kernel, for few tokens: a launch less, and the list stays in LDS.
#pragma once
#include "attend_few.h"
#include "block_select.h"

// One workgroup per (row, part of its list, KV head).  It scores the blocks (or takes the scores that a launch before left, where blocks are
// many: SCORED) and picks the list, every part for itself, with the four wavefronts that then attend to the part.  Keys of scores lie
// where the tiles go afterwards.  Bound by latency: from queries to codes, scores, digits, list, keys, values; us a pass, one token on 16000, lists
// of 8 blocks, 12.2 (two kernels 15.4), lists of 32 and the merge 15.2 (17.1); the rule that chooses has more.
constexpr int SELECTED_BLOCKS = 4096;      // of a cache, at most
constexpr int SELECTED_LIST = 1024;        // of a list, at most
struct BoundsAt {                          // of a request: six words of the table, behind the FewReqs
    uint64_t codes, units;
    int32_t room, pad_;
};
constexpr int BOUNDS_WORDS = 6;
static_assert(sizeof(BoundsAt) == 4 * BOUNDS_WORDS, "BOUNDS_WORDS");
struct SelectedArgs {
    int halvings, n_first, n_last;
    int blocks;                            // SCORED: keys per (row, KV head)
    const uint32_t* shared_keys;
    int* chosen;                           // the lists are wanted: [row][KV head][n_blocks]
};

template <int D, bool FP8, bool SCORED, class Tab>
__global__ __launch_bounds__(64 * FEW_WAVES, 2) void attend_selected_kernel(FewArgs a, SelectedArgs sa, Tab tab) {
    __shared__ __attribute__((aligned(16))) char lds[FEW_LDS<D, FP8>];
    __shared__ FewStats m_sh, l_sh;
    __shared__ __attribute__((aligned(16))) int8_t u[1][2 * D];
    __shared__ SelectTeam<FEW_WAVES> team;
    __shared__ uint32_t chunk_more[SELECTED_BLOCKS / 64 + 1], chunk_equal[SELECTED_BLOCKS / 64 + 1];
    __shared__ int list[SELECTED_LIST];
    static_assert(FEW_LDS<D, FP8> >= SELECTED_BLOCKS * 4, "room for the keys");
    uint32_t* const keys = reinterpret_cast<uint32_t*>(lds);
    const uint32_t* const table = tab.w;
    FewRows<true> rows;
    rows.g = rows.rows = a.g;
    int id = blockIdx.x;
    rows.kvh = id % a.hkv;
    id /= a.hkv;
    const int parts = a.list_parts, part = id % parts, row = id / parts, unit = row * a.hkv + rows.kvh;
    const int req = request_of(table, a.n_req, (uint32_t)row);
    const FewReq rq = reinterpret_cast<const FewReq*>(table + table_reqs_at(a.n_req))[req];
    const uint32_t* const bounds = table + table_reqs_at(a.n_req) + REQ_WORDS * a.n_req;
    const uint32_t* const pages = a.pages ? a.pages : bounds + BOUNDS_WORDS * a.n_req;
    rows.tok0 = row - rq.row0;
    const int own = (rq.P + rows.tok0) / 64;
    const int s0 = min(sa.n_first, own), s1 = max(s0, own + 1 - sa.n_last);   // blocks that can need a score
    if (own + 1 > a.n_blocks && s1 > s0) {
        if constexpr (SCORED) {
            const uint32_t* const from = sa.shared_keys + (size_t)unit * sa.blocks;
            for (int i = threadIdx.x * 4; i < s1 - s0; i += 64 * FEW_WAVES * 4) *reinterpret_cast<uint4*>(&keys[i]) = *reinterpret_cast<const uint4*>(&from[i]);
        } else {
            const BoundsAt at = reinterpret_cast<const BoundsAt*>(bounds)[req];
            score_blocks<D, 1>(a.q + (size_t)row * a.ld_q + (size_t)rows.kvh * a.g * D, a.ld_q, a.g, sa.halvings, 1,
                               reinterpret_cast<const int8_t*>(at.codes) + (size_t)rows.kvh * at.room * 2 * D,
                               reinterpret_cast<const float*>(at.units) + (size_t)rows.kvh * at.room, s0, s1, 0, SELECT_ROUND, u, keys, 0);
        }
        __syncthreads();
    }
    pick_blocks<FEW_WAVES>(keys - s0, own, a.n_blocks, sa.n_first, sa.n_last, team, chunk_more, chunk_equal, list);
    __syncthreads();
    if (sa.chosen && part == 0)
        for (int i = threadIdx.x; i < a.n_blocks; i += 64 * FEW_WAVES) sa.chosen[(size_t)unit * a.n_blocks + i] = list[i];
    attend_rows<D, FP8, true, 1>(a, rq, pages, rows, part, parts, unit, min(a.n_blocks, own + 1), list, lds, m_sh, l_sh);
}
