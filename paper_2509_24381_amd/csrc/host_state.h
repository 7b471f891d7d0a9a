// What the library's host files share: the objects behind the handles of the C ABI, and the ring of pinned staging buffers
// that calls put their descriptors into.
#pragma once
#include "../../include/rserve_prefill.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <vector>

#include "attention.h"
#include "common.h"
#include "last_error.h"

#define RS_HIP(expr)                                                                                    \
    do {                                                                                                \
        hipError_t e_ = (expr);                                                                         \
        if (e_ != hipSuccess) return rs_internal_fail(RS_EHIP, "%s: %s", #expr, hipGetErrorString(e_)); \
    } while (0)

inline size_t align_up(size_t v, size_t a) { return (v + a - 1) / a * a; }
inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

constexpr int RING_SLOTS = 32;
constexpr int RING_CHECKPOINT = 8;

struct rs_ctx {
    rs_layer_cfg cfg;
    int qkv_dim, q_dim, kv_dim, group;
    float2* rope_dev = nullptr;  // [max_pos][d/2] (cos, sin)
    // pinned staging ring for per-call descriptors
    char* pinned[RING_SLOTS] = {};
    char* pinned_dev[RING_SLOTS] = {};  // the same buffers as the device addresses them
    // A slot may be overwritten once the first kernel of the call that used it has run.  Recording an event behind that
    // kernel in every call would tell, but an event record holds the stream up for about 6 us; so events are recorded only
    // at checkpoints: after every RING_CHECKPOINT-th use, and - on the stream that is being left - whenever the caller's
    // stream changes.  Uses are numbered; the first checkpoint at or after use u is on u's stream and behind its kernel.
    hipEvent_t slot_done[RING_SLOTS] = {};
    long slot_recorded_at[RING_SLOTS];   // the use number slot_done[slot] was last recorded at (-1: never)
    size_t slot_bytes = 0;
    long use_count = 0;                   // uses so far; use u occupies slot u % RING_SLOTS
    hipStream_t last_stream = nullptr;
    int splitk_override = 0;  // RS_SPLITK environment variable (0 = heuristic)
    int mrope_b0 = 0, mrope_b1 = 0;  // rotary pair j turns with axis 0 below b0, axis 1 below b1, axis 2 above (set in rs_ctx_create)
    bool attn_plain_order = false;  // RS_ATTN_ORDER=plain: attention blocks that share a compute unit stay heaviest-first (no pairing)
    int attn_split = 0;       // RS_ATTN_SPLIT environment variable: parts a block's key range is cut into (0: decided per call)
    long few_tiles = -1;      // RS_ATTEND_FEW environment variable: what rs_attend's rule for requests of more rows compares with (-1: its constants)
    int gemm_few = 1;         // RS_NARROW environment variable: 0 keeps every call on the strip GEMMs (no tiles, no few-rows kernel)
    int n_cu = 256;           // compute units of the device: the number of strips a GEMM launch is cut into
    bool has_device = false;  // false: created on a host without a GPU; argument checks work, launches return RS_EHIP
    int device = -1;          // the GPU that was current in rs_ctx_create
    void* static_ws = nullptr;  // that GPU's copy of the static workspace (rs_prefill_chunk_static)
    bool select_ready = false;   // block_select_kernel has its LDS size (rs_attend_blocks)
    int lm_rows = 0;          // rows per launch of the first-token head (0: its LDS size not yet set, see rs_lm_head)
    // measurement hook: HIP events around every launch of one step of the layer
    int prof_step = -1;
    int prof_count = 0;
    int prof_every = 1;       // measure every n-th launch of the step
    int prof_seen = 0;        // launches of the step seen since rs_profile_enable
    bool prof_take = false;   // the launch in progress is being measured
    std::vector<hipEvent_t> prof_events;  // (start, stop) pairs
};

// A pool of fixed-size pages in caller-owned device memory.  A page holds 64 tokens of ONE layer: the K tiles [64][d] of
// all KV heads followed by their V^T tiles [d][64].  The free list lives on the host.
struct rs_kv_pool {
    rs_ctx* ctx;
    char* base;
    size_t page_bytes;
    int n_pages;
    bool fp8 = false;              // pages of E4M3 bytes (half the size) for 8-bit caches
    int n_caches = 0;              // paged caches alive on this pool
    std::vector<int> free_pages;   // stack: the back is handed out next
};

struct rs_kv {
    rs_ctx* ctx;
    int n_layers;
    int cap;  // contiguous: capacity in tokens, multiple of 64; paged: unused (see capacity())
    char* base;
    size_t k_bytes;      // one layer's K
    size_t layer_bytes;  // K + V^T
    std::vector<int> len;
    rs_kv_pool* pool = nullptr;             // paged caches only
    std::vector<std::vector<int>> pages;    // paged: pages[layer][block]
    bool fp8 = false;                       // one E4M3 byte per element; k_bytes counts bytes
    float k_scale = 1.0f, v_scale = 1.0f;   // 8-bit caches: value = decode(code) * scale
    // V behind the newest token, inside its block, may hold something other than zero (tokens that were dropped)
    std::vector<char> stale_tail;
    // bounds on the keys of finished blocks (rs_kv_attach_bounds); caller-owned device memory, null: none
    int8_t* bound_codes = nullptr;          // [layer][KV head][block][high, low][d]
    float* bound_units = nullptr;           // [layer][KV head][block]
    int bound_blocks = 0;                   // blocks there is room for
    std::vector<int> bounded;               // per layer: blocks 0 .. bounded - 1 have theirs
    void start_layers(int n) {
        len.assign(n, 0);
        stale_tail.assign(n, 0);
        bounded.assign(n, 0);
    }
    // tokens n .. of `layer` are gone: their bounds with them
    void dropped_from(int layer, int n) {
        if (n < len[layer] && n % 64 != 0) stale_tail[layer] = 1;
        bounded[layer] = std::min(bounded[layer], n / 64);
    }
    bool paged() const { return pool != nullptr; }
    uint8_t* kc_of(int layer) const { return reinterpret_cast<uint8_t*>(base + (size_t)layer * layer_bytes); }
    uint8_t* vc_of(int layer) const { return reinterpret_cast<uint8_t*>(base + (size_t)layer * layer_bytes + k_bytes); }
    bf16* k_of(int layer) const { return reinterpret_cast<bf16*>(base + (size_t)layer * layer_bytes); }
    bf16* vt_of(int layer) const { return reinterpret_cast<bf16*>(base + (size_t)layer * layer_bytes + k_bytes); }
    // new pages layer `layer` needs before it can hold n_tokens
    int pages_missing(int layer, long n_tokens) const {
        return paged() ? std::max<long>(0, (n_tokens + 63) / 64 - (long)pages[layer].size()) : 0;
    }
    void take_pages(int layer, long n_tokens) {  // the caller has checked that the pool has enough
        for (int k = pages_missing(layer, n_tokens); k > 0; --k) {
            pages[layer].push_back(pool->free_pages.back());
            pool->free_pages.pop_back();
        }
    }
    void give_back_pages(int layer, long n_tokens) {  // keeps the pages that hold the first n_tokens
        const size_t keep = (size_t)((n_tokens + 63) / 64);
        while (pages[layer].size() > keep) {
            pool->free_pages.push_back(pages[layer].back());
            pages[layer].pop_back();
        }
    }
    // the cache of `layer` as the kernels see it (row0 / T / P left to the caller; `pages` is a device pointer or a marker)
    ReqDesc view(int layer, const int* dev_pages) const {
        ReqDesc d{};
        d.cap = cap;
        d.hkv = ctx->cfg.n_kv_heads;
        if (paged()) {
            d.kcache = reinterpret_cast<bf16*>(pool->base);
            d.pages = dev_pages;
        } else {
            d.kcache = k_of(layer);
            d.vtcache = vt_of(layer);
        }
        return d;
    }
};

// The staging ring.  ring_acquire gives the next use's slot, waiting until what was staged there before has been read;
// ring_commit ends the use, behind the last kernel that reads the slot.
__attribute__((visibility("hidden"))) rs_status ring_acquire(rs_ctx* ctx, hipStream_t st, int* slot);
__attribute__((visibility("hidden"))) rs_status ring_commit(rs_ctx* ctx, hipStream_t st);

// RS_ESTATE if `st` is capturing a HIP graph (a replay would find stale descriptors).
__attribute__((visibility("hidden"))) rs_status refuse_capture(hipStream_t st);

// Bytes of a staging slot that the operators on caches need (rserve_attend.hip).
__attribute__((visibility("hidden"))) size_t attend_staging_bytes(const rs_layer_cfg& cfg);
