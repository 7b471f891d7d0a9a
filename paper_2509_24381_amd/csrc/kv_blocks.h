// Blocks of a cache as the append, export and import kernels are told of them.
#pragma once
#include "attention.h"
#include "common.h"

// ---------------------------------------------------------------- append
struct KVBlockItem {
    int req;
    int block;  // absolute 64-token block index in the request's cache
};

// ---------------------------------------------------------------- tiles of a cache in export / import (kv_transfer.h)
// The cache is described like a request (ReqDesc: contiguous planes, or the pool base for a paged cache).  The page
// numbers of a paged cache travel in the kernel arguments, a window of KV_PAGE_WINDOW blocks per launch starting at
// block `block0`; tokens [t0, t0 + n) are handled, t0 a multiple of 64 inside the window.
constexpr int KV_PAGE_WINDOW = 256;
struct KVPageWindow {
    int page[KV_PAGE_WINDOW];
};

template <int D>
RS_DEVICE bf16* kv_window_tile(const ReqDesc& rq, const KVPageWindow& win, int block0, bool v, int c, int block) {
    constexpr size_t TILE = (size_t)64 * D;  // elements
    if (rq.pages == nullptr)   // (any non-null value marks a paged cache here; the numbers come from the window)
        return (v ? rq.vtcache : rq.kcache) + ((size_t)c * (size_t)(rq.cap >> 6) + (size_t)block) * TILE;
    return rq.kcache + ((size_t)win.page[block - block0] * 2 * rq.hkv + (size_t)(v ? rq.hkv : 0) + (size_t)c) * TILE;
}
