// Descriptors of a call on caches, as its kernels get them: in the kernel arguments where they fit, else copied to the workspace ahead of the kernel.  Page numbers that do not fit
// beside them are read where the host left them: a wavefront does it once per 64 tiles.  (All of it read in place: three such reads, one after
// the other, at the start of every workgroup, as long as the copy.)
#pragma once
#include "common.h"

constexpr int TABLE_WORDS = 928;
// (Aligned for what lies in them: requests and copies with 64-bit addresses, behind arrays that are padded to 16 bytes.)
struct alignas(16) InlineTable { uint32_t w[TABLE_WORDS]; };
struct alignas(16) SmallTable { uint32_t w[112]; };   // of a few requests: a launch of 4 KB of arguments takes the host 1.3 us more
struct NoTable {};

constexpr int32_t CONTIGUOUS = INT32_MIN;

// Table: every request's first item, and its first unit (what few_merge_kernel joins), each padded to 16 bytes; requests.
__host__ __device__ inline int table_units_at(int n_req) { return (n_req + 3) & ~3; }
__host__ __device__ inline int table_reqs_at(int n_req) { return 2 * table_units_at(n_req); }

template <class Tab>
RS_DEVICE const uint32_t* table_of(const Tab& tab, const uint32_t* device_table) {
    if constexpr (std::is_same_v<Tab, NoTable>) return device_table;
    else return tab.w;
}
// The last request whose first item is at most `id`.
RS_DEVICE int request_of(const uint32_t* table, int n_req, uint32_t id) {
    if (n_req == 1) return 0;
    const int lane = threadIdx.x & 63;
    int at = -1;
    for (int i0 = 0; i0 < n_req; i0 += 64) {
        const bool before = i0 + lane < n_req && table[min(i0 + lane, n_req - 1)] <= id;
        at += __popcll(__builtin_amdgcn_ballot_w64(before));
    }
    return __builtin_amdgcn_readfirstlane(at);
}
