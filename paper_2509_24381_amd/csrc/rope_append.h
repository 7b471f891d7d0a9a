// Rotary positions on the way into the cache: the new tokens' queries are turned and stored, their keys turned, rounded (and
// quantised) and stored with their values into the caches, in one launch.
//
// Bound by HBM where there are many rows, by latency where there are few.  One workgroup takes the tokens of one request that fall
// in one 64-token block, either of one KV head (keys row by row; values turned through LDS, 8 tokens per store, when there are many) or
// of a share of the query heads.  A task is 16 features of a head whose pairs are complete in it: two 16-byte loads, 64 bytes of cosines
// and sines, two 16-byte stores.
//
//   (a, b) -> (a cos - b sin, b cos + a sin), in fp32 from fp32 cosines and sines of 64-bit angles, rounded to bfloat16 once; 8-bit caches
//   take the rounded key's code, so that they hold what a bfloat16 cache's content would be encoded as.
//
// Measured (28 query heads, 4 KV heads, d = 128), us of the kernel: one token 3 to 4.2, 64 single tokens 5.1, 2048 rows of 8 requests into 8-bit
// pages, 36 MB, 10.6 (3.4 TB/s).  With four tasks of a thread's queries loaded together as well: 11 to 12 (registers).
#pragma once
#include "attend_few.h"
#include "common.h"
#include "kv_fp8.h"

struct AppendItem {        // 48 bytes
    uint64_t k, v;         // K and V^T tile of KV head 0 of the block
    uint64_t head_bytes;   // from a KV head's tile to the next head's
    int32_t row0;          // first row of the call
    int32_t pos0;          // its slot in the request's cache
    int16_t slot, n;       // first place in the block, tokens
    int32_t zero_tail;     // V behind the last token of the block is to be zeroed
    float k_inv, v_inv;    // fl32(1 / scale) of 8-bit caches
};
static_assert(sizeof(AppendItem) == 48, "twelve words");

constexpr int NO_POSITIONS = INT32_MIN;
struct AppendArgs {          // (table: the items, then, if there are explicit ones, a rotary position per row)
    int positions;           // word of row 0's position (rows before this launch's included); NO_POSITIONS: the cache slots
    const bf16 *q, *k, *v;
    bf16* q_out;
    long ld_q, ld_k, ld_v, ld_q_out;
    const float2* cs;        // [position][rd / 2]
    int rd;                  // features that are turned (0: none)
    int hq, hkv;
    int q_slices;            // workgroups that share a block's queries
};

// Features `a` .. a + 7 and `b` .. b + 7 of a head, task j of D / 16: where they are, and their values turned.
template <bool INTERLEAVED>
RS_DEVICE void pair_task(int j, int rd, int& a, int& b) {
    if (16 * j >= rd || INTERLEAVED) {
        a = 16 * j;
        b = a + 8;
    } else {
        a = 8 * j;
        b = a + rd / 2;
    }
}
template <bool INTERLEAVED>
RS_DEVICE void turn_pairs(int j, int rd, const float2* cs, bf16x8& x, bf16x8& y) {
    if (16 * j >= rd) return;
    f32x4 t[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) t[i] = *reinterpret_cast<const f32x4*>(cs + 8 * j + 2 * i);   // pairs 8 j .. 8 j + 7
    bf16x8 ox, oy;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float co = t[e >> 1][2 * (e & 1)], si = t[e >> 1][2 * (e & 1) + 1];
        if constexpr (INTERLEAVED) {   // pair e: features 2 e, 2 e + 1 of the sixteen
            const float a = bf16_to_f32(e < 4 ? x[(2 * e) & 7] : y[(2 * e) & 7]), b = bf16_to_f32(e < 4 ? x[(2 * e + 1) & 7] : y[(2 * e + 1) & 7]);
            const bf16 p = f32_to_bf16(a * co - b * si), q = f32_to_bf16(b * co + a * si);
            if (e < 4) {
                ox[(2 * e) & 7] = p;
                ox[(2 * e + 1) & 7] = q;
            } else {
                oy[(2 * e) & 7] = p;
                oy[(2 * e + 1) & 7] = q;
            }
        } else {
            const float a = bf16_to_f32(x[e]), b = bf16_to_f32(y[e]);
            ox[e] = f32_to_bf16(a * co - b * si);
            oy[e] = f32_to_bf16(b * co + a * si);
        }
    }
    x = ox;
    y = oy;
}

constexpr int APPEND_FEW = 8;   // up to this many tokens of a block the values are stored one by one
template <int D, bool FP8, bool INTERLEAVED, class Tab>
__global__ __launch_bounds__(256) void rope_append_kernel(AppendArgs a, Tab tab) {
    constexpr int TASKS = D / 16, EL = FP8 ? 1 : 2;
    const uint32_t* const table = tab.w;
    const AppendItem it = reinterpret_cast<const AppendItem*>(table)[blockIdx.x];
    const int slot = it.slot, n = it.n;
    const auto angles = [&](int t) RS_INLINE {
        const int pos = a.positions == NO_POSITIONS ? it.pos0 + t : (int)table[a.positions + it.row0 + t];
        return a.cs + (size_t)pos * (a.rd / 2);
    };
    if ((int)blockIdx.y >= a.hkv) {   // queries
        const int per_token = a.hq * TASKS, total = n * per_token;
        for (int i = ((int)blockIdx.y - a.hkv) * 256 + (int)threadIdx.x; i < total; i += a.q_slices * 256) {
            const int t = i / per_token, head = i % per_token / TASKS, j = i % TASKS;
            int fa, fb;
            pair_task<INTERLEAVED>(j, a.rd, fa, fb);
            const bf16* src = a.q + (size_t)(it.row0 + t) * a.ld_q + head * D;
            bf16* dst = a.q_out + (size_t)(it.row0 + t) * a.ld_q_out + head * D;
            bf16x8 x = as_bf16x8(ld_global_16(src + fa)), y = as_bf16x8(ld_global_16(src + fb));
            turn_pairs<INTERLEAVED>(j, a.rd, angles(t), x, y);
            st_global_16(dst + fa, as_uint4(x));
            st_global_16(dst + fb, as_uint4(y));
        }
        return;
    }
    const int h = blockIdx.y;
    char* const kt = reinterpret_cast<char*>(it.k + (uint64_t)h * it.head_bytes);
    char* const vt = reinterpret_cast<char*>(it.v + (uint64_t)h * it.head_bytes);
    const bf16* const k0 = a.k + (size_t)it.row0 * a.ld_k + h * D;
    const bf16* const v0 = a.v + (size_t)it.row0 * a.ld_v + h * D;
    const int end = slot + n;
    const bool turned = n > APPEND_FEW || it.zero_tail;   // values go through LDS
    __shared__ __attribute__((aligned(16))) bf16 tile[64][D + 8];
    // all of a thread's loads first: its 16-byte chunks of values, its tasks of the keys
    constexpr int VN = 64 * (D / 8) / 256, KN = (64 * TASKS + 255) / 256;
    uint4 v[4], x[2], y[2];
    static_assert(VN <= 4 && KN <= 2, "head dim 128 at most");
    if (turned) {
#pragma unroll
        for (int j = 0; j < VN; ++j) {
            const int i = j * 256 + (int)threadIdx.x;
            if (i < n * (D / 8)) v[j] = ld_global_16(v0 + (size_t)(i / (D / 8)) * a.ld_v + i % (D / 8) * 8);
        }
    }
#pragma unroll
    for (int j = 0; j < KN; ++j) {
        const int i = j * 256 + (int)threadIdx.x;
        if (i < n * TASKS) {
            int fa, fb;
            pair_task<INTERLEAVED>(i % TASKS, a.rd, fa, fb);
            x[j] = ld_global_16(k0 + (size_t)(i / TASKS) * a.ld_k + fa);
            y[j] = ld_global_16(k0 + (size_t)(i / TASKS) * a.ld_k + fb);
        }
    }
    if (turned) {
#pragma unroll
        for (int j = 0; j < VN; ++j) {
            const int i = j * 256 + (int)threadIdx.x;
            if (i < n * (D / 8)) *reinterpret_cast<uint4*>(&tile[slot + i / (D / 8)][i % (D / 8) * 8]) = v[j];
        }
    }
#pragma unroll
    for (int j = 0; j < KN; ++j) {
        const int i = j * 256 + (int)threadIdx.x;
        if (i < n * TASKS) {
            const int t = i / TASKS;
            int fa, fb;
            pair_task<INTERLEAVED>(i % TASKS, a.rd, fa, fb);
            bf16x8 p = as_bf16x8(x[j]), q = as_bf16x8(y[j]);
            turn_pairs<INTERLEAVED>(i % TASKS, a.rd, angles(t), p, q);
            char* const dst = kt + (size_t)(slot + t) * D * EL;
            if constexpr (FP8) {
                *reinterpret_cast<uint2*>(dst + fa) = e4m3_from_bf16x8(p, it.k_inv);
                *reinterpret_cast<uint2*>(dst + fb) = e4m3_from_bf16x8(q, it.k_inv);
            } else {
                st_global_16(dst + fa * 2, as_uint4(p));
                st_global_16(dst + fb * 2, as_uint4(q));
            }
        }
    }
    const auto store_one = [&](int d, int place, bf16 value) RS_INLINE {
        if constexpr (FP8) reinterpret_cast<uint8_t*>(vt)[d * 64 + place] = (uint8_t)(e4m3_pair(bf16_to_f32(value) * it.v_inv, 0.0f) & 0xffu);
        else reinterpret_cast<bf16*>(vt)[d * 64 + place] = value;
    };
    if (!turned) {   // values, one by one
        for (int i = threadIdx.x; i < n * D; i += 256) store_one(i % D, slot + i / D, v0[(size_t)(i / D) * a.ld_v + i % D]);
        return;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < D * 8; i += 256) {   // feature i / 8, places 8 (i % 8) ..
        const int d = i >> 3, p0 = (i & 7) * 8;
        if (p0 + 7 < slot || (p0 >= end && !it.zero_tail)) continue;   // older tokens; nothing
        bf16x8 o;
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = p0 + e >= slot && p0 + e < end ? tile[p0 + e][d] : f32_to_bf16(0.0f);
        if (p0 >= slot && (p0 + 8 <= end || it.zero_tail)) {
            if constexpr (FP8) *reinterpret_cast<uint2*>(vt + d * 64 + p0) = e4m3_from_bf16x8(o, it.v_inv);
            else st_global_16(vt + d * 128 + p0 * 2, as_uint4(o));
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (p0 + e >= slot && (p0 + e < end || it.zero_tail)) store_one(d, p0 + e, o[e]);
        }
    }
}
