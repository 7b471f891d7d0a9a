// Attention of one query row without the matrix pipe, for rows whose result is not finite.
#pragma once
#include "common.h"

typedef const __attribute__((address_space(1))) char* global_bytes;

template <bool FP8>
RS_DEVICE float tile_element(global_bytes tile, int i) {
    if constexpr (FP8) return __builtin_amdgcn_cvt_f32_fp8((int)*reinterpret_cast<const __attribute__((address_space(1))) uint8_t*>(tile + i), 0);
    else return bf16_to_f32(*reinterpret_cast<const __attribute__((address_space(1))) bf16*>(tile + 2 * (size_t)i));
}

// One query row over tiles [i0, i1), by one wavefront, without the matrix pipe: what the attention kernels fall back on where a row's result is
// not finite.  A masked value enters their products with weight zero, and zero times an infinity or NaN is NaN; here it does not enter.
// Returns the reference (the largest score, as the product leaves it) and the row sum of weights 2^(sc (score - m)), and in o the unnormalised
// output of features lane + 64 i.
template <int D, bool FP8, class TileAt>
RS_DEVICE void exact_row(const bf16* q, float sc, int qpos, int i0, int i1, TileAt&& tile_at, float& m, float& l, float (&o)[D / 64]) {
    const int lane = threadIdx.x & 63;
    m = -INFINITY;
    l = 0.0f;
#pragma unroll
    for (int j = 0; j < D / 64; ++j) o[j] = 0.0f;
    for (int i = i0; i < i1; ++i) {
        global_bytes kt, vt;
        int block;
        tile_at(i, kt, vt, block);
        const int live = min(64, qpos + 1 - block * 64);   // keys that the row sees
        if (live <= 0) continue;
        float s = 0.0f;
        for (int d = 0; d < D; ++d) s = __builtin_fmaf(bf16_to_f32(q[d]), tile_element<FP8>(kt, lane * D + d), s);
        s = lane < live ? s : -INFINITY;
        float mx = s;
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) mx = fmaxf(mx, __shfl_xor(mx, off, WAVE));
        const float m_new = fmaxf(m, mx), ref = m_new == -INFINITY ? 0.0f : m_new;
        const float p = lane < live ? __builtin_amdgcn_exp2f((s - ref) * sc) : 0.0f, alpha = __builtin_amdgcn_exp2f((m - ref) * sc);
        l = l * alpha + wave_sum(p);
#pragma unroll
        for (int j = 0; j < D / 64; ++j) o[j] *= alpha;
        for (int k = 0; k < live; ++k) {
            const float w = __shfl(p, k, WAVE);
#pragma unroll
            for (int j = 0; j < D / 64; ++j) o[j] = __builtin_fmaf(w, tile_element<FP8>(vt, (lane + 64 * j) * 64 + k), o[j]);
        }
        m = m_new;
    }
}
