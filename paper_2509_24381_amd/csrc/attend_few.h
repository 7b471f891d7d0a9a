// Attention of few query rows per KV head: the tokens a request generates one at a time, a few drafted ones, or - with a
// list of blocks per token - any tokens that attend to selected blocks only.
//
//   out[row] = sum_k w_k value_k / sum_k w_k,   w_k = 2^(scale log2e q . key_k - m),  m a reference that tracks the maximum
//
// Bound by the bytes of the keys and values: a tile of 64 keys is 32 KB (d = 128, bfloat16), and the rows that share it - the g
// query heads of a KV head, times the tokens - give it 16 MFMAs of 16 clocks per 16 rows and product.  So nothing is shared
// between wavefronts and nothing goes through LDS: each wavefront owns whole tiles, loads a tile straight into the MFMA operand
// layout (16 rows x 64 bytes per instruction; the tile is contiguous, so every line is used whole), and the next tile's keys are
// under way while the softmax runs, its values while the next scores are formed: up to 32 KB in flight per wavefront.
//
// As in the chunk kernel (attention.h) the transposed products keep a query in one lane (lane & 15):
//   S^T[key, query] = K Q^T,   O^T[d, query] = V^T P^T   with v_mfma_f32_16x16x32_bf16
// and the assignment of MFMA rows to keys is chosen so that the four scores a lane holds of each of its sub-tiles are, put together, the
// consecutive keys that it has to feed to the second product.  8-bit tiles are loaded 16 codes at a time (the keys' order
// changes with it) and become bfloat16, exactly, in registers; their scales go into the softmax's scale and the output.
//
// Work item = (request, KV head, block of 16 NB stacked rows, part of the key range).  Four wavefronts take the item's tiles in
// turn and meet in LDS once; parts leave unnormalised sums, references and row sums in slots that few_merge_kernel joins.
#pragma once
#include "attention.h"
#include "common.h"
#include "exact_row.h"
#include "kv_fp8.h"

// Descriptors of a call: in the kernel arguments where they fit, else copied to the workspace ahead of the kernel (read in place they
// would cross the host link once per workgroup).
constexpr int TABLE_WORDS = 880;
struct InlineTable { uint32_t w[TABLE_WORDS]; };
struct NoTable {};

constexpr int32_t CONTIGUOUS = INT32_MIN;

// One request, 64 bytes.  The tile of block b (V: v) of KV head h:  k + h * head_bytes + index * block_bytes, index = b in a contiguous
// cache, the block's page in a paged one.
struct FewReq {
    uint64_t k, v;
    uint64_t head_bytes;
    uint32_t block_bytes;
    int32_t pages;         // number of block b: word pages + b of the table; CONTIGUOUS: b itself
    int32_t row0, T, P;    // first row, rows, position of the first row
    int32_t parts;         // parts of the key range
    int32_t slot0;         // of its first part
    float k_scale, v_scale;
    int32_t pad_;
};
static_assert(sizeof(FewReq) == 64, "sixteen words");

// Table: every request's first item, and its first unit (what few_merge_kernel joins), each padded to 16 bytes; requests; page numbers.
__host__ __device__ inline int table_units_at(int n_req) { return (n_req + 3) & ~3; }
__host__ __device__ inline int table_reqs_at(int n_req) { return 2 * table_units_at(n_req); }

template <bool INLINE, class Tab>
RS_DEVICE const uint32_t* table_of(const Tab& tab, const uint32_t* device_table) {
    if constexpr (INLINE) return tab.w;
    else return device_table;
}
// The last request whose first item is at most `id`.
RS_DEVICE int request_of(const uint32_t* table, int n_req, uint32_t id) {
    const int lane = threadIdx.x & 63;
    int at = -1;
    for (int i0 = 0; i0 < n_req; i0 += 64) {
        const bool before = i0 + lane < n_req && table[min(i0 + lane, n_req - 1)] <= id;
        at += __popcll(__builtin_amdgcn_ballot_w64(before));
    }
    return __builtin_amdgcn_readfirstlane(at);
}

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
RS_DEVICE uint4 ld_tile_16(global_bytes p) { return __builtin_bit_cast(uint4, *reinterpret_cast<const __attribute__((address_space(1))) u32x4*>(p)); }

// Eight E4M3 codes to bfloat16, exactly.
RS_DEVICE bf16x8 bf16x8_of_codes(uint32_t lo, uint32_t hi) {
    bf16x8 o;
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
    o[0] = a[0]; o[1] = a[1]; o[2] = b[0]; o[3] = b[1]; o[4] = c[0]; o[5] = c[1]; o[6] = d[0]; o[7] = d[1];
    return o;
}
struct FewArgs {
    const uint32_t* table;   // device table (not INLINE)
    int n_req, hkv, g;
    const bf16* q;
    long ld_q;
    bf16* out;
    long ld_out;
    float scale_log2e;
    float* slots;
    const int* chosen;       // LIST: [row][KV head][n_blocks], -1 behind the last
    int n_blocks, list_parts;
};

constexpr int FEW_WAVES = 4;
constexpr int FEW_MAX_PARTS = 64;
constexpr float FEW_HEADROOM = 8.0f;   // the reference moves when a score exceeds it by this many powers of two

template <int D, int NB>
struct FewSlot {   // [16 NB rows][D] sums, then references, then row sums
    static constexpr size_t FLOATS = (size_t)16 * NB * (D + 2);
};

template <int D, bool FP8, int NB, bool LIST, bool INLINE>
__global__ __launch_bounds__(64 * FEW_WAVES, NB == 1 ? 2 : 1) void attend_few_kernel(FewArgs a, std::conditional_t<INLINE, InlineTable, NoTable> tab) {
    constexpr int KS = D / 32, DT = D / 16, RB = FP8 ? D : 2 * D;
    constexpr int KL = FP8 ? 4 * (D / 64) : 4 * KS, VL = FP8 ? DT : 2 * DT;   // 16-byte loads per lane of a tile's keys, values
    __shared__ __attribute__((aligned(16))) float red[FEW_WAVES][16][D + 4];
    __shared__ float m_sh[FEW_WAVES][16 * NB], l_sh[FEW_WAVES][16 * NB];
    const uint32_t* const table = table_of<INLINE>(tab, a.table);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, c = lane >> 4;

    // ---- which rows, which tiles
    int req, kvh, part, parts, row_first, rows_here, tok0, unit;
    if constexpr (LIST) {
        int id = blockIdx.x;
        kvh = id % a.hkv;
        id /= a.hkv;
        parts = a.list_parts;
        part = id % parts;
        const int row = id / parts;
        req = request_of(table, a.n_req, (uint32_t)row);
        unit = row * a.hkv + kvh;
        row_first = row;
        rows_here = a.g;
    } else {
        req = request_of(table, a.n_req, blockIdx.x);
        unit = row_first = rows_here = part = parts = kvh = 0;
    }
    const FewReq rq = reinterpret_cast<const FewReq*>(table + table_reqs_at(a.n_req))[req];
    int kb0, kb1;
    const int* list = nullptr;
    if constexpr (LIST) {
        tok0 = row_first - rq.row0;
        list = a.chosen + (size_t)unit * a.n_blocks;
        const int n = min(a.n_blocks, (rq.P + tok0) / 64 + 1);   // (the list ends there)
        kb0 = (int)((long)n * part / parts);
        kb1 = (int)((long)n * (part + 1) / parts);
    } else {
        int id = (int)(blockIdx.x - table[req]);
        parts = rq.parts;
        kvh = id % a.hkv;
        id /= a.hkv;
        part = id % parts;
        const int rb = id / parts;
        unit = rb * a.hkv + kvh;
        row_first = rb * 16 * NB;                                 // of the request's T g stacked rows
        rows_here = min(16 * NB, rq.T * a.g - row_first);
        tok0 = row_first / a.g;
        const int n = (rq.P + (row_first + rows_here - 1) / a.g) / 64 + 1;
        kb0 = (int)((long)n * part / parts);
        kb1 = (int)((long)n * (part + 1) / parts);
    }
    const auto token_of = [&](int col) RS_INLINE { return LIST ? tok0 : (row_first + col) / a.g; };
    const auto head_of = [&](int col) RS_INLINE { return kvh * a.g + (LIST ? col : (row_first + col) % a.g); };
    const auto tile_at = [&](int i, global_bytes& kt, global_bytes& vt, int& block) RS_INLINE {
        block = i;
        if constexpr (LIST) {
            block = list[i];
            if (block < 0) return false;
        }
        const uint64_t index = rq.pages == CONTIGUOUS ? (uint32_t)block : table[rq.pages + block];
        const uint64_t off = (uint64_t)kvh * rq.head_bytes + index * rq.block_bytes;
        kt = (global_bytes)(rq.k + off);
        vt = (global_bytes)(rq.v + off);
        return true;
    };

    // ---- queries
    bf16x8 qf[NB][KS];
    int qpos[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        const int col = min(nb * 16 + r, rows_here - 1);   // (rows past the end repeat the last one and are not stored)
        const int tok = token_of(col);
        qpos[nb] = rq.P + tok;
        const bf16* p = a.q + (size_t)(rq.row0 + tok) * a.ld_q + head_of(col) * D;
#pragma unroll
        for (int kk = 0; kk < KS; ++kk)
            qf[nb][kk] = *reinterpret_cast<const bf16x8*>(p + (FP8 ? (kk >> 1) * 64 + c * 16 + (kk & 1) * 8 : kk * 32 + c * 8));
    }
    const int seen_by_all = rq.P + tok0;   // every row of the item sees the keys up to here
    const float sc = FP8 ? a.scale_log2e * rq.k_scale : a.scale_log2e;

    f32x4 acc[NB][DT];
    float m[NB], l[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        m[nb] = -INFINITY;
        l[nb] = 0.0f;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) acc[nb][dt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    const uint32_t k_off = (uint32_t)(((r >> 2) * (FP8 ? 16 : 8) + (r & 3)) * RB + c * 16);
    const uint32_t v_off = (uint32_t)(r * (FP8 ? 64 : 128) + c * 16);
    uint4 kf[KL], vf[VL];
    const auto load_k = [&](global_bytes kt) RS_INLINE {
#pragma unroll
        for (int i = 0; i < KL; ++i) {
            constexpr int PER = KL / 4;   // loads of a sub-tile of 16 keys
            const int t = i / PER, kk = i % PER;
            const int key = FP8 ? t * 4 : (t >> 1) * 32 + (t & 1) * 4;
            kf[i] = ld_tile_16(kt + k_off + (key * RB + kk * 64));
        }
    };
    const auto load_v = [&](global_bytes vt) RS_INLINE {
#pragma unroll
        for (int i = 0; i < VL; ++i) vf[i] = ld_tile_16(vt + v_off + (FP8 ? i * 16 * 64 : (i >> 1) * 16 * 128 + (i & 1) * 64));
    };

    // ---- tiles kb0 + wave, + 4, ...
    global_bytes kt = nullptr, vt = nullptr;
    int block = 0, kb = kb0 + wave;
    bool have = kb < kb1 && tile_at(kb, kt, vt, block);
    if (have) {
        load_k(kt);
        load_v(vt);
    }
    while (have) {
        f32x4 s[NB][4];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int kk = 0; kk < KS; ++kk) {
                bf16x8 kfrag;
                if constexpr (FP8) {
                    const uint4 w = kf[t * (KS / 2) + (kk >> 1)];
                    kfrag = (kk & 1) ? bf16x8_of_codes(w.z, w.w) : bf16x8_of_codes(w.x, w.y);
                } else {
                    kfrag = as_bf16x8(kf[t * KS + kk]);
                }
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
                    s[nb][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kfrag, qf[nb][kk], kk == 0 ? f32x4{0.0f, 0.0f, 0.0f, 0.0f} : s[nb][t], 0, 0, 0);
            }
        const int key0 = block * 64;
        global_bytes vt_next = nullptr;
        kb += FEW_WAVES;
        have = kb < kb1 && tile_at(kb, kt, vt_next, block);
        if (have) load_k(kt);
        bf16x8 pf[NB][2];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            if (key0 + 63 > seen_by_all) {
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int key = key0 + (FP8 ? c * 16 + t * 4 : (t >> 1) * 32 + c * 8 + (t & 1) * 4) + e;
                        s[nb][t][e] = key <= qpos[nb] ? s[nb][t][e] : -INFINITY;
                    }
            }
            float mx = s[nb][0][0];
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) mx = fmaxf(mx, s[nb][t][e]);
            mx = fmaxf(mx, __shfl_xor(mx, 16, WAVE));
            mx = fmaxf(mx, __shfl_xor(mx, 32, WAVE)) * sc;
            const bool move = mx > m[nb] + FEW_HEADROOM;   // (at first m is minus infinity)
            if (__builtin_amdgcn_ballot_w64(move)) {
                const float m_new = move ? mx : m[nb];
                const float alpha = m[nb] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m[nb] - m_new);
                m[nb] = m_new;
                l[nb] *= alpha;
#pragma unroll
                for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[nb][dt][e] *= alpha;
            }
            const float ref = m[nb] == -INFINITY ? 0.0f : m[nb];
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[nb][t][e], sc, -ref));
                    l[nb] += p;
                    pf[nb][t >> 1][(t & 1) * 4 + e] = f32_to_bf16(p);
                }
        }
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int s2 = 0; s2 < 2; ++s2) {
                bf16x8 vfrag;
                if constexpr (FP8) vfrag = s2 ? bf16x8_of_codes(vf[dt].z, vf[dt].w) : bf16x8_of_codes(vf[dt].x, vf[dt].y);
                else vfrag = as_bf16x8(vf[dt * 2 + s2]);
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) acc[nb][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vfrag, pf[nb][s2], acc[nb][dt], 0, 0, 0);
            }
        if (have) load_v(vt_next);
    }

    // ---- the four wavefronts meet
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        l[nb] += __shfl_xor(l[nb], 16, WAVE);
        l[nb] += __shfl_xor(l[nb], 32, WAVE);
        if (c == 0) {
            m_sh[wave][nb * 16 + r] = m[nb];
            l_sh[wave][nb * 16 + r] = l[nb];
        }
    }
    __syncthreads();
    constexpr int PER = D / 16;   // features of a thread
    float* const slot = a.slots + (size_t)(rq.slot0 + unit * parts + part) * FewSlot<D, NB>::FLOATS;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        float big = m_sh[0][nb * 16 + r];
#pragma unroll
        for (int w = 1; w < FEW_WAVES; ++w) big = fmaxf(big, m_sh[w][nb * 16 + r]);
        const float weight = m[nb] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m[nb] - big);
        if (nb > 0) __syncthreads();   // (the last rows' readers are done)
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
            f32x4 o = acc[nb][dt];
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] *= weight;
            *reinterpret_cast<f32x4*>(&red[wave][r][dt * 16 + c * 4]) = o;
        }
        __syncthreads();
        const int row = threadIdx.x >> 4, f0 = (threadIdx.x & 15) * PER, col = nb * 16 + row;
        float M = m_sh[0][col], L = 0.0f, o[PER];
#pragma unroll
        for (int w = 1; w < FEW_WAVES; ++w) M = fmaxf(M, m_sh[w][col]);
#pragma unroll
        for (int w = 0; w < FEW_WAVES; ++w) L += l_sh[w][col] == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(m_sh[w][col] - M) * l_sh[w][col];
        bool bad = !(fabsf(L) <= 3.402823466e38f);
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            o[j] = ((red[0][row][f0 + j] + red[1][row][f0 + j]) + (red[2][row][f0 + j] + red[3][row][f0 + j])) * (FP8 ? rq.v_scale : 1.0f);
            bad |= !(fabsf(o[j]) <= 3.402823466e38f);
        }
        const bool live = col < rows_here;
        const int col_c = min(col, rows_here - 1);
        bf16* const op = a.out + (size_t)(rq.row0 + token_of(col_c)) * a.ld_out + head_of(col_c) * D;
        const unsigned long long any = __builtin_amdgcn_ballot_w64(bad && live);
        const bool again = ((any >> (lane & 48)) & 0xffffu) != 0;   // (a row's sixteen threads are neighbours)
        if (!again && parts > 1) {
#pragma unroll
            for (int j = 0; j < PER; j += 4) *reinterpret_cast<f32x4*>(slot + (size_t)col * D + f0 + j) = f32x4{o[j], o[j + 1], o[j + 2], o[j + 3]};
            if (f0 == 0) {
                slot[(size_t)16 * NB * D + col] = M;
                slot[(size_t)16 * NB * (D + 1) + col] = L;
            }
        } else if (!again && live) {
            const float inv = 1.0f / L;
            if constexpr (PER == 8) {
                bf16x8 h;
#pragma unroll
                for (int j = 0; j < 8; ++j) h[j] = f32_to_bf16(o[j] * inv);
                *reinterpret_cast<bf16x8*>(op + f0) = h;
            } else {
                bf16x4 h;
#pragma unroll
                for (int j = 0; j < 4; ++j) h[j] = f32_to_bf16(o[j] * inv);
                *reinterpret_cast<bf16x4*>(op + f0) = h;
            }
        }
        if (__builtin_expect(any != 0, 0)) {
            for (int i = 0; i < 4; ++i) {   // the wavefront's four rows
                if (((any >> (16 * i)) & 0xffffu) == 0) continue;
                const int bc = nb * 16 + wave * 4 + i, tok = token_of(bc), head = head_of(bc);
                float em, el, eo[D / 64];
                exact_row<D, FP8>(a.q + (size_t)(rq.row0 + tok) * a.ld_q + head * D, sc, rq.P + tok, kb0, kb1, tile_at, em, el, eo);
                bf16* const bp = a.out + (size_t)(rq.row0 + tok) * a.ld_out + head * D;
#pragma unroll
                for (int j = 0; j < D / 64; ++j) {
                    const float v = eo[j] * (FP8 ? rq.v_scale : 1.0f);
                    if (parts > 1) slot[(size_t)bc * D + lane + 64 * j] = v;
                    else bp[lane + 64 * j] = f32_to_bf16(v / el);
                }
                if (parts > 1 && lane == 0) {
                    slot[(size_t)16 * NB * D + bc] = em;
                    slot[(size_t)16 * NB * (D + 1) + bc] = el;
                }
            }
        }
    }
}

// Joins the parts of an item:  M = max_p m_p,  out = sum_p 2^(m_p - M) O_p / sum_p 2^(m_p - M) l_p.  One workgroup per item and 32
// features, a quarter of the parts per 64 threads (16 rows x 4 chunks of 8 features).
template <int D, int NB, bool LIST, bool INLINE>
__global__ __launch_bounds__(256) void few_merge_kernel(FewArgs a, std::conditional_t<INLINE, InlineTable, NoTable> tab) {
    constexpr int MAXP = FEW_MAX_PARTS / 4;
    __shared__ float m_sh[4][16];
    __shared__ float red[4][64][9];
    const uint32_t* const table = table_of<INLINE>(tab, a.table);
    int req, parts, unit, kvh, row_first, rows_here;
    if constexpr (LIST) {
        unit = blockIdx.x;
        kvh = unit % a.hkv;
        row_first = unit / a.hkv;
        req = request_of(table, a.n_req, (uint32_t)row_first);
    } else {
        req = request_of(table + table_units_at(a.n_req), a.n_req, blockIdx.x);
        unit = (int)(blockIdx.x - table[table_units_at(a.n_req) + req]);
        row_first = kvh = 0;
    }
    const FewReq rq = reinterpret_cast<const FewReq*>(table + table_reqs_at(a.n_req))[req];
    parts = LIST ? a.list_parts : rq.parts;
    if (parts <= 1) return;
    if constexpr (LIST) {
        rows_here = a.g;
    } else {
        kvh = unit % a.hkv;
        row_first = unit / a.hkv * 16 * NB;
        rows_here = min(16 * NB, rq.T * a.g - row_first);
    }
    const int group = threadIdx.x >> 6, row = (threadIdx.x & 63) >> 2, f0 = blockIdx.y * 32 + (threadIdx.x & 3) * 8;
    for (int nb = 0; nb < NB; ++nb) {
        const int col = nb * 16 + row;
        if (nb * 16 >= rows_here) return;   // (the whole workgroup)
        const float* const base = a.slots + (size_t)(rq.slot0 + unit * parts) * FewSlot<D, NB>::FLOATS;
        float mp[MAXP], M = -INFINITY, L = 0.0f, o[8] = {};
#pragma unroll
        for (int i = 0; i < MAXP; ++i) {
            const int p = i * 4 + group;
            mp[i] = p < parts ? base[(size_t)p * FewSlot<D, NB>::FLOATS + (size_t)16 * NB * D + col] : -INFINITY;
            M = fmaxf(M, mp[i]);
        }
        if (nb > 0) __syncthreads();
        if ((threadIdx.x & 3) == 0) m_sh[group][row] = M;
        __syncthreads();
        M = fmaxf(fmaxf(m_sh[0][row], m_sh[1][row]), fmaxf(m_sh[2][row], m_sh[3][row]));
#pragma unroll
        for (int i = 0; i < MAXP; ++i) {
            const int p = i * 4 + group;
            if (p >= parts) continue;
            const float* const sp = base + (size_t)p * FewSlot<D, NB>::FLOATS;
            // (a part none of whose keys count has a row sum of zero and no reference)
            const float lp = sp[(size_t)16 * NB * (D + 1) + col], w = lp == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(mp[i] - M);
            L += w * lp;
            const f32x4 x = *reinterpret_cast<const f32x4*>(sp + (size_t)col * D + f0), y = *reinterpret_cast<const f32x4*>(sp + (size_t)col * D + f0 + 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                o[e] += w * x[e];
                o[4 + e] += w * y[e];
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) red[group][threadIdx.x & 63][e] = o[e];
        red[group][threadIdx.x & 63][8] = L;
        __syncthreads();
        if (group == 0 && col < rows_here) {
            const int t = threadIdx.x;
            const float inv = 1.0f / ((red[0][t][8] + red[1][t][8]) + (red[2][t][8] + red[3][t][8]));
            bf16x8 h;
#pragma unroll
            for (int e = 0; e < 8; ++e) h[e] = f32_to_bf16(((red[0][t][e] + red[1][t][e]) + (red[2][t][e] + red[3][t][e])) * inv);
            const int tok = LIST ? row_first - rq.row0 : (row_first + col) / a.g, head = kvh * a.g + (LIST ? col : (row_first + col) % a.g);
            *reinterpret_cast<bf16x8*>(a.out + (size_t)(rq.row0 + tok) * a.ld_out + head * D + f0) = h;
        }
    }
}

// A call's table from the staging buffer to the workspace.
static __global__ __launch_bounds__(256) void copy_table_kernel(const uint4* __restrict__ src, uint4* __restrict__ dst, int n) {
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i < n) dst[i] = src[i];
}
