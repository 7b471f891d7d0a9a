// Which blocks a token attends to: bounds on the keys of finished blocks, and the selection from them.
#pragma once
#include "attend_few.h"
#include "common.h"
#include "lanes.h"

typedef __attribute__((ext_vector_type(4))) int i32x4;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
RS_DEVICE uint4 ld_once_16(global_bytes p) {   // with the streaming hint
    return __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const __attribute__((address_space(1))) u32x4*>(p)));
}

constexpr float BOUND_LIMIT = 1.2676506002282294e30f;   // 2^100
constexpr int BOUND_LEAST = -100;

// The smallest e >= -100 with top <= 127 * 2^e  (0 <= top <= 2^100).
RS_DEVICE int code_exponent(float top) {
    // top = m 2^x, m in [1/2, 1): e = x - 7 where 128 m <= 127, x - 6 above
    const int x = __builtin_amdgcn_frexp_expf(top);
    const int e = x - 7 + (__builtin_amdgcn_frexp_mantf(top) * 128.0f > 127.0f ? 1 : 0);
    return top <= 127.0f / BOUND_LIMIT ? BOUND_LEAST : e;
}
RS_DEVICE float limited(float x) { return x == x ? fminf(fmaxf(x, -BOUND_LIMIT), BOUND_LIMIT) : 0.0f; }

// ---------------------------------------------------------------- bounds
// One wavefront per (block, KV head), bound by reading K once: all of a tile's loads are in flight together, a lane holding 8 (8-bit: 16)
// features of a sixteenth (an eighth) of the keys.  Maxima and minima do not depend on the order they are taken in, and
// codes are whole numbers: the result is the same bits whatever computes it.
//   e the least exponent with max |k| <= 127 2^e (limited to 2^100, NaN as 0),  high = ceil(max_key k / 2^e),  low = floor(min_key k / 2^e)
// Measured: 512 blocks of 4 KV heads, 34 MB, 9.6 us (3.5 TB/s; 3 us of it before the first bytes arrive); 32 blocks 5.8 us.
struct BoundsReq {          // 64 bytes: a FewReq with the bounds' memory in it
    uint64_t k;
    uint64_t head_bytes;
    uint32_t block_bytes;
    int32_t pages;
    uint64_t codes, units;  // of the layer
    int32_t room;           // blocks from a KV head's bounds to the next head's
    int32_t first;          // first block
    float k_scale;
    int32_t pad_[3];
};
static_assert(sizeof(BoundsReq) == 64, "sixteen words");

template <int D, bool FP8, class Tab>
__global__ __launch_bounds__(256) void key_bounds_kernel(int n_req, int hkv, int items, Tab tab) {
    constexpr int F = FP8 ? 16 : 8, CH = D / F, STEP = 64 / CH, N = 64 / STEP;   // features of a lane, lanes per key, keys per load, loads
    const uint32_t* const table = tab.w;
    const int lane = threadIdx.x & 63, id = (int)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (id >= items) return;
    const int r = request_of(table, n_req, (uint32_t)id);
    const BoundsReq rq = reinterpret_cast<const BoundsReq*>(table + table_reqs_at(n_req))[r];
    const int local = id - (int)table[r], h = local % hkv, block = rq.first + local / hkv;
    const uint64_t index = rq.pages == CONTIGUOUS ? (uint32_t)block : table[rq.pages + block];
    global_bytes kt = (global_bytes)(rq.k + (uint64_t)h * rq.head_bytes + index * rq.block_bytes);
    uint4 v[N];
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = ld_once_16(kt + (size_t)i * 1024 + lane * 16);   // (32768 tokens: 10.2 -> 9.8 us with the hint)
    const auto value = [&](const uint4& w, int e) RS_INLINE {
        const uint32_t x = e * (FP8 ? 1 : 2) / 4 == 0 ? w.x : e * (FP8 ? 1 : 2) / 4 == 1 ? w.y : e * (FP8 ? 1 : 2) / 4 == 2 ? w.z : w.w;
        if constexpr (FP8) {
            const f32x2 p = (e & 2) ? __builtin_amdgcn_cvt_pk_f32_fp8((int)x, true) : __builtin_amdgcn_cvt_pk_f32_fp8((int)x, false);
            return p[e & 1] * rq.k_scale;
        } else {
            return __builtin_bit_cast(float, (e & 1) ? x & 0xffff0000u : x << 16);
        }
    };
    float hi[F], lo[F];
#pragma unroll
    for (int e = 0; e < F; ++e) {
        hi[e] = -INFINITY;
        lo[e] = INFINITY;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float x = limited(value(v[i], e));
            hi[e] = fmaxf(hi[e], x);
            lo[e] = fminf(lo[e], x);
        }
        hi[e] = of_quarters(of_row<CH>(hi[e], larger_of()), larger_of());
        lo[e] = of_quarters(of_row<CH>(lo[e], smaller_of()), smaller_of());
    }
    float top = 0.0f;
#pragma unroll
    for (int e = 0; e < F; ++e) top = fmaxf(top, fmaxf(hi[e], -lo[e]));
    top = of_row<1>(top, larger_of());
    const int ex = __builtin_amdgcn_readfirstlane(code_exponent(top));
    if (ex > 0) {
        // A quotient by a unit above one may be too small for fp32, and zero; its code is 1 or -1 all the same.  (Without the branch: 9.2 -> 9.5 us.)
        const float half = __builtin_ldexpf(0.5f, ex);
#pragma unroll
        for (int e = 0; e < F; ++e) {
            hi[e] = hi[e] > 0.0f ? fmaxf(hi[e], half) : hi[e];
            lo[e] = lo[e] < 0.0f ? fminf(lo[e], -half) : lo[e];
        }
    }
    int8_t* const codes = reinterpret_cast<int8_t*>(rq.codes) + ((size_t)h * rq.room + block) * 2 * D;
    if (lane < CH) {
        union { int8_t b[F]; uint32_t w[F / 4]; } ch, cl;
#pragma unroll
        for (int e = 0; e < F; ++e) {
            ch.b[e] = (int8_t)(int)ceilf(__builtin_ldexpf(hi[e], -ex));
            cl.b[e] = (int8_t)(int)floorf(__builtin_ldexpf(lo[e], -ex));
        }
#pragma unroll
        for (int i = 0; i < F / 4; ++i) {
            reinterpret_cast<uint32_t*>(codes + lane * F)[i] = ch.w[i];
            reinterpret_cast<uint32_t*>(codes + D + lane * F)[i] = cl.w[i];
        }
    }
    if (lane == 0) reinterpret_cast<float*>(rq.units)[(size_t)h * rq.room + block] = __builtin_ldexpf(1.0f, ex);
}

// ---------------------------------------------------------------- selection
// One workgroup per (KV head, a few consecutive tokens of a request).
//  1. every token's p and n (see the score in the header), int8, into LDS;
//  2. scores of 16 blocks x 4 tokens (of 16 it has room for) per v_mfma_i32_16x16x64_i8 chain (the contraction runs over high and low codes), as keys
//     that order like the scores, into LDS;
//     score[block] = unit sum_d (p_d high_d - n_d low_d),  p and n the heads' positive and negative codes, summed: whole numbers, one product
//  3. a team per token finds the score that the last selected block has, digit by digit of the keys' range (a histogram in LDS per
//     digit: integers, in any order the same), and writes the blocks down in ascending order.
// These are the kernels for many tokens, many requests and very long caches; otherwise attend_selected_kernel takes the same steps itself.
// With many tokens a workgroup has four, a wavefront each, and takes all three steps.  With few (WIDE) it has one, and where that has more
// blocks than a workgroup scores at once, the first two steps are a launch of their own, of a workgroup per 256 blocks: a compute unit alone
// gets 33 bytes per ns, 16 us for the bounds of 2046 blocks.  (One launch, the last workgroup to finish selecting, behind the fence that makes
// keys visible across the chip: longer than a second launch, 7 us.  Keys stored and loaded past the L2s, without a fence, have not been measured.)
// Measured: one token on 2046 blocks 6.0 and 6.2 us, 256 tokens on 250 blocks 10.6: chains from queries to codes, scores, digits, list.  (Reductions
// over lanes stay in registers; through LDS the three took 7.3, 7.5 and 12.4.)
struct SelectReq {          // 64 bytes
    uint64_t codes, units;
    int32_t room;
    int32_t row0, T, P;
    int32_t pad_[8];
};
static_assert(sizeof(SelectReq) == 64, "sixteen words");
struct SelectArgs {
    int n_req, hkv, g, halvings;
    const bf16* q;
    long ld_q;
    int tokens;             // tokens of a workgroup: 1 if WIDE, else at most 4
    int blocks;             // keys there is room for per token, a multiple of 4
    int split;              // WIDE: workgroups that share a token's blocks in the score step
    uint32_t* shared_keys;  // WIDE, split > 1: the keys between the launches, [row][KV head][blocks]
    int n_blocks, n_first, n_last;
    int* chosen;
    // the attention kernel's table, from the staging buffer to the workspace: workgroups (x >= groups, y = 0) copy it
    const uint4* copy_from;
    uint4* copy_to;
    int copy_chunks, groups;
};
constexpr int SELECT_MAX_BLOCKS = 32768;   // 128 KB of keys
static_assert(SELECT_MAX_BLOCKS % 4 == 0, "keys of a token are whole 16-byte chunks");

RS_DEVICE uint32_t key_of_score(float s) {
    const uint32_t b = __builtin_bit_cast(uint32_t, s + 0.0f);   // (minus zero is zero)
    return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}

// What a team shares in LDS.
template <int TEAM>
struct alignas(16) SelectTeam {
    uint32_t hist[4 * 256];          // of each digit's search
    uint32_t low[TEAM], high[TEAM];
};

// A key that exactly `take` of key[lo .. hi) are above, 0 < take < hi - lo, but for *equals of those equal to it.  TEAM wavefronts, which
// count together and then all find the digit from the counts.
template <int TEAM>
RS_DEVICE uint32_t cut_of_keys(const uint32_t* key, int lo, int hi, int take, SelectTeam<TEAM>& sh, int* equals) {
    const int lane = threadIdx.x & 63, member = TEAM == 1 ? lane : (int)threadIdx.x, wave = TEAM == 1 ? 0 : (int)threadIdx.x >> 6;
    const auto meet = [&]() RS_INLINE {
        if constexpr (TEAM > 1) __syncthreads();
        else __builtin_amdgcn_wave_barrier();   // (one wavefront's LDS accesses are in order)
    };
    for (int i = member; i < 256; i += 64 * TEAM) *reinterpret_cast<uint4*>(&sh.hist[i * 4]) = make_uint4(0u, 0u, 0u, 0u);
    uint32_t low = 0xffffffffu, high = 0u;
    for (int b = lo + member; b < hi; b += 64 * TEAM) {
        low = min(low, key[b]);
        high = max(high, key[b]);
    }
    low = of_wave(low, smaller_of());
    high = of_wave(high, larger_of());
    if constexpr (TEAM > 1) {
        if (lane == 0) {
            sh.low[wave] = low;
            sh.high[wave] = high;
        }
        __syncthreads();
        low = of_row<1>(sh.low[lane % TEAM], smaller_of());   // (a row of lanes has them all)
        high = of_row<1>(sh.high[lane % TEAM], larger_of());
        static_assert(TEAM <= 16, "a row of lanes");
    }
    low = __builtin_amdgcn_readfirstlane(low);
    high = __builtin_amdgcn_readfirstlane(high);
    uint32_t prefix = 0, left = (uint32_t)take;
    int top = high == low ? 0 : 32 - __builtin_clz(high - low);   // bits of key - low that are not known yet
    for (int digit = 0; top > 0; ++digit) {
        const int shift = max(top - 8, 0);
        const uint32_t mask = (1u << (top - shift)) - 1u;
        uint32_t* const hist = sh.hist + digit * 256;
        meet();
        for (int b = lo + member; b < hi; b += 64 * TEAM) {
            const uint32_t x = key[b] - low;
            if (digit == 0 || (x >> top) == prefix) atomicAdd(&hist[(x >> shift) & mask], 1u);
        }
        meet();
        // lane: digits 4 lane .. 4 lane + 3, counted from the largest
        const uint4 h = *reinterpret_cast<const uint4*>(&hist[lane * 4]);
        const uint32_t mine = h.x + h.y + h.z + h.w, sum = sum_from_lane(mine), above = sum - mine;
        uint32_t rest = left - above, d = 3;   // (of the one lane that has the digit)
        const uint32_t count[4] = {h.x, h.y, h.z, h.w};
#pragma unroll
        for (int i = 3; i > 0; --i)
            if (d == (uint32_t)i && rest > count[i]) {
                rest -= count[i];
                d = i - 1;
            }
        const uint32_t in_digit = d == 3 ? h.w : d == 2 ? h.z : d == 1 ? h.y : h.x;
        const int who = (int)__builtin_ctzll(__builtin_amdgcn_ballot_w64(above < left && left <= sum));
        left = __builtin_amdgcn_readlane(rest, who);
        prefix = (prefix << (top - shift)) | ((uint32_t)who * 4 + __builtin_amdgcn_readlane(d, who));
        top = shift;
        if (top > 0 && left == (uint32_t)__builtin_amdgcn_readlane(in_digit, who)) {
            // all of that digit belong: all from its smallest key on; (prefix << top is not 0: some keys are left out)
            *equals = 0;
            return low + (prefix << top) - 1u;
        }
    }
    *equals = (int)left;
    return low + prefix;
}

constexpr int SELECT_U = 4;                            // groups of 16 blocks that a wavefront has in flight
constexpr int SELECT_ROUND = 4 * 16 * SELECT_U;        // blocks that a workgroup scores at a time
// Scores of blocks [s0, s1) for nt <= TOKENS tokens, whose queries of the KV head start at q, as keys into `to`: by four wavefronts, from s0 +
// start on, `step` further each time.  u: the tokens' p and n.
template <int D, int TOKENS>
RS_DEVICE void score_blocks(const bf16* q, long ld_q, int g, int halvings, int nt, const int8_t* codes, const float* units, int s0, int s1, int start, int step,
                            int8_t (*u)[2 * D], uint32_t* to, int ld_to) {
    constexpr int KK = 2 * D / 64, U = SELECT_U;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    constexpr int W = D / 64;   // features of a lane: W lane ..
    const int r = lane & 15, c = lane >> 4;
    i32x4 x[U][KK];
    float unit[U];
    const auto load = [&](int b) RS_INLINE {   // bounds of the wavefront's blocks b ..
#pragma unroll
        for (int v = 0; v < U; ++v) {
            const int block = min(b + v * 16 + r, s1 - 1);
            const int8_t* const src = codes + (size_t)block * 2 * D + c * 16;
#pragma unroll
            for (int k = 0; k < KK; ++k) x[v][k] = *reinterpret_cast<const i32x4*>(src + k * 64);
            unit[v] = units[block];
        }
    };
    // a wavefront's token, eight heads at a time, their loads in flight together and before the bounds'
    const bf16* const query = q + (size_t)min(wave, nt - 1) * ld_q + lane * W;
    typedef __attribute__((ext_vector_type(W))) __bf16 heads_t;
    heads_t qh[8];
    const auto load_heads = [&](int i0) RS_INLINE {
#pragma unroll
        for (int i = 0; i < 8; ++i) qh[i] = *reinterpret_cast<const heads_t*>(query + (size_t)min(i0 + i, g - 1) * D);
    };
    load_heads(0);
    int b = s0 + start + wave * 16 * U;
    load(b);   // (under way while the queries become codes)
    if (wave < nt) {
        int p[W] = {}, n[W] = {};
        float top = 0.0f;
        for (int i0 = 0;;) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int j = 0; j < W; ++j) top = fmaxf(top, fabsf(limited((float)qh[i][j])));
            i0 += 8;
            if (i0 >= g) break;
            load_heads(i0);
        }
        const int ex = code_exponent(of_wave(top, larger_of()));
        for (int i0 = 0; i0 < g; i0 += 8) {
            if (g > 8) load_heads(i0);
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int j = 0; j < W; ++j) {
                    const int code = i0 + i < g ? (int)rintf(__builtin_ldexpf(limited((float)qh[i][j]), -ex)) : 0;
                    p[j] += max(code, 0);
                    n[j] += max(-code, 0);
                }
        }
        const int half = (1 << halvings) >> 1;
#pragma unroll
        for (int j = 0; j < W; ++j) {
            u[wave][lane * W + j] = (int8_t)((p[j] + half) >> halvings);
            u[wave][D + lane * W + j] = (int8_t)(-((n[j] + half) >> halvings));
        }
    }
    __syncthreads();
    i32x4 uf[KK];   // (rows past the tokens' are not used)
#pragma unroll
    for (int k = 0; k < KK; ++k) uf[k] = *reinterpret_cast<const i32x4*>(&u[TOKENS == 1 ? 0 : r & 3][k * 64 + c * 16]);
    while (b < s1) {
#pragma unroll
        for (int v = 0; v < U; ++v) {
            i32x4 dot = {0, 0, 0, 0};
#pragma unroll
            for (int k = 0; k < KK; ++k) dot = __builtin_amdgcn_mfma_i32_16x16x64_i8(uf[k], x[v][k], dot, 0, 0, 0);
            const int block = b + v * 16 + r;   // token 4 c + e
            if (c == 0 && block < s1)
#pragma unroll
                for (int e = 0; e < TOKENS; ++e)
                    if (e < nt) to[e * ld_to + block - s0] = key_of_score((float)dot[e] * unit[v]);
        }
        b += step;
        if (b < s1) load(b);
    }
}

// The blocks that a token whose own block is `own` attends to, ascending, -1 behind the last of n_blocks; key[b]: block b's score.  A team of TEAM
// wavefronts; chunk_more, chunk_equal: a word per 64 blocks each (TEAM > 1).
template <int TEAM>
RS_DEVICE void pick_blocks(const uint32_t* key, int own, int n_blocks, int n_first, int n_last, SelectTeam<TEAM>& sh, uint32_t* chunk_more, uint32_t* chunk_equal,
                           int* out) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned long long below = lane == 0 ? 0ull : ~0ull >> (64 - lane);   // the lanes before this one
    const int lo = min(n_first, own + 1), hi = max(lo, own + 1 - n_last);   // blocks lo .. hi - 1 compete
    const int take = min(max(n_blocks - (own + 1 - (hi - lo)), 0), hi - lo);
    uint32_t cut = 0;   // the take-th largest key; of the blocks that have it, the first `equals`
    int equals = 0;
    const bool some = take > 0 && take < hi - lo;
    if (some) cut = cut_of_keys<TEAM>(key, lo, hi, take, sh, &equals);
    // is block b taken for sure; does it have the cut's key
    const auto taken = [&](int b, bool& eq) RS_INLINE {
        const bool competes = b >= lo && b < hi;
        const uint32_t k = some && competes ? key[b] : 0u;
        eq = some && competes && k == cut;
        return competes ? (some ? k > cut : take > 0) : b <= own;
    };
    const int chunks = own / 64 + 1;   // of 64 blocks
    if constexpr (TEAM == 1) {
        int done = 0;
        for (int ch = 0; ch < chunks && done < n_blocks; ++ch) {
            bool eq;
            bool sel = taken(ch * 64 + lane, eq);
            const unsigned long long eqs = __builtin_amdgcn_ballot_w64(eq);
            if (eq) sel = __popcll(eqs & below) < equals;
            equals -= min(equals, (int)__popcll(eqs));
            const unsigned long long sels = __builtin_amdgcn_ballot_w64(sel);
            const int at = done + (int)__popcll(sels & below);
            if (sel && at < n_blocks) out[at] = ch * 64 + lane;
            done += (int)__popcll(sels);
        }
        for (int i = min(done, n_blocks) + lane; i < n_blocks; i += 64) out[i] = -1;
    } else {
        for (int ch = wave; ch < chunks; ch += TEAM) {
            bool eq;
            const bool sel = taken(ch * 64 + lane, eq);
            const uint32_t more = (uint32_t)__popcll(__builtin_amdgcn_ballot_w64(sel)), equal = (uint32_t)__popcll(__builtin_amdgcn_ballot_w64(eq));
            if (lane == 0) {
                chunk_more[ch] = more;
                chunk_equal[ch] = equal;
            }
        }
        __syncthreads();
        uint32_t more_before = 0, equal_before = 0;   // in the chunks before these 64
        for (int c0 = 0; c0 < chunks; c0 += 64) {
            const bool there = c0 + lane < chunks;
            const uint32_t more_from = sum_from_lane(there ? chunk_more[c0 + lane] : 0u), equal_from = sum_from_lane(there ? chunk_equal[c0 + lane] : 0u);
            const uint32_t more_end = more_before + __builtin_amdgcn_readlane(more_from, 0), equal_end = equal_before + __builtin_amdgcn_readlane(equal_from, 0);
            for (int ch = c0 + wave; ch < min(chunks, c0 + 64); ch += TEAM) {
                const int more = (int)(more_end - __builtin_amdgcn_readlane(more_from, ch - c0)), equal = (int)(equal_end - __builtin_amdgcn_readlane(equal_from, ch - c0));
                bool eq;
                bool sel = taken(ch * 64 + lane, eq);
                const unsigned long long eqs = __builtin_amdgcn_ballot_w64(eq);
                if (eq) sel = equal + (int)__popcll(eqs & below) < equals;
                const unsigned long long sels = __builtin_amdgcn_ballot_w64(sel);
                const int at = more + min(equal, equals) + (int)__popcll(sels & below);
                if (sel && at < n_blocks) out[at] = ch * 64 + lane;
            }
            more_before = more_end;
            equal_before = equal_end;
        }
        const int all = min(n_blocks, own + 1);
        for (int i = all + (int)threadIdx.x; i < n_blocks; i += 64 * TEAM) out[i] = -1;
    }
}

enum SelectSteps { SELECT_ALL = 0, SELECT_SCORES = 1, SELECT_FROM_SCORES = 2 };
template <int D, bool WIDE, int STEPS, class Tab>
__global__ __launch_bounds__(STEPS == SELECT_FROM_SCORES ? 1024 : 256) void block_select_kernel(SelectArgs a, Tab tab) {
    static_assert(WIDE || STEPS == SELECT_ALL, "only few tokens take two launches");
    constexpr int WAVES = STEPS == SELECT_FROM_SCORES ? 16 : 4, TEAM = WIDE ? WAVES : 1, TEAMS = WAVES / TEAM;
    extern __shared__ __attribute__((aligned(16))) uint32_t keys[];   // [tokens][blocks]
    __shared__ __attribute__((aligned(16))) int8_t u[4][2 * D];
    __shared__ __attribute__((aligned(16))) SelectTeam<TEAM> team_sh[TEAMS];
    __shared__ uint32_t chunk_more[TEAM == 1 ? 1 : SELECT_MAX_BLOCKS / 64], chunk_equal[TEAM == 1 ? 1 : SELECT_MAX_BLOCKS / 64];
    const uint32_t* const table = tab.w;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = blockIdx.y;
    if (STEPS != SELECT_FROM_SCORES && (int)blockIdx.x >= a.groups) {
        const int i = ((int)blockIdx.x - a.groups) * 64 * WAVES + (int)threadIdx.x;
        if (h == 0 && i < a.copy_chunks) a.copy_to[i] = a.copy_from[i];
        return;
    }
    const int split = STEPS == SELECT_SCORES ? a.split : 1, share = (int)blockIdx.x % split, item = (int)blockIdx.x / split;
    const int req = request_of(table, a.n_req, (uint32_t)item);
    const SelectReq rq = reinterpret_cast<const SelectReq*>(table + table_reqs_at(a.n_req))[req];
    const int t0 = (item - (int)table[req]) * a.tokens, nt = min(a.tokens, rq.T - t0);
    const int b_last = (rq.P + t0 + nt - 1) / 64;          // own block of the last token
    // blocks that can need a score
    const int s0 = min(a.n_first, b_last), s1 = max(s0, b_last + 1 - a.n_last);
    const bool scored = b_last + 1 > a.n_blocks && s1 > s0;   // (else every token takes all it has, or none but the forced ones)
    uint32_t* const shared = STEPS == SELECT_ALL ? nullptr : a.shared_keys + ((size_t)(rq.row0 + t0) * a.hkv + h) * a.blocks;
    uint32_t* const to = STEPS == SELECT_SCORES ? shared : keys;   // where the scores' keys go
    if (scored) {
        if constexpr (STEPS == SELECT_FROM_SCORES)
            for (int i = threadIdx.x * 4; i < s1 - s0; i += 64 * WAVES * 4) *reinterpret_cast<uint4*>(&keys[i]) = *reinterpret_cast<const uint4*>(&shared[i]);
        else
            score_blocks<D, WIDE ? 1 : 4>(a.q + (size_t)(rq.row0 + t0) * a.ld_q + (size_t)h * a.g * D, a.ld_q, a.g, a.halvings, nt,
                                          reinterpret_cast<const int8_t*>(rq.codes) + (size_t)h * rq.room * 2 * D,
                                          reinterpret_cast<const float*>(rq.units) + (size_t)h * rq.room, s0, s1, share * SELECT_ROUND, split * SELECT_ROUND, u, to,
                                          a.blocks);
        __syncthreads();
    }
    if constexpr (STEPS == SELECT_SCORES) return;
    for (int t = TEAM == 1 ? wave : 0; t < nt; t += TEAMS)
        pick_blocks<TEAM>(keys + t * a.blocks - s0, (rq.P + t0 + t) / 64, a.n_blocks, a.n_first, a.n_last, team_sh[TEAM == 1 ? wave : 0], chunk_more, chunk_equal,
                          a.chosen + ((size_t)(rq.row0 + t0 + t) * a.hkv + h) * a.n_blocks);
}
