// Attention of few query rows per KV head: the tokens a request generates one at a time, a few drafted ones, or - with a
// list of blocks per token - any tokens that attend to selected blocks only.
//
//   out[row] = sum_k w_k value_k / sum_k w_k,   w_k = 2^(scale log2e (q . key_k - m)),  m a reference that tracks the maximum
//
// Bound by the bytes of the keys and values: a tile of 64 keys is 32 KB (d = 128, bfloat16), and the rows that share it - the g
// query heads of a KV head, times the tokens - give it 16 MFMAs of 16 clocks per 16 rows and product.  So wavefronts share no tiles: each
// streams its own through its own LDS, by DMA, without barriers, in units of 4 KB - a quarter of a tile's keys, then of its values - and two
// places: the unit after the next is under way as soon as this one is in registers.  (Loads straight into the MFMA operand layout, where
// neighbouring lanes are different keys, need no LDS, but the address unit then takes 64 clocks for a load of a KB instead of 16: a
// compute unit gets 16 bytes per clock, whatever the cache they come from.)  A workgroup takes 34 KB of LDS and 115 to 120 registers (d = 128), so that four share
// a compute unit; units of 8 KB and two of them: one token on 2000 11.7 us a pass instead of 10.3, selected blocks 59.6 instead of 57.3.
//
// As in the chunk kernel (attention.h) the transposed products keep a query in one lane (lane & 15):
//   S^T[key, query] = K Q^T,   O^T[d, query] = V^T P^T   with v_mfma_f32_16x16x32_bf16
// and the assignment of MFMA rows to keys is chosen so that the four scores a lane holds of each of its sub-tiles are, put together, the
// consecutive keys that it has to feed to the second product.  8-bit tiles are loaded 16 codes at a time (the keys' order
// changes with it) and become bfloat16, exactly, in registers; their scales go into the softmax's scale and the output.
// Scores, references, row sums and output sums are fp32.  References are scores as the products leave them, and a weight's exponent is their
// difference times the scale: zero, exactly, for the key that is the reference.  (With the scale in the reference, whose rounding an fma does not
// repeat, all weights of a row move by that rounding, and from scores of 2^32 on out of fp32's range.)
//  A weight becomes bfloat16 for the second product, whose operands have 16 bits; the row
// sum takes it before that.  The output is rounded once.  (Errors against 64 bits are 0.0021 to 0.0023 of the output then; 0.0017, the output's own
// rounding, with weights of 32 bits, which would take a second product for what the first leaves of each.)  A masked key has weight zero; where its value is an infinity or NaN the row
// comes out not finite and is done again by exact_row, which leaves masked values alone.
//
// Work item = (request, KV head, part of the key range), with up to 64 stacked rows.  A wavefront has 16 of them (RB = 1), and with up to 16
// rows the four wavefronts of a workgroup share the item's tiles, with up to 32 two pairs do, with more each takes every tile, which the
// others' loads have brought into the caches; or it has 32 (RB = 2), so that tiles are loaded half as often, for 174 to 179 registers
// and longer chains.  They meet in LDS once per 16 rows; parts leave unnormalised sums, references and row sums in slots that
// few_merge_kernel joins.
//
// Measured, us of this kernel (28 query heads, 4 KV heads, d = 128): one token on 2000, 4.1 MB, 6.3 and the merge 3.8, what dependent loads
// take; 64 single tokens on up to 8000, 468 MB, 83 (5.6 TB/s); 16 on up to 32000, 8 bits, 318 MB, 55 (5.8 TB/s); 24 requests of 3 drafted tokens on
// up to 6000 and one of 12, 64 and 8 heads, 240 MB, 46 to 47 (5.1 TB/s, RB = 2); 256 tokens with 32 selected blocks each, 1.07 GB from the L2s (90 %
// of the reads hit), 46 to 48 (23 TB/s: LDS, which takes and gives every byte, is busy for 60 % of that).
#pragma once
#include "attention.h"
#include "common.h"
#include "exact_row.h"
#include "lanes.h"
#include "kv_fp8.h"

// Descriptors of a call: in the kernel arguments where they fit, else copied to the workspace ahead of the kernel.  Page numbers that do not fit
// beside them are read where the host left them: a wavefront does it once per 64 tiles.  (All of it read in place: three such reads, one after
// the other, at the start of every workgroup, as long as the copy.)
constexpr int TABLE_WORDS = 928;
struct InlineTable { uint32_t w[TABLE_WORDS]; };
struct SmallTable { uint32_t w[112]; };   // of a few requests: a launch of 4 KB of arguments takes the host 1.3 us more
struct NoTable {};

constexpr int32_t CONTIGUOUS = INT32_MIN;

// One request, 48 bytes.  The keys' tile of block b of KV head h:  k + (h head_tiles + index) tile in a contiguous cache, index = b, and
// k + (2 Hkv index + h) tile in a paged one, index = the block's page; values Hkv head_tiles tiles further on (a page holds its KV heads'
// keys, then their values: head_tiles = 1).
struct FewReq {
    uint64_t k;
    int32_t head_tiles;
    int32_t pages;         // its first page number's place among the page numbers; CONTIGUOUS: the cache is
    int32_t row0, T, P;    // first row, rows, position of the first row
    int32_t parts;         // parts of the key range
    int32_t slot0;         // of its first part
    float k_scale, v_scale;
    int32_t once;          // nothing of it that is read is read again soon
};
constexpr int REQ_WORDS = 12;
static_assert(sizeof(FewReq) == 4 * REQ_WORDS, "REQ_WORDS");

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

// Eight E4M3 codes to bfloat16, exactly.
RS_DEVICE bf16x8 bf16x8_of_codes(uint32_t lo, uint32_t hi) {
    bf16x8 o;
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
    o[0] = a[0]; o[1] = a[1]; o[2] = b[0]; o[3] = b[1]; o[4] = c[0]; o[5] = c[1]; o[6] = d[0]; o[7] = d[1];
    return o;
}
struct FewArgs {
    const uint32_t* table;   // device table (NoTable)
    const uint32_t* pages;   // page numbers; null: behind the table's requests
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

#define RS_UNIT __device__ __forceinline__
constexpr int FEW_WAVES = 4;
constexpr int FEW_MAX_PARTS = 64;
constexpr float FEW_HEADROOM = 8.0f;   // the reference moves when a score exceeds it by this many powers of two

// Blocks of 16 rows that `rows` of them are handled as: 1, 2 or 4.
__host__ __device__ inline int few_row_blocks(int rows) { return rows <= 16 ? 1 : rows <= 32 ? 2 : 4; }

template <int D>
struct FewSlot {   // of a part and 16 rows: [16][D] sums, then references, then row sums
    static constexpr size_t FLOATS = (size_t)16 * (D + 2);
};

constexpr int FEW_GROUP = 64;          // stacked rows of an item
// An item's rows, and where they are in q and out.
template <bool LIST>
struct FewRows {
    int kvh, g, first, tok0, rows;   // first: of the request's stacked rows; tok0: its token.  (LIST: the g heads of one token)
    __device__ __forceinline__ int token(int i) const { return LIST ? tok0 : (first + i) / g; }
    __device__ __forceinline__ int head(int i) const { return kvh * g + (LIST ? i : (first + i) % g); }
    // Takes the rows of group `group` of a request's `all`.
    __device__ __forceinline__ void take(int group, int all) {
        first = group * FEW_GROUP;
        rows = min(FEW_GROUP, all - first);
        tok0 = first / g;
    }
};

constexpr int FEW_UNIT = 4096;   // bytes of a unit (a tile's keys or values, if they are fewer)
// How a wavefront streams a tile: its keys, then its values (V^T), in PER units each of BYTES bytes.  16-byte chunks sit at places
// of their row that make the 8 lanes of a read, which are 8 keys or features of one chunk, meet different banks; a load instruction
// fills 1 KB of LDS linearly by lane, each lane fetching the chunk that belongs in its place.
template <int D, bool FP8>
struct FewUnit {
    static constexpr int EL = FP8 ? 1 : 2;
    static constexpr int TILE = 64 * D * EL;                    // bytes of a tile's keys, or values
    static constexpr int PER = TILE > FEW_UNIT ? TILE / FEW_UNIT : 1;
    static constexpr int BYTES = TILE / PER, LOADS = BYTES / 1024;
    static constexpr int SUBS = 4 / PER;                        // sub-tiles of 16 keys in a K unit
    static constexpr int K_ROW = D * EL, K_CHUNKS = K_ROW / 16;   // a key's bytes, chunks
    static constexpr int K_READS = K_CHUNKS / 4;                // 16-byte reads of a lane per 16 keys
    static constexpr int V_ROW = 64 * EL;                       // a feature's bytes
    static constexpr int V_READS = V_ROW / 64;                  // 16-byte reads of a lane per 16 features
    static_assert(SUBS >= 1, "a K unit is whole sub-tiles");
    // Key of MFMA row i of sub-tile t: the scores a lane ends up with - rows 4 c .. 4 c + 3 of every sub-tile - are the keys it multiplies
    // with values, consecutive ones: 8 of every 32, or with 8-bit values, which come 16 to a chunk, 16 of 64.
    RS_UNIT static int key_of(int t, int i) {
        return FP8 ? (i >> 2) * 16 + t * 4 + (i & 3) : (t >> 1) * 32 + (i >> 2) * 8 + (t & 1) * 4 + (i & 3);
    }
    // A K unit's rows in LDS are its keys in order, four groups of 4 SUBS neighbours (bfloat16 with SUBS = 4: two times four groups of 8).
    // Row of MFMA row i of the unit's first sub-tile, rows from there to sub-tile t, and back: MFMA row of a row; key of a row of unit h.
    static constexpr int GROUP = FP8 || SUBS < 4 ? 4 * SUBS : 8;
    RS_UNIT static int row_of(int i) { return (i >> 2) * GROUP + (i & 3); }
    RS_UNIT static constexpr int sub_step(int t) { return !FP8 && SUBS == 4 ? (t >> 1) * 32 + (t & 1) * 4 : t * 4; }
    RS_UNIT static int mfma_row(int row) { return (row / GROUP & 3) * 4 + (row & 3); }
    RS_UNIT static constexpr int key_of_row(int h, int row) {
        if (SUBS == 4) return row;
        if (FP8) return row / GROUP * 16 + h * GROUP + row % GROUP;
        return SUBS == 2 ? h * 32 + row : (h >> 1) * 32 + row / 4 * 8 + (h & 1) * 4 + row % 4;
    }
    RS_UNIT static int k_swizzle(int row) {   // of a row's chunks: from its MFMA row
        const int i = mfma_row(row);
        return K_CHUNKS == 16 ? i : K_CHUNKS == 8 ? i & 7 : (i >> 1) & 3;
    }
    RS_UNIT static int v_swizzle(int feature) { return V_ROW == 128 ? feature & 7 : (feature >> 1) & 3; }
    RS_UNIT static uint32_t k_place(int row, int chunk) { return (uint32_t)(row * K_ROW + (chunk ^ k_swizzle(row)) * 16); }
    RS_UNIT static uint32_t v_place(int feature, int chunk) { return (uint32_t)(feature * V_ROW + (chunk ^ v_swizzle(feature)) * 16); }
    // Load instruction i fills rows K_LOAD i .. of the unit, keys that are neighbours: where in them a lane's chunk is, and where they are
    // in the tile.  (Values: contiguous, and every instruction like the first: a KB is 8 or 16 features.)
    static constexpr int K_LOAD = 1024 / K_ROW;
    RS_UNIT static uint32_t k_source(int i, int lane) {
        return (uint32_t)(lane / K_CHUNKS * K_ROW + (lane % K_CHUNKS ^ k_swizzle(i * K_LOAD + lane / K_CHUNKS)) * 16);
    }
    RS_UNIT static constexpr int k_start(int h, int i) { return key_of_row(h, i * K_LOAD) * K_ROW; }
    RS_UNIT static uint32_t v_source(int lane) { return v_place(lane / (V_ROW / 16), lane % (V_ROW / 16)); }
};

constexpr int FEW_ONCE = 2;   // cache policy (nt)
// LDS of a workgroup: each wavefront's keys and values, in the end all their sums; and, apart from it (the compiler waits for the DMA into
// whatever it cannot tell from what it reads), references and row sums.
template <int D, bool FP8>
constexpr int FEW_LDS = FEW_WAVES * (2 * FewUnit<D, FP8>::BYTES > 16 * (D + 4) * 4 ? 2 * FewUnit<D, FP8>::BYTES : 16 * (D + 4) * 4);
typedef float FewStats[FEW_WAVES][16];
// Part `part` of `parts` of an item of n tiles, or of a list's n blocks: unit `unit` of its request (of all, with lists) writes its rows or slots.
template <int D, bool FP8, bool LIST, int RB>
RS_DEVICE void attend_rows(const FewArgs& a, const FewReq& rq, const uint32_t* pages, const FewRows<LIST>& rows, int part, int parts, int unit, int n,
                           const int* list, char* lds, FewStats& m_sh, FewStats& l_sh) {
    typedef FewUnit<D, FP8> U;
    constexpr int KS = D / 32, DT = D / 16, NT = U::SUBS, DTU = DT / U::PER;   // sub-tiles of a K unit, feature blocks of a V unit
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, c = lane >> 4;
    // (a part, and a wavefront's share of it: the quotient, one more for as many of the first as the remainder)
    const int kb0 = n / parts * part + min(part, n % parts), held = n / parts + (part < n % parts);
    const int sets = max(few_row_blocks(rows.rows) / RB, 1), set = wave & (sets - 1), sharers = FEW_WAVES / sets, share = wave / sets;
    const int row0 = set * RB * 16;                                 // a wavefront's first row, of 16 RB
    const bool two = RB == 2 && rows.rows > row0 + 16;
    const int slot_blocks = few_row_blocks(LIST ? a.g : min(rq.T * a.g, FEW_GROUP));   // of a part (the last group may have fewer)
    const uint64_t k_head = rq.k + (uint64_t)rows.kvh * (uint32_t)rq.head_tiles * U::TILE;
    const uint64_t v_head = k_head + (uint64_t)a.hkv * (uint32_t)rq.head_tiles * U::TILE;
    const auto tile_at = [&](int i, global_bytes& kt, global_bytes& vt, int& block) RS_INLINE {   // (exact_row's)
        block = i;
        if constexpr (LIST) block = list[i];
        const uint64_t at = rq.pages == CONTIGUOUS ? (uint64_t)(uint32_t)block : (uint64_t)pages[rq.pages + block] * (uint32_t)(2 * a.hkv);
        kt = (global_bytes)(k_head + at * U::TILE);
        vt = (global_bytes)(v_head + at * U::TILE);
    };

    // ---- queries
    bf16x8 qf[RB][KS];
    int qpos[RB];
#pragma unroll
    for (int b = 0; b < RB; ++b) {
        const int i = min(row0 + b * 16 + r, rows.rows - 1);   // (rows past the end repeat the last one and are not stored)
        qpos[b] = rq.P + rows.token(i);
        const bf16* p = a.q + (size_t)(rq.row0 + rows.token(i)) * a.ld_q + rows.head(i) * D;
#pragma unroll
        for (int kk = 0; kk < KS; ++kk)
            qf[b][kk] = *reinterpret_cast<const bf16x8*>(p + (FP8 ? (kk >> 1) * 64 + c * 16 + (kk & 1) * 8 : kk * 32 + c * 8));
    }
    const int seen_by_all = rq.P + rows.tok0;   // every row of the item sees the keys up to here
    const float sc = FP8 ? a.scale_log2e * rq.k_scale : a.scale_log2e;

    f32x4 acc[RB][DT];
    float m[RB], l[RB];
#pragma unroll
    for (int b = 0; b < RB; ++b) {
        m[b] = -INFINITY;
        l[b] = 0.0f;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) acc[b][dt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    // ---- this wavefront's share of the tiles: neighbours, so that page numbers read across the host link are few lines; of a list every
    // sharers-th, so that wavefronts all over the chip pass the same blocks at about the same time and find them in the L2s.  Their places
    // (page or block) are in a register, a lane each, 64 at a time.
    const int own = held / sharers + (share < held % sharers);
    const int first = kb0 + (LIST ? share : held / sharers * share + min(share, held % sharers)), stride = LIST ? sharers : 1;
    const int tiles = row0 < rows.rows ? own : 0, last = first + max(own - 1, 0) * stride;
    int place = 0, number = 0;
    const auto look_up = [&](int j0) RS_INLINE {   // of tiles j0 .. j0 + 63
        const int i = min(first + (j0 + lane) * stride, last);
        number = LIST ? list[i] : i;
        place = rq.pages == CONTIGUOUS ? number : (int)pages[rq.pages + number];
    };
    typedef __attribute__((address_space(3))) void* lds_ptr;
    char* const mine = lds + wave * 2 * U::BYTES;
    const uint32_t place_bytes = (rq.pages == CONTIGUOUS ? 1u : 2u * (uint32_t)a.hkv) * U::TILE;
    uint32_t k_src[8];   // where a lane's 16 bytes of a load instruction come from
    static_assert(U::LOADS <= 8, "k_src");
#pragma unroll
    for (int i = 0; i < U::LOADS; ++i) k_src[i] = U::k_source(i, lane);
    const uint32_t v_src = U::v_source(lane);
    // unit h of tile j: 0 .. PER - 1 its keys, then its values; unit h goes to place h & 1
    const auto fetch = [&](int j, int h) RS_INLINE {
        const bool keys = h < U::PER;
        const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
            (void*)((keys ? k_head : v_head) + (uint64_t)(uint32_t)__builtin_amdgcn_readlane(place, j & 63) * place_bytes), 0, U::TILE, 0x00020000);
        char* const to = mine + (h & 1) * U::BYTES;
        const auto load = [&](auto policy) RS_INLINE {
#pragma unroll
            for (int i = 0; i < U::LOADS; ++i) {
                const uint32_t from = keys ? k_src[i] : v_src;   // (named: template-dependent arguments of the builtin break the host-side stub)
                const int further = keys ? U::k_start(h, i) : h % U::PER * U::BYTES + i * 1024;
                constexpr int aux = decltype(policy)::value;
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_ptr)(uintptr_t)(uint32_t)(uintptr_t)(to + i * 1024), 16, from, further, 0, aux);
            }
        };
        if (!LIST && rq.once) load(std::integral_constant<int, FEW_ONCE>{});
        else load(std::integral_constant<int, 0>{});
    };
    // (the compiler does not see LDS written by DMA, nor may it move a refill above the reads of what it overwrites)
    const auto wait_loads = [&](bool others) RS_INLINE {   // others: U::LOADS younger ones may be in flight
        __builtin_amdgcn_sched_barrier(0);
        if (others) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(U::LOADS) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    const auto reads_done = [&]() RS_INLINE {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    uint32_t k_at[4], v_at[2];   // a lane's fragments: sub-tile 0, features 0 .. 15
#pragma unroll
    for (int i = 0; i < U::K_READS; ++i) k_at[i] = U::k_place(U::row_of(r), i * 4 + c);
#pragma unroll
    for (int i = 0; i < U::V_READS; ++i) v_at[i] = U::v_place(r, i * 4 + c);

    if (tiles > 0) {
        look_up(0);
        fetch(0, 0);
        fetch(0, 1);
    }
    int block = __builtin_amdgcn_readlane(number, 0);
    for (int j = 0; j < tiles; ++j) {
        const int key0 = block * 64;
        const bool more = j + 1 < tiles;
        f32x4 s[RB][4];
        // (the unit after the next: of this tile, or, places looked up in time, of the next one)
        const auto refill = [&](auto hc) RS_INLINE {
            constexpr int h = decltype(hc)::value, n = h + 2;
            if constexpr (n < 2 * U::PER) {
                fetch(j, n);
            } else {
                if constexpr (n == 2 * U::PER)
                    if (more && ((j + 1) & 63) == 0) look_up(j + 1);
                if (more) fetch(j + 1, n - 2 * U::PER);
            }
        };
        static_for<0, U::PER>([&](auto hc) RS_INLINE {
            constexpr int h = decltype(hc)::value;
            wait_loads(true);
            uint4 kf[8];
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < U::K_READS; ++i)
                    kf[t * U::K_READS + i] = *reinterpret_cast<const uint4*>(mine + (h & 1) * U::BYTES + k_at[i] + U::sub_step(t) * U::K_ROW);
            reads_done();
            refill(hc);
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int kk = 0; kk < KS; ++kk) {
                    bf16x8 kfrag;
                    if constexpr (FP8) {
                        const uint4 w = kf[t * U::K_READS + (kk >> 1)];
                        kfrag = (kk & 1) ? bf16x8_of_codes(w.z, w.w) : bf16x8_of_codes(w.x, w.y);
                    } else {
                        kfrag = as_bf16x8(kf[t * U::K_READS + kk]);
                    }
#pragma unroll
                    for (int b = 0; b < RB; ++b) {
                        f32x4& to = s[b][h * NT + t];
                        to = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kfrag, qf[b][kk], kk == 0 ? f32x4{0.0f, 0.0f, 0.0f, 0.0f} : to, 0, 0, 0);
                    }
                }
        });
        bf16x8 pf[RB][2];
#pragma unroll
        for (int b = 0; b < RB; ++b) {
            if (b > 0 && !two) {   // (no rows: weights of zero)
                pf[b][0] = pf[b][1] = bf16x8{};
                continue;
            }
            if (key0 + 63 > seen_by_all) {
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[b][t][e] = key0 + U::key_of(t, c * 4 + e) <= qpos[b] ? s[b][t][e] : -INFINITY;
            }
            float mx = s[b][0][0];
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) mx = fmaxf(mx, s[b][t][e]);
            mx = of_quarters(mx, larger_of());
            const bool move = (mx - m[b]) * sc > FEW_HEADROOM;   // (at first m is minus infinity)
            if (__builtin_amdgcn_ballot_w64(move)) {
                const float m_new = move ? mx : m[b];
                const float alpha = m[b] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m[b] - m_new) * sc);
                m[b] = m_new;
                l[b] *= alpha;
#pragma unroll
                for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[b][dt][e] *= alpha;
            }
            const float ref = m[b] == -INFINITY ? 0.0f : m[b];
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float p = __builtin_amdgcn_exp2f((s[b][t][e] - ref) * sc);
                    l[b] += p;
                    pf[b][t >> 1][(t & 1) * 4 + e] = f32_to_bf16(p);
                }
        }
        static_for<0, U::PER>([&](auto hc) RS_INLINE {
            constexpr int h = decltype(hc)::value;
            wait_loads(h + 1 < U::PER || more);
            uint4 vf[8];
#pragma unroll
            for (int dt = 0; dt < DTU; ++dt)
#pragma unroll
                for (int i = 0; i < U::V_READS; ++i)
                    vf[dt * U::V_READS + i] = *reinterpret_cast<const uint4*>(mine + ((U::PER + h) & 1) * U::BYTES + v_at[i] + dt * 16 * U::V_ROW);
            reads_done();
            refill(std::integral_constant<int, U::PER + h>{});
#pragma unroll
            for (int dt = 0; dt < DTU; ++dt)
#pragma unroll
                for (int s2 = 0; s2 < 2; ++s2) {
                    bf16x8 vfrag;
                    if constexpr (FP8) vfrag = s2 ? bf16x8_of_codes(vf[dt].z, vf[dt].w) : bf16x8_of_codes(vf[dt].x, vf[dt].y);
                    else vfrag = as_bf16x8(vf[dt * U::V_READS + s2]);
#pragma unroll
                    for (int b = 0; b < RB; ++b) {
                        f32x4& to = acc[b][h * DTU + dt];
                        to = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vfrag, pf[b][s2], to, 0, 0, 0);
                    }
                }
        });
        block = __builtin_amdgcn_readlane(number, (j + 1) & 63);
    }

    constexpr int SUMS = 16 * (D + 4) * 4;   // bytes of a wavefront's sums
    const auto sums_of = [&](int w, int row) RS_INLINE { return reinterpret_cast<float*>(lds + w * SUMS) + row * (D + 4); };
    constexpr int PER = D / 16;   // features of a thread
    const int row = threadIdx.x >> 4, f0 = (threadIdx.x & 15) * PER;
    // ---- the wavefronts of the same rows meet: each brings its sums to the largest reference among them
    static_for<0, RB>([&](auto bc) RS_INLINE {
        constexpr int own_block = decltype(bc)::value;
        if (own_block > 0) {
            if (rows.rows <= 16 * own_block) return;
            __syncthreads();
        }
        const float m_own = m[own_block], l_own = of_quarters(l[own_block], sum_of());
        if (c == 0) {
            m_sh[wave][r] = m_own;
            l_sh[wave][r] = l_own;
        }
        __syncthreads();
        float big = m_own;
        for (int w = set; w < FEW_WAVES; w += sets) big = fmaxf(big, m_sh[w][r]);
        const float weight = m_own == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m_own - big) * sc);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
            f32x4 o = acc[own_block][dt];
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] *= weight;
            *reinterpret_cast<f32x4*>(sums_of(wave, r) + dt * 16 + c * 4) = o;
        }
        __syncthreads();
        for (int sb = 0; sb < sets; ++sb) {
            const int b = sb * RB + own_block;   // block of 16 rows
            if (b * 16 >= rows.rows) break;
            float M = -INFINITY, L = 0.0f, o[PER] = {};
            for (int w = sb; w < FEW_WAVES; w += sets) M = fmaxf(M, m_sh[w][row]);
            for (int w = sb; w < FEW_WAVES; w += sets) {
                L += l_sh[w][row] == 0.0f ? 0.0f : __builtin_amdgcn_exp2f((m_sh[w][row] - M) * sc) * l_sh[w][row];
#pragma unroll
                for (int j = 0; j < PER; ++j) o[j] += sums_of(w, row)[f0 + j];
            }
            bool bad = !(fabsf(L) <= 3.402823466e38f);
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                if constexpr (FP8) o[j] *= rq.v_scale;
                bad |= !(fabsf(o[j]) <= 3.402823466e38f);
            }
            const int i = b * 16 + row;
            const bool live = i < rows.rows;
            const int ic = min(i, rows.rows - 1);
            bf16* const op = a.out + (size_t)(rq.row0 + rows.token(ic)) * a.ld_out + rows.head(ic) * D;
            float* const slot = a.slots + (size_t)(rq.slot0 + (unit * parts + part) * slot_blocks + b) * FewSlot<D>::FLOATS;
            const unsigned long long any = __builtin_amdgcn_ballot_w64(bad && live);
            const bool again = ((any >> (lane & 48)) & 0xffffu) != 0;   // (a row's sixteen threads are neighbours)
            if (!again && parts > 1) {
#pragma unroll
                for (int j = 0; j < PER; j += 4) *reinterpret_cast<f32x4*>(slot + (size_t)row * D + f0 + j) = f32x4{o[j], o[j + 1], o[j + 2], o[j + 3]};
                if (f0 == 0) {
                    slot[(size_t)16 * D + row] = M;
                    slot[(size_t)16 * (D + 1) + row] = L;
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
                for (int k = 0; k < 4; ++k) {   // the wavefront's four rows
                    if (((any >> (16 * k)) & 0xffffu) == 0) continue;
                    const int bi = b * 16 + wave * 4 + k, tok = rows.token(bi), head = rows.head(bi);
                    float em, el, eo[D / 64];
                    exact_row<D, FP8>(a.q + (size_t)(rq.row0 + tok) * a.ld_q + head * D, sc, rq.P + tok, kb0, kb0 + held, tile_at, em, el, eo);
                    bf16* const bp = a.out + (size_t)(rq.row0 + tok) * a.ld_out + head * D;
#pragma unroll
                    for (int j = 0; j < D / 64; ++j) {
                        const float v = eo[j] * (FP8 ? rq.v_scale : 1.0f);
                        if (parts > 1) slot[(size_t)(wave * 4 + k) * D + lane + 64 * j] = v;
                        else bp[lane + 64 * j] = f32_to_bf16(v / el);
                    }
                    if (parts > 1 && lane == 0) {
                        slot[(size_t)16 * D + wave * 4 + k] = em;
                        slot[(size_t)16 * (D + 1) + wave * 4 + k] = el;
                    }
                }
            }
        }
    });
}

template <int D, bool FP8, bool LIST, int RB, class Tab>
__global__ __launch_bounds__(64 * FEW_WAVES, 2) void attend_few_kernel(FewArgs a, Tab tab) {
    __shared__ __attribute__((aligned(16))) char lds[FEW_LDS<D, FP8>];
    __shared__ FewStats m_sh, l_sh;
    const uint32_t* const table = table_of(tab, a.table);
    FewRows<LIST> rows;
    int id = blockIdx.x, req, part, parts, unit, n;   // n: tiles, or blocks of the list
    const int* list = nullptr;
    rows.g = a.g;
    if constexpr (LIST) {
        rows.kvh = id % a.hkv;
        id /= a.hkv;
        parts = a.list_parts;
        part = id % parts;
        rows.tok0 = id / parts;
        req = request_of(table, a.n_req, (uint32_t)rows.tok0);
        unit = rows.tok0 * a.hkv + rows.kvh;
    } else {
        req = request_of(table, a.n_req, blockIdx.x);
    }
    const FewReq rq = reinterpret_cast<const FewReq*>(table + table_reqs_at(a.n_req))[req];
    const uint32_t* const pages = a.pages ? a.pages : table + table_reqs_at(a.n_req) + REQ_WORDS * a.n_req;
    if constexpr (LIST) {
        rows.tok0 -= rq.row0;
        rows.rows = a.g;
        list = a.chosen + (size_t)unit * a.n_blocks;
        n = min(a.n_blocks, (rq.P + rows.tok0) / 64 + 1);   // (the list ends there)
    } else {
        id -= (int)table[req];
        parts = rq.parts;
        rows.kvh = id % a.hkv;
        id /= a.hkv;
        part = id % parts;
        rows.take(id / parts, rq.T * a.g);
        unit = id / parts * a.hkv + rows.kvh;
        n = (rq.P + rows.token(rows.rows - 1)) / 64 + 1;
    }
    attend_rows<D, FP8, LIST, RB>(a, rq, pages, rows, part, parts, unit, n, list, lds, m_sh, l_sh);
}

// Joins the parts of 16 rows:  M = max_p m_p,  out = sum_p 2^(c (m_p - M)) O_p / sum_p 2^(c (m_p - M)) l_p, c the scale log2e.  One workgroup per 16 rows and 32
// features, a quarter of the parts per 64 threads (16 rows x 4 chunks of 8 features).  3 to 5 us, the latency of a launch and of loads that
// follow one another.  (Joining in the kernel before, by the last workgroup to arrive, behind a fence across the chip: 64 single tokens 84 -> 198 us; with slots that are
// themselves stored and loaded past the L2s, without a fence, it has not been measured.)
template <int D, bool LIST, class Tab>
__global__ __launch_bounds__(256) void few_merge_kernel(FewArgs a, Tab tab) {
    __shared__ float m_sh[4][16];
    __shared__ float red[4][64][9];
    const uint32_t* const table = table_of(tab, a.table);
    FewRows<LIST> rows;
    rows.g = a.g;
    int req, parts, unit, b = 0;
    if constexpr (LIST) {
        const int rbn = few_row_blocks(a.g);
        b = blockIdx.x % rbn;
        unit = blockIdx.x / rbn;
        rows.kvh = unit % a.hkv;
        rows.tok0 = unit / a.hkv;
        req = request_of(table, a.n_req, (uint32_t)rows.tok0);
    } else {
        req = request_of(table + table_units_at(a.n_req), a.n_req, blockIdx.x);
        unit = 0;
    }
    const FewReq rq = reinterpret_cast<const FewReq*>(table + table_reqs_at(a.n_req))[req];
    parts = LIST ? a.list_parts : rq.parts;
    if (parts <= 1) return;
    if constexpr (LIST) {
        rows.tok0 -= rq.row0;
        rows.rows = a.g;
    } else {
        int id = (int)(blockIdx.x - table[table_units_at(a.n_req) + req]);   // (four row blocks per KV head and group, if there are)
        const int most = few_row_blocks(min(rq.T * a.g, FEW_GROUP));
        rows.kvh = id % a.hkv;
        id /= a.hkv;
        b = id % most;
        rows.take(id / most, rq.T * a.g);
        unit = id / most * a.hkv + rows.kvh;
    }
    if (b * 16 >= rows.rows) return;
    const int group = threadIdx.x >> 6, row = (threadIdx.x & 63) >> 2, f0 = blockIdx.y * 32 + (threadIdx.x & 3) * 8, i = b * 16 + row;
    const int slot_blocks = few_row_blocks(LIST ? a.g : min(rq.T * a.g, FEW_GROUP));
    const float* const base = a.slots + (size_t)(rq.slot0 + unit * parts * slot_blocks + b) * FewSlot<D>::FLOATS;
    const size_t next = (size_t)slot_blocks * FewSlot<D>::FLOATS;
    const float sc = a.scale_log2e * rq.k_scale;   // (bfloat16 caches: times one)
    // four parts at a time, all their loads in flight together, on to a running reference M
    float M = -INFINITY, L = 0.0f, o[8] = {};
    for (int p0 = group; p0 < parts; p0 += 16) {
        float mp[4], lp[4];
        f32x4 x[4], y[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float* const sp = base + (size_t)min(p0 + 4 * k, parts - 1) * next;
            mp[k] = sp[(size_t)16 * D + row];
            lp[k] = sp[(size_t)16 * (D + 1) + row];
            x[k] = *reinterpret_cast<const f32x4*>(sp + (size_t)row * D + f0);
            y[k] = *reinterpret_cast<const f32x4*>(sp + (size_t)row * D + f0 + 4);
        }
        float big = M;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (p0 + 4 * k < parts) big = fmaxf(big, mp[k]);
        const float alpha = M == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((M - big) * sc);
        M = big;
        if (L != 0.0f) {   // (sums of nothing stay, whatever the reference)
            L *= alpha;
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] *= alpha;
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            // (a part none of whose keys count has a row sum of zero and no reference)
            const float w = p0 + 4 * k >= parts || lp[k] == 0.0f ? 0.0f : __builtin_amdgcn_exp2f((mp[k] - M) * sc);
            if (p0 + 4 * k >= parts) continue;
            L += w * lp[k];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                o[e] += w * x[k][e];
                o[4 + e] += w * y[k][e];
            }
        }
    }
    if ((threadIdx.x & 3) == 0) m_sh[group][row] = M;
    __syncthreads();
    {
        const float big = fmaxf(fmaxf(m_sh[0][row], m_sh[1][row]), fmaxf(m_sh[2][row], m_sh[3][row]));
        const float w = L == 0.0f ? 0.0f : __builtin_amdgcn_exp2f((M - big) * sc);
        L *= w;
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] *= w;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) red[group][threadIdx.x & 63][e] = o[e];
    red[group][threadIdx.x & 63][8] = L;
    __syncthreads();
    if (group == 0 && i < rows.rows) {
        const int t = threadIdx.x;
        const float inv = 1.0f / ((red[0][t][8] + red[1][t][8]) + (red[2][t][8] + red[3][t][8]));
        bf16x8 h;
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] = f32_to_bf16(((red[0][t][e] + red[1][t][e]) + (red[2][t][e] + red[3][t][e])) * inv);
        *reinterpret_cast<bf16x8*>(a.out + (size_t)(rq.row0 + rows.token(i)) * a.ld_out + rows.head(i) * D + f0) = h;
    }
}

// A call's table from the staging buffer to the workspace.
static __global__ __launch_bounds__(256) void copy_table_kernel(const uint4* __restrict__ src, uint4* __restrict__ dst, int n) {
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i < n) dst[i] = src[i];
}
