// A few rows of an attention over a cache in 4 bits, by the wavefronts of a workgroup or by one alone (attend_q4.hip, and attend_q4_tile.hip for own parts beside a
// prefix that it takes).  The mathematics and the arrangement of scores and sums are those of attend_rows.h; a wavefront streams codes from memory into its registers, makes
// fp16 values of them there, and feeds the matrix cores with those.
//
// A code is four bits of a word: masked into the last bits of an fp16 it is an integer, and one multiply-add makes the value of it, two at a time.
// Keys (A operand of S^T = K Q^T): lane & 15 is the key, lane >> 4 says which quarter of its features the lane holds; the order of a word's features in the
// operand is that in which they come out, and queries are laid out alike.  Values (A operand of O^T = V^T P^T): the lane holds the codes of eight keys for VD
// neighbouring features; a byte permute puts two keys' codes of two features side by side, so the turn from rows of features to pairs of keys costs nothing beside
// the unpacking.
//
// Bound by bytes where there are many, and close behind by the unpacking, some 300 instructions for 32 keys of 128 features: 32 sequences of 500 to 8000 keys, 8 heads of 128, four query heads
// each, 175 MB, 45 us, 3.9 TB/s, and 50 where 1.6 GB of caches take turns.  One sequence of 2049 keys, 32 heads, is a launch and a chain of loads, 9.7 us.
#pragma once

#include "attend_rows.h"
#include "q4.h"

namespace griffin {

typedef __attribute__((ext_vector_type(8))) _Float16 q4_f16x8;
typedef __attribute__((ext_vector_type(2))) uint32_t q4_u32x2;

__device__ __forceinline__ att_f32x4 q4_mfma(att_u32x4 a, att_u32x4 b, att_f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(q4_f16x8, a), __builtin_bit_cast(q4_f16x8, b), c, 0, 0, 0);
}

constexpr uint32_t Q4_ONES = 0x3C003C00u;    // two fp16

struct AttendQ4Params : AttendParams {
    Q4Shape s;
    // Own parts that the device cuts, by the lengths that it has: into about 2^deal parts of all heads together, and no more than one more of every tile of rows.
    // deal < 0: they are cut as the plan says.
    int32_t deal;
    int32_t quantum;         // keys a part is a multiple of, but for a sequence's last
    int32_t rows_own;        // rows of a tile
    int64_t slots_own;       // where the own parts' slots begin: [part][kv head][row of the tile]
    int4 *cuts;              // [sequence] first part, parts of a tile of rows, keys of a part, for the join
};

// The sums of the lanes up to each one
__device__ __forceinline__ uint32_t q4_wave_scan(uint32_t v)
{
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, true);             // row_shr 1, 2, 4, 8: within 16 lanes
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);            // row_bcast 15: the first and third sixteen's sums to the second and fourth
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);            // row_bcast 31: the first half's to the second
    return v;
}

// A part of a sequence's own keys: part number `part` of `parts` of tile `tile`'s, `keys` each; the sequence had `held` before the step
struct Q4Cut {
    int32_t b, tile, part, parts, keys, held;
};

// Own part j of a kv head, in the order of sequences, tiles of rows and keys.  With U quanta in all a part is c = ceil(U kv_heads / 2^deal) of them at most; a sequence of q is cut into
// ceil(q / c) parts, as even as quanta allow.  Every wavefront counts for itself, a lane four sequences that are 64 apart.  The first of all notes the cuts for the join.
__device__ __forceinline__ bool q4_deal(const AttendQ4Params &p, int32_t j, bool first_of_all, int lane, Q4Cut &cut)
{
    constexpr int TURNS = GRIFFIN_MAX_SEQS / 64;
    int32_t held[TURNS];
    uint32_t tiles[TURNS], quanta[TURNS], all = 0;
#pragma unroll
    for (int i = 0; i < TURNS; ++i) {
        const int b = i * 64 + lane;
        tiles[i] = quanta[i] = 0;
        held[i] = 0;
        if (i > 0 && p.seqs.n <= i * 64)
            continue;
        if (b < p.seqs.n) {
            const int32_t tokens = p.each.by > 0 ? p.each.by : p.seqs.cu[b + 1] - p.seqs.cu[b], len = p.lens[b];
            held[i] = len < 0 ? 0 : len < p.max_len ? len : p.max_len;
            const int32_t keys = held[i] + tokens < p.max_len ? held[i] + tokens : p.max_len;
            tiles[i] = (uint32_t)(tokens * p.group + p.rows_own - 1) / (uint32_t)p.rows_own;
            quanta[i] = tokens > 0 ? (uint32_t)(keys + p.quantum - 1) / (uint32_t)p.quantum : 0;
        }
        all += tiles[i] * quanta[i];
    }
    const uint64_t whole = (uint64_t)(uint32_t)__builtin_amdgcn_readlane(q4_wave_scan(all), 63) * (uint32_t)p.kv_heads;
    const uint64_t share = (whole + ((uint64_t)1 << p.deal) - 1) >> p.deal;
    const uint32_t most = share < INT32_MAX ? (uint32_t)share : INT32_MAX;
    uint32_t first = 0;                                    // parts of the sequences before these 64
    bool found = false;
#pragma unroll
    for (int i = 0; i < TURNS; ++i) {
        if (i > 0 && p.seqs.n <= i * 64)
            break;
        uint32_t n = (quanta[i] + most - 1) / (most > 0 ? most : 1);
        const uint32_t each = n > 0 ? (quanta[i] + n - 1) / n : 1;
        n = (quanta[i] + each - 1) / each;
        const uint32_t mine = tiles[i] * n, run = q4_wave_scan(mine);
        if (first_of_all && i * 64 + lane < p.seqs.n)
            p.cuts[i * 64 + lane] = make_int4(first + run - mine, n, each * p.quantum, 0);
        const uint64_t behind = __ballot(first + run > (uint32_t)j);
        if (behind && !found) {
            const int l = __builtin_ctzll(behind);
            const uint32_t within = j - first - __builtin_amdgcn_readlane(run - mine, l);
            cut.b = i * 64 + l;
            cut.parts = __builtin_amdgcn_readlane(n, l);
            cut.keys = __builtin_amdgcn_readlane(each, l) * p.quantum;
            cut.held = __builtin_amdgcn_readlane(held[i], l);
            cut.tile = within / (uint32_t)cut.parts;
            cut.part = within - cut.tile * cut.parts;
            found = true;
            if (!first_of_all)
                return true;
        }
        first += __builtin_amdgcn_readlane(run, 63);
    }
    return found;
}

// Own item `id` of [part][kv head], or as the plan has cut them; false: no row needs it
template <int ROWS>
__device__ __forceinline__ bool q4_own_item(const AttendQ4Params &p, int32_t id, AttendItem &it)
{
    if (p.deal < 0)
        return att_own_item<ROWS, false>(p, id, it);
    const int32_t j = p.by_kv_heads(id);
    Q4Cut cut = {0, 0, 0, 1, 0, 0};
    if (!q4_deal(p, j, id == 0 && __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) == 0, threadIdx.x & 63, cut))
        return false;
    it.hk = id - j * p.kv_heads;
    it.pages = p.pages + (int64_t)cut.b * p.ld_pages;
    it.last_entry = (p.max_len - 1) >> p.page_shift;
    it.token0 = p.seqs.cu[cut.b];
    it.rows = (p.seqs.cu[cut.b + 1] - p.seqs.cu[cut.b]) * p.group;
    it.first = cut.tile * ROWS;
    it.own = cut.held;
    const int32_t last = it.first + ROWS < it.rows ? it.first + ROWS - 1 : it.rows - 1;               // the tile's last row sees the most keys
    const int32_t end = it.own + p.by_group(last) + 1 < p.max_len ? it.own + p.by_group(last) + 1 : p.max_len;
    it.hole = it.hole_end = 0;
    it.begin = cut.part * cut.keys;
    it.end = it.begin + cut.keys < end ? it.begin + cut.keys : end;
    it.split = 0;
    it.slot0 = p.slots_own + ((int64_t)j * p.kv_heads + it.hk) * p.rows_own;
    it.alone = cut.parts == 1 && p.n_prefix == 0;
    return it.begin < it.end;                              // else no row reads this part's sums
}

template <bool F32, int DB>
struct Q4Att {
    static constexpr int KS = 32;                          // keys a step, two tiles of 16
    static constexpr int NW = DB / 32;                     // words of codes of a key that a lane holds (four lanes share a key)
    static constexpr int NP = NW > 4 ? 2 : 1;              // ... and (scale, middle) pairs
    static constexpr int VD = DB / 16 < 8 ? DB / 16 : 8;   // consecutive features of a value that a lane holds
    static constexpr int NC = DB / (16 * VD);              // ... and how many such runs, 16 VD apart
    static constexpr int NO = NC * VD;                     // tiles of 16 features of the output
    static constexpr int NF = F32 ? 2 : 1;                 // fp16 that make up a query's feature, and a weight
};

template <bool F32, int DB, int NT>
struct Q4Rows {
    using S = Q4Att<F32, DB>;
    att_u32x4 q[NT][S::NF][S::NW];
    int32_t end[NT];             // keys from here on are not seen by the lane's row
    float scale2[NT];            // of the row's scores: the queries were scaled by a power of two
    float m[NT];
    att_f32x4 l[NT];             // the row's sum in every element
    att_f32x4 o[NT][S::NO];
};

template <bool F32, int DB>
struct Q4Keys {
    using S = Q4Att<F32, DB>;
    uint32_t k[2][S::NW], pair[2][S::NP];
};
template <bool F32, int DB>
struct Q4Vals {
    using S = Q4Att<F32, DB>;
    uint32_t v[8][S::NC], pair[8][S::NC];
};

// A tile of 16 keys: its page's number, and where it lies.  A page's part of a kv head is one buffer, so that a load takes all that is the same for the wavefront from
// scalar registers and 32 bits from the lane: with addresses of 64 bits every load of four bytes has an addition before it.
struct Q4Tile {
    int32_t page;
    __amdgpu_buffer_rsrc_t K, V;
    int32_t codes, pairs;

    __device__ __forceinline__ void look_up(const AttendQ4Params &p, const AttendItem &it, int32_t key) { page = att_look_up(p, it, key); }

    __device__ __forceinline__ void set(const AttendQ4Params &p, const AttendItem &it, int32_t key)
    {
        key -= key < it.hole_end ? 0 : it.hole_end;
        const uint32_t in = key & ((1 << p.page_shift) - 1);
        const uint64_t block = ((uint64_t)att_page(__builtin_amdgcn_readfirstlane(page), p.last_page) * (uint32_t)p.kv_heads + it.hk) * p.s.head_bytes;
        K = __builtin_amdgcn_make_buffer_rsrc((char *)p.K + block, 0, p.s.head_bytes, 0x00020000);
        V = __builtin_amdgcn_make_buffer_rsrc((char *)p.V + block, 0, p.s.head_bytes, 0x00020000);
        codes = in * p.s.row_bytes;
        pairs = p.s.pairs_at + in * p.s.groups * 4;
    }
};

// the lane's place in a tile
template <bool F32, int DB>
struct Q4Stage {
    using S = Q4Att<F32, DB>;
    uint32_t at_k, at_kp[S::NP], at_v[4][S::NC], at_vp[4][S::NC];       // of values: keys 4 (lane >> 4) + j
    __device__ __forceinline__ Q4Stage(const AttendQ4Params &p, int lane)
    {
        // features from dim on meet queries that are zero, or end in outputs that are not stored: some of the row's own will do
        const int f = (lane >> 4) * S::NW * 8 < p.dim ? (lane >> 4) * S::NW * 8 : 0;
        at_k = (lane & 15) * p.s.row_bytes + f / 2;
#pragma unroll
        for (int j = 0; j < S::NP; ++j) {
            const uint32_t g = (uint32_t)(f + 32 * j) >> p.s.group_shift;
            at_kp[j] = ((lane & 15) * p.s.groups + (g < p.s.groups ? g : p.s.groups - 1)) * 4;
        }
#pragma unroll
        for (int c = 0; c < S::NC; ++c) {
            const int d = (c * 16 + (lane & 15)) * S::VD < p.dim ? (c * 16 + (lane & 15)) * S::VD : 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                at_v[j][c] = ((lane >> 4) * 4 + j) * p.s.row_bytes + d / 2;
                at_vp[j][c] = (((lane >> 4) * 4 + j) * p.s.groups + (d >> p.s.group_shift)) * 4;
            }
        }
    }

    __device__ __forceinline__ void load_keys(Q4Keys<F32, DB> &f, const Q4Tile (&of)[2]) const
    {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if constexpr (S::NW == 2)
                *(q4_u32x2 *)f.k[i] = __builtin_amdgcn_raw_buffer_load_b64(of[i].K, at_k, of[i].codes, 0);
            else
#pragma unroll
                for (int w = 0; w < S::NW; w += 4)
                    *(att_u32x4 *)(f.k[i] + w) = __builtin_amdgcn_raw_buffer_load_b128(of[i].K, at_k + w * 4, of[i].codes, 0);
#pragma unroll
            for (int j = 0; j < S::NP; ++j)
                f.pair[i][j] = __builtin_amdgcn_raw_buffer_load_b32(of[i].K, at_kp[j], of[i].pairs, 0);
        }
    }

    __device__ __forceinline__ void load_vals(Q4Vals<F32, DB> &f, const Q4Tile (&of)[2]) const
    {
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int c = 0; c < S::NC; ++c) {
                if constexpr (S::VD == 4)
                    f.v[j][c] = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(of[j >> 2].V, at_v[j & 3][c], of[j >> 2].codes, 0);
                else
                    f.v[j][c] = __builtin_amdgcn_raw_buffer_load_b32(of[j >> 2].V, at_v[j & 3][c], of[j >> 2].codes, 0);
                f.pair[j][c] = __builtin_amdgcn_raw_buffer_load_b32(of[j >> 2].V, at_vp[j & 3][c], of[j >> 2].pairs, 0);
            }
    }
};

template <bool F32, int DB, int NT>
using Q4Scores = att_f32x4[NT][2];

__device__ __forceinline__ uint32_t q4_word(q4_pair v) { return __builtin_bit_cast(uint32_t, v); }

template <bool F32, int DB, int NT>
__device__ __forceinline__ void q4_scores(Q4Scores<F32, DB, NT> &s, const Q4Keys<F32, DB> &f, const Q4Rows<F32, DB, NT> &r)
{
    using S = Q4Att<F32, DB>;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int w = 0; w < S::NW; ++w) {
            const q4_pair scale = q4_scales(f.pair[i][w / 4]), middle = q4_middles(f.pair[i][w / 4]);
            att_u32x4 a;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                a[j] = q4_word(q4_value_pair(f.k[i][w] >> 4 * j, scale, middle));
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int h = 0; h < S::NF; ++h)
                    s[n][i] = q4_mfma(a, r.q[n][h][w], w == 0 && h == 0 ? att_f32x4{0, 0, 0, 0} : s[n][i]);
        }
}

// Keys from r.end on, and those in the hole, out of the scores
template <bool F32, int DB, int NT>
__device__ __forceinline__ void q4_mask(Q4Scores<F32, DB, NT> &s, const Q4Rows<F32, DB, NT> &r, const AttendItem &it, int32_t key0, int lane)
{
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int32_t key = key0 + 16 * i + (lane >> 4) * 4 + e;
                s[n][i][e] = key < r.end[n] && !it.missing(key) ? s[n][i][e] : -INFINITY;
            }
}

// Scores to weights, cut to fp16 (fp32: and what that leaves rounded to fp16 in turn): the rows' reference carried on, moved only when scores outgrow it by more than 8 (base 2), so
// that weights are up to 2^8 times its.  Sums are of the weights as they are multiplied, by a product with ones: what cutting takes off all of them cancels.  What it takes off fp16 below its normal
// numbers is another share of each, up to all: of many keys of little weight a pair that was cut twice would lose up to twice the rounding's bound, and all of them the same way.
template <bool F32, int DB, int NT>
__device__ __forceinline__ void q4_softmax(Q4Scores<F32, DB, NT> &s, att_u32x4 (&w)[NT][Q4Att<F32, DB>::NF], Q4Rows<F32, DB, NT> &r)
{
    using S = Q4Att<F32, DB>;
    float top[NT];
    bool grown = false;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        top[n] = -INFINITY;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                top[n] = fmaxf(top[n], s[n][i][e]);
        top[n] *= r.scale2[n];
        grown |= top[n] > r.m[n] + 8.0f;
    }
    if (__any(grown))
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const float m = fmaxf(r.m[n], lane_groups_max(top[n]));
            const float f = m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(r.m[n] - m);        // nothing seen yet: nothing to scale
            r.m[n] = m;
            r.l[n] *= f;
#pragma unroll
            for (int e = 0; e < S::NO; ++e)
                r.o[n][e] *= f;
        }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        // 2^7 times the weights, up to 2^15: fp16 keeps their bits down to 2^-21 of the reference's, and 2^-31 of it below (of a pair, 2^-11, and 2^-32 below).  The quotient does not see it.
        const float base = r.m[n] == -INFINITY ? -7.0f : r.m[n] - 7.0f;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
                x[e] = __builtin_amdgcn_exp2f(s[n][i][e] * r.scale2[n] - base);
#pragma unroll
            for (int e = 0; e < 4; e += 2) {
                const q4_pair v = __builtin_bit_cast(q4_pair, __builtin_amdgcn_cvt_pkrtz(x[e], x[e + 1]));
                w[n][0][2 * i + e / 2] = q4_word(v);
                if constexpr (F32) {
                    const q4_pair rest = {(_Float16)(x[e] - (float)v[0]), (_Float16)(x[e + 1] - (float)v[1])};
                    w[n][1][2 * i + e / 2] = q4_word(rest);
                }
            }
        }
#pragma unroll
        for (int h = 0; h < S::NF; ++h)
            r.l[n] = q4_mfma(att_u32x4{Q4_ONES, Q4_ONES, Q4_ONES, Q4_ONES}, w[n][h], r.l[n]);
    }
}

// O^T += V^T P^T
template <bool F32, int DB, int NT>
__device__ __forceinline__ void q4_weigh(const att_u32x4 (&w)[NT][Q4Att<F32, DB>::NF], const Q4Vals<F32, DB> &f, Q4Rows<F32, DB, NT> &r)
{
    using S = Q4Att<F32, DB>;
#pragma unroll
    for (int c = 0; c < S::NC; ++c) {
        q4_pair scale[4], middle[4];                       // of keys 2h and 2h + 1
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            scale[h] = __builtin_bit_cast(q4_pair, __builtin_amdgcn_perm(f.pair[2 * h + 1][c], f.pair[2 * h][c], 0x05040100));
            middle[h] = __builtin_bit_cast(q4_pair, __builtin_amdgcn_perm(f.pair[2 * h + 1][c], f.pair[2 * h][c], 0x07060302));
        }
#pragma unroll
        for (int e = 0; e < S::VD; e += 2) {               // features e and e + 1: a byte
            att_u32x4 a[2];
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                const uint32_t x = __builtin_amdgcn_perm(f.v[2 * h + 1][c], f.v[2 * h][c], 0x0C000C00u | (4 + e / 2) << 16 | e / 2);
                a[0][h] = q4_word(q4_value_pair(x, scale[h], middle[h]));
                a[1][h] = q4_word(q4_value_pair(x >> 4, scale[h], middle[h]));
            }
#pragma unroll
            for (int g = 0; g < 2; ++g)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int h = 0; h < S::NF; ++h)
                        r.o[n][c * S::VD + e + g] = q4_mfma(a[g], w[n][h], r.o[n][c * S::VD + e + g]);
        }
    }
}

// whether either of a (scale, middle) word is infinite or NaN
__device__ __forceinline__ bool q4_odd(uint32_t pair) { return (pair & 0x7C00u) == 0x7C00u || (pair & 0x7C000000u) == 0x7C000000u; }

// Before a masked step's second product: what stands behind the last key, or in the hole, is any memory's content and becomes zero, and so do groups of NaN,
// which must not reach the rows that do not see them, as 0 x NaN would; true if there were any of these: they are added at the end to those that do.
template <bool F32, int DB>
__device__ __forceinline__ bool q4_clear(Q4Vals<F32, DB> &f, const AttendItem &it, int32_t key0, int lane)
{
    using S = Q4Att<F32, DB>;
    bool odd = false;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int32_t key = key0 + 16 * (j >> 2) + (lane >> 4) * 4 + (j & 3);
        const bool in = key < it.end && !it.missing(key);
#pragma unroll
        for (int c = 0; c < S::NC; ++c) {
            const bool bad = q4_odd(f.pair[j][c]);
            odd |= in && bad;
            f.pair[j][c] = in && !bad ? f.pair[j][c] : 0;
        }
    }
    return __any(odd);
}

// where a key's (scale, middle) words lie in a pool
__device__ __forceinline__ uint64_t q4_pairs_of(const AttendQ4Params &p, const AttendItem &it, int32_t key)
{
    const uint32_t page = att_page(__builtin_amdgcn_readfirstlane(att_look_up(p, it, key)), p.last_page);
    const uint32_t in = (key - (key < it.hole_end ? 0 : it.hole_end)) & ((1 << p.page_shift) - 1);
    return ((uint64_t)page * (uint32_t)p.kv_heads + it.hk) * p.s.head_bytes + p.s.pairs_at + in * p.s.groups * 4;
}

// ... of the keys from `key` on of one step
template <bool F32, int DB, int NT>
__device__ __forceinline__ void q4_add_odd(const AttendQ4Params &p, const AttendItem &it, Q4Rows<F32, DB, NT> &r, int32_t key)
{
    using S = Q4Att<F32, DB>;
    const int32_t stop = key + S::KS < it.end ? key + S::KS : it.end;
    for (; key < stop; ++key) {
        const char *at = (const char *)p.V + q4_pairs_of(p, it, key);
#pragma unroll
        for (int c = 0; c < S::NC; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) {                  // elements i of the lane's sums: features (c 16 + (lane >> 4) 4 + i) VD + e
                const int d = (c * 16 + (threadIdx.x >> 4 & 3) * 4 + i) * S::VD;
                const bool odd = d < p.dim && q4_odd(*(const uint32_t *)(at + (d < p.dim ? d >> p.s.group_shift : 0) * 4));
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < S::VD; ++e)
                        r.o[n][c * S::VD + e][i] = odd && key < r.end[n] && !it.missing(key) ? __builtin_nanf("") : r.o[n][c * S::VD + e][i];
            }
    }
}

// A row's queries in the order of the codes' pairs, scaled so that the largest lies in [128, 256); returns what its scores are to be multiplied by: a normal number, as
// scores that are masked are -Inf, and -Inf x 0 would be NaN.  Scores are below 2^31 before that, so a factor of 2^-126 or less leaves nothing that fp32 weights could tell from zero.
template <bool F32, int NW>
__device__ __forceinline__ float q4_load_row(const AttendQ4Params &p, att_u32x4 (&q)[F32 ? 2 : 1][NW], int64_t at, int lane)
{
    float x[NW][8], top = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        const int d = ((lane >> 4) * NW + w) * 8;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            x[w][j] = 0;
        if (d < p.dim) {
            if (F32) {
                *(float4 *)x[w] = *(const float4 *)((const float *)p.q + at + d);
                *(float4 *)(x[w] + 4) = *(const float4 *)((const float *)p.q + at + d + 4);
            } else {
                const uint4 b = *(const uint4 *)((const uint16_t *)p.q + at + d);
                x[w][0] = bf16_lo(b.x); x[w][1] = bf16_hi(b.x); x[w][2] = bf16_lo(b.y); x[w][3] = bf16_hi(b.y);
                x[w][4] = bf16_lo(b.z); x[w][5] = bf16_hi(b.z); x[w][6] = bf16_lo(b.w); x[w][7] = bf16_hi(b.w);
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
            top = fmaxf(top, fabsf(x[w][j]));
    }
    const int up = 8 - __builtin_amdgcn_frexp_expf(lane_groups_max(top));      // infinite: frexp gives 0, and the queries stay infinite
#pragma unroll
    for (int w = 0; w < NW; ++w)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float a = ldexpf(x[w][j], up), b = ldexpf(x[w][j + 4], up);
            const q4_pair v = {(_Float16)a, (_Float16)b};
            q[0][w][j] = q4_word(v);
            if constexpr (F32) {
                const q4_pair rest = {(_Float16)(a - (float)v[0]), (_Float16)(b - (float)v[1])};
                q[1][w][j] = q4_word(rest);
            }
        }
    return fmaxf(ldexpf(p.scale2, -up), 0x1p-126f);
}

// The item's rows first .. first + 16 NT - 1, by the WAVES wavefronts of a workgroup (in turn, a step each) or by one alone
template <bool F32, int DB, int NT, int WAVES>
__device__ __forceinline__ void attend_q4(const AttendQ4Params &p, float *lds, const AttendItem &it)
{
    using S = Q4Att<F32, DB>;
    const int32_t begin = it.begin, end = it.end, own = it.own, rows = it.rows, first = it.first;
    const int lane = threadIdx.x & 63, wave = WAVES == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int32_t key0 = begin + wave * S::KS;
    constexpr int STRIDE = WAVES * S::KS;
    const Q4Stage<F32, DB> in(p, lane);
    Q4Tile at[2][2];
    const auto look_up = [&](Q4Tile (&of)[2], int32_t key) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            of[i].look_up(p, it, key + 16 * i);
    };
    const auto set = [&](Q4Tile (&of)[2], int32_t key) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            of[i].set(p, it, key + 16 * i);
    };
    look_up(at[0], key0);
    look_up(at[1], key0 + STRIDE);
    Q4Rows<F32, DB, NT> r;
    int32_t least = end;                                   // keys that all rows see
    if (own >= 0 && own + p.by_group(first) + 1 < end)
        least = own + p.by_group(first) + 1;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        int32_t row = first + 16 * n + (lane & 15);
        row = row < rows ? row : rows - 1;                 // rows behind the last repeat it and are not stored
        const int32_t token = p.by_group(row), head = it.hk * p.group + row - token * p.group;
        r.end[n] = end;
        if (own >= 0) {
            const int32_t sees = own + token + 1;
            r.end[n] = sees < end ? sees : end;
        }
        r.scale2[n] = q4_load_row<F32, S::NW>(p, r.q[n], (int64_t)(it.token0 + token) * p.ldq + (int64_t)head * p.hsq, lane);
        r.m[n] = -INFINITY;
        r.l[n] = att_f32x4{0, 0, 0, 0};
#pragma unroll
        for (int c = 0; c < S::NO; ++c)
            r.o[n][c] = att_f32x4{0, 0, 0, 0};
    }
    bool odd = false;
    if (key0 < end) {
        // Two steps are on their way while one is computed: step i's registers take step i + 2 as soon as they have been read, and i + 4's pages are looked up.  Of heads wider than
        // 128 values are one step ahead: with two there would be registers for one wavefront a SIMD.
        constexpr int VALS = DB > 128 ? 1 : 2;
        Q4Keys<F32, DB> fk[2];
        Q4Vals<F32, DB> fv[VALS];
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (key0 + i * STRIDE < end) {
                set(at[i], key0 + i * STRIDE);
                in.load_keys(fk[i], at[i]);
                if (i < VALS)
                    in.load_vals(fv[i], at[i]);
                look_up(at[i], key0 + (i + 2) * STRIDE);
            }
        while (true) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                att_f32x4 s[NT][2];
                att_u32x4 w[NT][S::NF];
                q4_scores<F32, DB, NT>(s, fk[i], r);
                __builtin_amdgcn_sched_barrier(0);
                const bool more = key0 + 2 * STRIDE < end;
                if (more) {
                    set(at[i], key0 + 2 * STRIDE);
                    in.load_keys(fk[i], at[i]);
                    look_up(at[i], key0 + 4 * STRIDE);
                }
                __builtin_amdgcn_sched_barrier(0);
                if (key0 + S::KS > least || it.touches_hole(key0, S::KS)) {
                    q4_mask<F32, DB, NT>(s, r, it, key0, lane);
                    odd |= q4_clear<F32, DB>(fv[i % VALS], it, key0, lane);
                }
                q4_softmax<F32, DB, NT>(s, w, r);
                q4_weigh<F32, DB, NT>(w, fv[i % VALS], r);
                __builtin_amdgcn_sched_barrier(0);
                if (VALS == 2 ? more : key0 + STRIDE < end)
                    in.load_vals(fv[i % VALS], at[VALS == 2 ? i : i ^ 1]);
                key0 += STRIDE;
                if (key0 >= end)
                    goto done;
            }
        }
    done:;
    }
    if (odd)
        for (key0 = begin + wave * S::KS; key0 < end; key0 += WAVES * S::KS)
            if (key0 + S::KS > least || it.touches_hole(key0, S::KS))
                q4_add_odd<F32, DB, NT>(p, it, r, key0);
    float sum[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n)
        sum[n] = r.l[n][0];
    att_finish<!F32, S, DB, false, NT, WAVES>(p, lds, it, r.m, sum, r.o);
}

constexpr int Q4_TILE_WAVES = 4;         // of a workgroup of attend_q4_tile.hip
constexpr int q4_tile_rows(int32_t dim) { return 16 * Q4_TILE_WAVES * (dim > 128 ? 1 : 2); }
// launches the `wgs` workgroups of p on tiles of q4_tile_rows(dim) rows, and behind them p.items_own own items of 16 rows, a workgroup each or, `each`, a
// wavefront each (dim <= 128); bf16 outside the cache only
int launch_attend_q4_tiles(const AttendQ4Params &p, int32_t wgs, bool each, hipStream_t st);

}  // namespace griffin
