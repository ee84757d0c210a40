// Attention of a step's new tokens over the prefix that all sequences share and over each sequence's own pages
// (griffin_attention): o = sum_k softmax_k(scale q.k) v_k.
//
// One pass over the keys with the running maximum m and sum l of the softmax: a step forms the scores of a few keys, takes
// m' = max(m, scores), scales o and l by 2^(m - m') and adds the step's weights and weighted values (exponents to base 2, the factor
// log2(e) goes into the scale).  A row is a token and a head; the rows of all heads that share a kv head go together, and in the prefix those of all
// sequences, so that keys and values are read once for 16 to 64 rows.
//
// A wavefront streams keys on its own, global memory -> registers -> matrix cores, no LDS.  Scores are formed transposed, S^T = K Q^T, with
// keys as the rows of the A operand: the result's column, lane & 15, is the query row, so m, l and the factors are a lane's own.  The result's
// rows are keys 4 (lane >> 4) .. + 3 of a tile of 16, and exactly these, as they stand, are the k positions that lane has to hold in the B operand of
// O^T = V^T P^T, if V's A operand takes its keys in the same order.  That operand wants consecutive keys of one feature where memory has
// consecutive features of one key: a lane loads the 8 x 8 block (keys x features) whose transpose is its share of eight A operands (row r of operand e:
// feature 8 r + e) and turns it with 32 byte permutes.
//
// Long key ranges are cut into chunks for as many workgroups as fill the chip; each leaves its rows' o, m and l, and a second kernel joins them.
//
// Bound by bytes while few rows share a key, with the latency of a step's loads on top: a part that one step covers is two launches' latency, 4.5 us of it the join's.
// Measured: 64 continuations of 1024 shared tokens and 1 to 120 of their own, 40 heads of 128, 102 MB, 32 us warm = 3.2 TB/s; 8 sequences behind 30000 shared
// keys of 8 heads of 128, four query heads each, 125 MB, 31 us = 4.0 TB/s; one row of 513 keys of 32 heads 8.3 us and the join.
// The products of 16 rows a key are a twentieth of the matrix cores' rate when keys arrive at a copy's, of 64 rows a quarter: the arrangement is made for loads.
#include <algorithm>

#include "attend.h"

namespace griffin {

// Shapes of a wavefront's step for one type and padded head width DB
template <bool BF16, int DB>
struct AttShape {
    static constexpr int KT = BF16 ? 2 : 1;                // tiles of 16 keys a step
    static constexpr int KS = 16 * KT;                     // keys a step
    static constexpr int E = BF16 ? 8 : 4;                 // features in 16 bytes
    static constexpr int NQ = DB / (4 * E);                // 16-byte pieces of a key that a lane holds (four lanes share a key)
    static constexpr int VD = DB / 16 < E ? DB / 16 : E;   // consecutive features of a value that a lane holds
    static constexpr int NC = DB / (16 * VD);              // ... and how many such runs, 16 VD apart
    static constexpr int NO = NC * VD;                     // tiles of 16 features of the output
    static constexpr int VK = BF16 ? 8 : 4;                // keys of a step whose values a lane holds
    static constexpr int VW = BF16 ? VD / 2 : VD;          // words of such a run
};

// rows of one wavefront: their queries and where they end, and what it has summed
template <bool BF16, int DB, int NT>
struct AttRows {
    using S = AttShape<BF16, DB>;
    att_u32x4 q[NT][S::NQ];
    int32_t end[NT];             // keys from here on are not seen by the lane's row
    float m[NT], l[NT];
    att_f32x4 o[NT][S::NO];
};

// a step's keys and values in registers
template <bool BF16, int DB>
struct AttKeys {
    using S = AttShape<BF16, DB>;
    att_u32x4 k[S::KT][S::NQ];
};
template <bool BF16, int DB>
struct AttVals {
    using S = AttShape<BF16, DB>;
    uint32_t v[S::VK][S::NC][S::VW];
};

template <bool BF16, int DB, int NT>
using AttScores = att_f32x4[NT][AttShape<BF16, DB>::KT];

// A step's tiles of 16 keys: their pages' numbers (looked up a step ahead of their use) and places, and the lane's place in a tile.
template <bool BF16, int DB, bool FULL>
struct AttStage {
    using S = AttShape<BF16, DB>;
    static constexpr int ES = BF16 ? 2 : 4;
    const char *K, *V;                       // of the kv head
    uint32_t at_k, at_v[4];                  // of values: keys 4 (lane >> 4) + j
    int32_t page[S::KT];
    uint64_t base[S::KT];

    __device__ __forceinline__ AttStage(const AttendParams &p, int hk, int lane)
    {
        const uint32_t stride = (uint32_t)p.token_stride * ES;
        K = (const char *)p.K + hk * p.head_stride * ES;
        V = (const char *)p.V + hk * p.head_stride * ES;
        at_k = (lane & 15) * stride + (lane >> 4) * 16;
        // features from dim on end in outputs that are not stored: any of the row's own will do
        const int d = FULL || (lane & 15) * S::VD < p.dim ? (lane & 15) * S::VD : 0;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            at_v[j] = ((lane >> 4) * 4 + j) * stride + d * ES;
    }

    __device__ __forceinline__ void look_up(const AttendParams &p, const AttendItem &it, int32_t key0)
    {
#pragma unroll
        for (int i = 0; i < S::KT; ++i)
            page[i] = att_look_up(p, it, key0 + 16 * i);
    }

    __device__ __forceinline__ void place(const AttendParams &p, const AttendItem &it, int32_t key0)
    {
#pragma unroll
        for (int i = 0; i < S::KT; ++i)
            base[i] = att_place<ES>(p, it, page[i], key0 + 16 * i);
    }

    __device__ __forceinline__ void load_keys(AttKeys<BF16, DB> &f, const AttendParams &p, int lane) const
    {
#pragma unroll
        for (int i = 0; i < S::KT; ++i)
#pragma unroll
            for (int s = 0; s < S::NQ; ++s) {
                // features from dim on are zero here and in the queries: they add nothing, whatever the row's gap holds
                if (FULL || (s * 4 + (lane >> 4)) * S::E < p.dim)
                    f.k[i][s] = *(const att_u32x4 *)(K + base[i] + at_k + s * 64);
                else
                    f.k[i][s] = att_u32x4{0, 0, 0, 0};
            }
    }

    __device__ __forceinline__ void load_vals(AttVals<BF16, DB> &f, const AttendParams &p, int lane) const
    {
#pragma unroll
        for (int j = 0; j < S::VK; ++j)
#pragma unroll
            for (int c = 0; c < S::NC; ++c) {
                const char *at = V + base[j >> 2] + at_v[j & 3];
                if (FULL || c == 0 || c * 16 * S::VD + (lane & 15) * S::VD < p.dim)
                    at += c * 16 * S::VD * ES;
                if (S::VW == 4)
                    *(att_u32x4 *)f.v[j][c] = *(const att_u32x4 *)at;
                else
                    *(uint2 *)f.v[j][c] = *(const uint2 *)at;
            }
    }
};

template <bool BF16, int DB, int NT>
__device__ __forceinline__ void att_scores(AttScores<BF16, DB, NT> &s, const AttKeys<BF16, DB> &f, const AttRows<BF16, DB, NT> &r)
{
    using S = AttShape<BF16, DB>;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < S::KT; ++i)
            s[n][i] = att_f32x4{0, 0, 0, 0};
#pragma unroll
    for (int c = 0; c < S::NQ; ++c)
#pragma unroll
        for (int i = 0; i < S::KT; ++i)
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                if constexpr (BF16)
                    s[n][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(att_bf16x8, f.k[i][c]), __builtin_bit_cast(att_bf16x8, r.q[n][c]),
                                                                      s[n][i], 0, 0, 0);
                else
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        s[n][i] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(f.k[i][c][e]), __uint_as_float(r.q[n][c][e]), s[n][i], 0, 0, 0);
            }
}

// Scores to weights: the rows' maximum and sum carried on, o scaled to the new maximum
template <bool BF16, int DB, int NT>
__device__ __forceinline__ void att_softmax(AttScores<BF16, DB, NT> &s, AttRows<BF16, DB, NT> &r, float scale2)
{
    using S = AttShape<BF16, DB>;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < S::KT; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                top = fmaxf(top, s[n][i][e]);
        const float m = fmaxf(r.m[n], lane_groups_max(top) * scale2);
        const float base = m == -INFINITY ? 0.0f : m;          // nothing seen yet: weights 2^-inf = 0
        const float f = __builtin_amdgcn_exp2f(r.m[n] - base);
        r.m[n] = m;
        float l = 0;
#pragma unroll
        for (int i = 0; i < S::KT; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s[n][i][e] = __builtin_amdgcn_exp2f(s[n][i][e] * scale2 - base);
                l += s[n][i][e];
            }
        r.l[n] = r.l[n] * f + l;
#pragma unroll
        for (int c = 0; c < S::NO; ++c)
            r.o[n][c] *= f;
    }
}

// Keys from r.end on, and those in the hole, out of the scores
template <bool BF16, int DB, int NT>
__device__ __forceinline__ void att_mask(AttScores<BF16, DB, NT> &s, const AttRows<BF16, DB, NT> &r, const AttendItem &it, int32_t key0, int lane)
{
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < AttShape<BF16, DB>::KT; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int32_t key = key0 + 16 * i + (lane >> 4) * 4 + e;
                s[n][i][e] = key < r.end[n] && !it.missing(key) ? s[n][i][e] : -INFINITY;
            }
}

// O^T += V^T P^T
template <bool BF16, int DB, int NT>
__device__ __forceinline__ void att_weigh(const AttScores<BF16, DB, NT> &s, const AttVals<BF16, DB> &f, AttRows<BF16, DB, NT> &r)
{
    using S = AttShape<BF16, DB>;
    if constexpr (BF16) {
        att_u32x4 w[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                w[n][2 * i] = f32x2_to_bf16x2(s[n][i][0], s[n][i][1]);
                w[n][2 * i + 1] = f32x2_to_bf16x2(s[n][i][2], s[n][i][3]);
            }
#pragma unroll
        for (int c = 0; c < S::NC; ++c)
#pragma unroll
            for (int e = 0; e < S::VD; ++e) {
                att_u32x4 a;
#pragma unroll
                for (int h = 0; h < 4; ++h)        // feature e of keys 2h and 2h + 1
                    a[h] = __builtin_amdgcn_perm(f.v[2 * h + 1][c][e / 2], f.v[2 * h][c][e / 2], e & 1 ? 0x07060302 : 0x05040100);
#pragma unroll
                for (int n = 0; n < NT; ++n)
                    r.o[n][c * S::VD + e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(att_bf16x8, a), __builtin_bit_cast(att_bf16x8, w[n]),
                                                                                   r.o[n][c * S::VD + e], 0, 0, 0);
            }
    } else {
#pragma unroll
        for (int c = 0; c < S::NC; ++c)
#pragma unroll
            for (int e = 0; e < S::VD; ++e)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int n = 0; n < NT; ++n)
                        r.o[n][c * S::VD + e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(f.v[i][c][e]), s[n][0][i], r.o[n][c * S::VD + e], 0, 0, 0);
    }
}

// Before a masked step's second product.  Infinite and NaN values of keys that a row does not see must not reach it, as 0 x Inf would.  Values behind the last
// key are made zero, and so are infinite and NaN ones; if there were any of these (`true`), they are added to the rows that do see them at the end
// (att_add_infinite).
template <bool BF16, int DB>
__device__ __forceinline__ bool att_clear_infinite(AttVals<BF16, DB> &f, const AttendItem &it, int32_t key0, int lane)
{
    using S = AttShape<BF16, DB>;
    uint32_t odd = 0;
#pragma unroll
    for (int j = 0; j < S::VK; ++j) {
        const int32_t key = key0 + 16 * (j >> 2) + (lane >> 4) * 4 + (j & 3);
        const uint32_t in = key < it.end && !it.missing(key) ? ~0u : 0;
#pragma unroll
        for (int c = 0; c < S::NC; ++c)
#pragma unroll
            for (int w = 0; w < S::VW; ++w) {
                const uint32_t m = BF16 ? att_finite_mask(f.v[j][c][w]) : ((f.v[j][c][w] & 0x7F800000u) == 0x7F800000u ? 0 : ~0u);
                f.v[j][c][w] &= m & in;
                odd |= ~m & in;
            }
    }
    return __any(odd != 0);
}

// ... of the keys from `key` on of one step
template <bool BF16, int DB, bool FULL, int NT>
__device__ __forceinline__ void att_add_infinite(const AttendParams &p, const AttendItem &it, AttRows<BF16, DB, NT> &r, int32_t key)
{
    using S = AttShape<BF16, DB>;
    const int32_t stop = key + S::KS < it.end ? key + S::KS : it.end;
    for (; key < stop; ++key) {
        const char *at = (const char *)p.V + it.hk * p.head_stride * (BF16 ? 2 : 4) + att_place<BF16 ? 2 : 4>(p, it, att_look_up(p, it, key), key);
#pragma unroll
        for (int c = 0; c < S::NC; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) {                  // elements i of the lane's sums: features (c 16 + (lane >> 4) 4 + i) VD + e
                __builtin_amdgcn_sched_barrier(0);
                const int d = (c * 16 + (threadIdx.x >> 4 & 3) * 4 + i) * S::VD;
#pragma unroll
                for (int e = 0; e < S::VD; ++e) {
                    const float x = FULL || d + e < p.dim ? load_scalar<BF16>(at, d + e) : 0.0f;
                    const bool odd = (__float_as_uint(x) & 0x7F800000u) == 0x7F800000u;
#pragma unroll
                    for (int n = 0; n < NT; ++n)
                        r.o[n][c * S::VD + e][i] += odd && key < r.end[n] && !it.missing(key) ? x : 0.0f;
                }
            }
    }
}

// Where a row's sums of a chunk lie
__device__ __forceinline__ int64_t att_slot(const AttendParams &p, const AttendItem &it, int32_t row)
{
    const int32_t token = p.by_group(row), head = it.hk * p.group + row - token * p.group;
    return ((int64_t)(it.token0 + token) * p.n_heads + head) * (p.chunks_prefix + p.chunks_own) + it.split;
}

// Features d .. d + 7 of a row: the sums themselves for the join, or the output
template <bool BF16, bool FULL>
__device__ __forceinline__ void att_store8(const AttendParams &p, const AttendItem &it, int32_t row, int d, float (&x)[8], float l)
{
    if (!FULL && d >= p.dim)
        return;
    if (p.part) {
        float *at = p.part + att_slot(p, it, row) * p.dim + d;
        *(float4 *)at = make_float4(x[0], x[1], x[2], x[3]);
        *(float4 *)(at + 4) = make_float4(x[4], x[5], x[6], x[7]);
        return;
    }
    const float f = l == 0.0f ? 0.0f : 1.0f / l;           // a row without keys: zeros
#pragma unroll
    for (int j = 0; j < 8; ++j)
        x[j] *= f;
    const int32_t token = p.by_group(row), head = it.hk * p.group + row - token * p.group;
    char *at = (char *)p.out + ((int64_t)(it.token0 + token) * p.ldo + (int64_t)head * p.hso + d) * (BF16 ? 2 : 4);
    if (BF16)
        *(uint4 *)at = make_uint4(f32x2_to_bf16x2(x[0], x[1]), f32x2_to_bf16x2(x[2], x[3]), f32x2_to_bf16x2(x[4], x[5]), f32x2_to_bf16x2(x[6], x[7]));
    else {
        *(float4 *)at = make_float4(x[0], x[1], x[2], x[3]);
        *(float4 *)(at + 16) = make_float4(x[4], x[5], x[6], x[7]);
    }
}

// The item's rows first .. first + 16 NT - 1, by the WAVES wavefronts of a workgroup (in turn, a step each) or by one alone
template <bool BF16, int DB, bool FULL, int NT, int WAVES>
__device__ __forceinline__ void attend_rows(const AttendParams &p, float *lds, const AttendItem &it)
{
    using S = AttShape<BF16, DB>;
    constexpr int ES = BF16 ? 2 : 4;
    const int32_t begin = it.begin, end = it.end, own = it.own, rows = it.rows, first = it.first, hk = it.hk;
    const int lane = threadIdx.x & 63, wave = WAVES == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int32_t key0 = begin + wave * S::KS;
    constexpr int STRIDE = WAVES * S::KS;
    AttStage<BF16, DB, FULL> in(p, hk, lane);
    in.look_up(p, it, key0);
    AttRows<BF16, DB, NT> r;
    int32_t least = end;                                   // keys that all rows see
    if (own >= 0 && own + p.by_group(first) + 1 < end)
        least = own + p.by_group(first) + 1;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        int32_t row = first + 16 * n + (lane & 15);
        row = row < rows ? row : rows - 1;                 // rows behind the last repeat it and are not stored
        const int32_t token = p.by_group(row), head = hk * p.group + row - token * p.group;
        r.end[n] = end;
        if (own >= 0) {
            const int32_t sees = own + token + 1;
            r.end[n] = sees < end ? sees : end;
        }
        const char *at = (const char *)p.q + ((int64_t)(it.token0 + token) * p.ldq + (int64_t)head * p.hsq) * ES + (lane >> 4) * 16;
#pragma unroll
        for (int s = 0; s < S::NQ; ++s) {
            if (FULL || (s * 4 + (lane >> 4)) * S::E < p.dim)
                r.q[n][s] = *(const att_u32x4 *)(at + s * 64);
            else
                r.q[n][s] = att_u32x4{0, 0, 0, 0};
        }
        r.m[n] = -INFINITY;
        r.l[n] = 0;
#pragma unroll
        for (int c = 0; c < S::NO; ++c)
            r.o[n][c] = att_f32x4{0, 0, 0, 0};
    }
    bool odd = false;
    if (key0 < end) {
        AttKeys<BF16, DB> fk;
        AttVals<BF16, DB> fv;
        in.place(p, it, key0);
        in.load_keys(fk, p, lane);
        in.load_vals(fv, p, lane);
        in.look_up(p, it, key0 + STRIDE);
        for (; key0 < end; key0 += STRIDE) {
            // the next step's keys leave as soon as this step's scores have taken the registers' old content, its values after the second product.  Two
            // steps on their way (222 registers instead of 177) are 1 to 6 % slower: most parts are a step or two a wavefront.
            att_f32x4 s[NT][S::KT];
            att_scores<BF16, DB, NT>(s, fk, r);
            __builtin_amdgcn_sched_barrier(0);
            const bool more = key0 + STRIDE < end;
            if (more) {
                in.place(p, it, key0 + STRIDE);
                in.load_keys(fk, p, lane);
                in.look_up(p, it, key0 + 2 * STRIDE);
            }
            __builtin_amdgcn_sched_barrier(0);
            if (key0 + S::KS > least || it.touches_hole(key0, S::KS)) {
                att_mask<BF16, DB, NT>(s, r, it, key0, lane);
                odd |= att_clear_infinite<BF16, DB>(fv, it, key0, lane);
            }
            att_softmax<BF16, DB, NT>(s, r, p.scale2);
            att_weigh<BF16, DB, NT>(s, fv, r);
            __builtin_amdgcn_sched_barrier(0);
            if (more)
                in.load_vals(fv, p, lane);
        }
    }
    if (odd)
        for (key0 = begin + wave * S::KS; key0 < end; key0 += WAVES * S::KS)
            if (key0 + S::KS > least || it.touches_hole(key0, S::KS))
                att_add_infinite<BF16, DB, FULL, NT>(p, it, r, key0);
#pragma unroll
    for (int n = 0; n < NT; ++n)
        r.l[n] = lane_groups_sum(r.l[n]);
    if constexpr (WAVES == 1) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int32_t row = first + 16 * n + (lane & 15);
            if (row >= rows)
                continue;
            if (p.part && lane < 16)
                p.part_ml[att_slot(p, it, row)] = make_float2(r.m[n], r.l[n]);
#pragma unroll
            for (int c = 0; c < S::NC; ++c)
#pragma unroll
                for (int h = 0; h < S::VD / 2; ++h) {      // eight consecutive features of the lane's run of 4 VD
                    float x[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        x[j] = r.o[n][c * S::VD + (h * 8 + j) % S::VD][(h * 8 + j) / S::VD];
                    att_store8<BF16, FULL>(p, it, row, (c * 16 + (lane >> 4) * 4) * S::VD + h * 8, x, r.l[n]);
                }
        }
        return;
    }
    // The wavefronts' sums come together in LDS, up to 128 features of 16 rows at a time; then every thread joins and stores eight features of a row.
    constexpr int W = DB < 128 ? DB : 128, CW = W / (16 * S::VD);          // features, and runs of a lane, at a time
    float *ml = lds + WAVES * 16 * (W + 4);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int here = rows - first - 16 * n < 16 ? rows - first - 16 * n : 16;
        if (here <= 0)
            break;
#pragma unroll
        for (int part = 0; part < S::NC / CW; ++part) {
            if (n > 0 || part > 0)
                __syncthreads();
            if ((lane & 15) < here) {
                float *mine = lds + (wave * 16 + (lane & 15)) * (W + 4);
#pragma unroll
                for (int c = 0; c < CW; ++c)
#pragma unroll
                    for (int h = 0; h < S::VD; ++h) {      // four consecutive features
                        att_f32x4 x;
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            x[j] = r.o[n][(part * CW + c) * S::VD + (h * 4 + j) % S::VD][(h * 4 + j) / S::VD];
                        *(att_f32x4 *)(mine + (c * 16 + (lane >> 4) * 4) * S::VD + h * 4) = x;
                    }
                if (lane < 16) {
                    ml[wave * 32 + lane] = r.m[n];
                    ml[wave * 32 + 16 + lane] = r.l[n];
                }
            }
            __syncthreads();
            for (int item = threadIdx.x; item < here * (W / 8); item += WAVES * 64) {
                const int at = item / (W / 8), d = item % (W / 8) * 8;
                float m = -INFINITY, l = 0, x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
                for (int w = 0; w < WAVES; ++w)
                    m = fmaxf(m, ml[w * 32 + at]);
                const float base = m == -INFINITY ? 0.0f : m;
#pragma unroll
                for (int w = 0; w < WAVES; ++w) {
                    const float f = __builtin_amdgcn_exp2f(ml[w * 32 + at] - base);
                    const float *from = lds + (w * 16 + at) * (W + 4) + d;
                    l += ml[w * 32 + 16 + at] * f;
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        x[j] += from[j] * f;
                }
                const int32_t row = first + 16 * n + at;
                if (p.part && part == 0 && d == 0)
                    p.part_ml[att_slot(p, it, row)] = make_float2(m, l);
                att_store8<BF16, FULL>(p, it, row, part * W + d, x, l);
            }
        }
    }
}

// floats of LDS in which WAVES wavefronts' sums come together
template <int DB, int WAVES>
constexpr int att_lds_floats() { return WAVES * 16 * ((DB < 128 ? DB : 128) + 4) + WAVES * 32; }

// LONE: own items go a wavefront each
template <bool BF16, int DB, bool FULL, int NTP, int NTO, bool LONE>
__global__ __launch_bounds__(ATT_WAVES * 64, DB > 128 || (!BF16 && DB > 64 && NTP > 1) ? 1 : 2) void attend_rows_kernel(AttendParams p)
{
    __shared__ __align__(16) float lds[att_lds_floats<DB, ATT_WAVES>()];
    AttendItem it;
    if ((int32_t)blockIdx.x < p.wgs_prefix) {
        att_prefix_item<16 * NTP>(p, blockIdx.x, it);
        attend_rows<BF16, DB, FULL, NTP, ATT_WAVES>(p, lds, it);
        return;
    }
    int32_t id = blockIdx.x - p.wgs_prefix;
    if (LONE) {
        id = id * ATT_WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        if (id >= p.items_own)
            return;
    }
    if (att_own_item<16 * NTO, false>(p, id, it))
        attend_rows<BF16, DB, FULL, NTO, LONE ? 1 : ATT_WAVES>(p, lds, it);
}

// Parts so short and few that one launch does them: twice as many wavefronts an item instead of chunks, nothing to join
template <bool BF16, int DB, bool FULL>
__global__ __launch_bounds__(ATT_FEW_WAVES * 64) void attend_few_kernel(AttendParams p)
{
    extern __shared__ __align__(16) float few_lds[];
    AttendItem it;
    if (att_own_item<16, false>(p, blockIdx.x, it))
        attend_rows<BF16, DB, FULL, 1, ATT_FEW_WAVES>(p, few_lds, it);
}

// Joins a row's chunks: with M = max m_c, o = sum o_c 2^(m_c - M) / sum l_c 2^(m_c - M).  A row per WPR wavefronts; a wavefront takes
// 64 / (DB / 4) chunks at a time, four features a lane.
template <bool BF16, int DB, int WPR>
__global__ __launch_bounds__(256) void attend_join_kernel(AttendParams p)
{
    constexpr int LANES = DB / 4, PAR = 64 / LANES;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sub = lane / LANES, d = lane % LANES * 4;
    const int64_t row = (int64_t)blockIdx.x * (4 / WPR) + (WPR == 1 ? wave : 0);
    if (WPR == 1 && row >= (int64_t)p.tokens * p.n_heads)
        return;
    const int32_t token = __builtin_amdgcn_readfirstlane(p.by_heads((int32_t)row)), head = __builtin_amdgcn_readfirstlane((int32_t)row - token * p.n_heads);
    const int b = att_sequence(token, p.each, p.seqs.cu, p.seqs.n);
    const int32_t held = p.lens[b] < 0 ? 0 : (p.lens[b] < p.max_len ? p.lens[b] : p.max_len);
    const int32_t seen = held + token - p.seqs.cu[b] + 1 < p.max_len ? held + token - p.seqs.cu[b] + 1 : p.max_len;
    const int chunks = p.chunks_prefix + (seen + p.chunk_own - 1) / p.chunk_own;
    const int64_t slot0 = row * (p.chunks_prefix + p.chunks_own);
    // chunks c, c + WPR PAR, ... with a running maximum of their own, U on their way at a time
    constexpr int U = 8;
    float m = -INFINITY, l = 0;
    att_f32x4 o = {0, 0, 0, 0};
    const int d_in = d < p.dim ? d : 0;
    for (int c = (WPR == 1 ? 0 : wave * PAR) + sub; c < chunks; c += U * WPR * PAR) {
        float2 ml[U];
        att_f32x4 x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int at = c + u * WPR * PAR < chunks ? c + u * WPR * PAR : c;
            ml[u] = p.part_ml[slot0 + at];
            x[u] = *(const att_f32x4 *)(p.part + (slot0 + at) * p.dim + d_in);
        }
        float top = m;
#pragma unroll
        for (int u = 0; u < U; ++u)
            top = fmaxf(top, ml[u].x);
        const float base = top == -INFINITY ? 0.0f : top, f = __builtin_amdgcn_exp2f(m - base);
        m = top;
        l *= f;
        o *= f;
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (c + u * WPR * PAR < chunks) {
                const float g = __builtin_amdgcn_exp2f(ml[u].x - base);
                l += ml[u].y * g;
                o += x[u] * g;
            }
    }
#pragma unroll
    for (int off = LANES; off < 64; off <<= 1) {
        const float m2 = __shfl_xor(m, off), l2 = __shfl_xor(l, off), top = fmaxf(m, m2), base = top == -INFINITY ? 0.0f : top;
        const float f = __builtin_amdgcn_exp2f(m - base), f2 = __builtin_amdgcn_exp2f(m2 - base);
        m = top;
        l = l * f + l2 * f2;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            o[e] = o[e] * f + __shfl_xor(o[e], off) * f2;
    }
    if (WPR > 1) {
        __shared__ __align__(16) float lds[WPR][LANES * 4 + 4];
        if (sub == 0) {
            *(att_f32x4 *)&lds[wave][d] = o;
            if (d == 0) {
                lds[wave][LANES * 4] = m;
                lds[wave][LANES * 4 + 1] = l;
            }
        }
        __syncthreads();
        if (wave != 0)
            return;
        m = -INFINITY;
        l = 0;
        o = att_f32x4{0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < WPR; ++w)
            m = fmaxf(m, lds[w][LANES * 4]);
        const float base = m == -INFINITY ? 0.0f : m;
#pragma unroll
        for (int w = 0; w < WPR; ++w) {
            const float f = __builtin_amdgcn_exp2f(lds[w][LANES * 4] - base);
            l += lds[w][LANES * 4 + 1] * f;
            o += *(const att_f32x4 *)&lds[w][d] * f;
        }
    }
    if (sub != 0 || d >= p.dim)
        return;
    const float f = l == 0.0f ? 0.0f : 1.0f / l;
    const int64_t at = (int64_t)token * p.ldo + (int64_t)head * p.hso + d;
    if (BF16)
        *(uint2 *)((uint16_t *)p.out + at) = make_uint2(f32x2_to_bf16x2(o[0] * f, o[1] * f), f32x2_to_bf16x2(o[2] * f, o[3] * f));
    else
        *(att_f32x4 *)((float *)p.out + at) = o * f;
}

// ------------------------------------------------------------------ host side
struct AttPlan {
    bool tile_prefix, tile_own;         // many rows: attend_tile.hip
    bool lone;                          // own items of a few rows go a wavefront each
    bool ahead, few;                    // own items take the prefix, too; all of it in one launch of attend_few_kernel
    int ntp, nto;                       // else tiles of 16 rows that a wavefront takes
    int32_t rows_prefix, rows_own;      // rows of a workgroup
    int32_t chunk_prefix, chunk_own, chunks_prefix, chunks_own, tiles_prefix, tiles_own;
};

static AttPlan attend_plan(const griffin_kv_cache &C, const griffin_kv_batch &B, const SeqTable &seqs, int32_t n_heads)
{
    AttPlan pl;
    const int32_t tile_keys = att_tile_keys(C.dim);
    const bool bf16 = C.dtype == GRIFFIN_BF16;
    const int widest = C.dim > 128 ? 1 : 2;                // what the registers hold beside a step's keys and values
    const int32_t group = n_heads / C.kv_heads;
    const int64_t rows = (int64_t)seqs.cu[seqs.n] * group;
    int64_t longest = 0;
    for (int b = 0; b < seqs.n; ++b)
        longest = std::max(longest, (int64_t)(seqs.cu[b + 1] - seqs.cu[b]) * group);
    // Own parts of more than 64 rows go through LDS, 256 rows a workgroup.  (16 sequences of 2000 keys, us there / here: 48 rows 38 / 36, 80 rows 42 / 58, 128 rows
    // 46 / 62; one sequence of 64 rows 16.6 / 14.2.)  So does a prefix of more rows than that where there is enough to multiply: its workgroups are fewer and
    // larger, and another launch if own parts do not go there, too.  (8 kv heads of 128, us there / here: 80 rows of 8192 keys 26.7 / 21.7, of 32768 42.7 / 43.0; 192
    // rows of 2048 keys 33 / 21, of 8192 34.6 / 33.2, of 32768 57 / 81; 448 rows of 2048 keys 37 / 27, of 8192 45 / 54.)
    pl.tile_own = bf16 && longest > 64;
    pl.tile_prefix = bf16 && (pl.tile_own || (rows > 64 && (double)rows * B.n_prefix * C.kv_heads * C.dim >= 0x1p31));
    pl.nto = longest <= 32 ? 1 : widest;
    pl.ntp = rows <= 16 ? 1 : widest;
    if (!pl.tile_own && !pl.tile_prefix && pl.nto == widest)        // compiled pairs: (1, 1), (2, 1), (2, 2)
        pl.ntp = widest;
    pl.rows_own = pl.tile_own ? att_tile_rows(C.dim) : 16 * pl.nto;
    pl.rows_prefix = pl.tile_prefix ? att_tile_rows(C.dim) : 16 * pl.ntp;
    int64_t tiles = 0;
    for (int b = 0; b < seqs.n; ++b)
        tiles += ((int64_t)(seqs.cu[b + 1] - seqs.cu[b]) * group + pl.rows_own - 1) / pl.rows_own;
    pl.tiles_own = (int32_t)tiles;
    pl.tiles_prefix = B.n_prefix > 0 ? (int32_t)((rows + pl.rows_prefix - 1) / pl.rows_prefix) : 0;
    // Own parts that fill the chip as they are, a wavefront each, are not cut, unless the longest may keep the others waiting.  (2560 parts of up to 60 keys, a
    // wavefront each / a workgroup each: 11.7 / 12.8 us, caches cold 20.6 / 20.2; 2048 of up to 200: 27 / 28.5, 62 / 60; 1280 of up to 500: 41 / 36, 93 / 87;
    // 768 of up to 500: 29 / 25, 58 / 55; two fp32 prompts of 1500 and 9 tokens, 32 heads of 64: 161 / 113.)
    pl.lone = !pl.tile_own && C.kv_heads * tiles >= 1024 && B.max_len <= 256;
    // As many keys a chunk as leave a workgroup a CU, or two of the smaller ones, which a CU holds at a time.  (More of them, us for 512 / 1024 / 2048: 48 rows of 16384
    // keys 23 / 30 / 32, 32 rows of 30000 31 / 35 / 41; fewer, 256, the same within 3 %.  Tiles, 256 / 512: 192 rows of 32768 keys 71 / 85, a prompt of 2048 63 / 70;
    // heads of 256, 256 / 512: 15.7 / 18.4.)  Own parts that have a launch for themselves behind tiles of the prefix are cut finer: the longest is known here, most are shorter, and
    // nothing else runs beside it (48 of 5 to 700 keys, 512 / 1024 / 2048 workgroups: 75 / 70 / 68 us).  Own parts of many rows are one chunk if they fill the chip.
    const int64_t step = ATT_WAVES * (bf16 ? 32 : 16);
    const int64_t work_prefix = C.kv_heads * (int64_t)pl.tiles_prefix * B.n_prefix, work_own = C.kv_heads * tiles * B.max_len;
    const auto chunk = [&](bool tile, int64_t work) {
        const int64_t quantum = tile ? tile_keys : step, wgs = tile || pl.lone || C.dim > 128 ? 256 : 512;
        return (int32_t)((std::max((work + wgs - 1) / wgs, (int64_t)1) + quantum - 1) / quantum * quantum);
    };
    const bool together = pl.tile_prefix == pl.tile_own && !pl.lone;
    pl.chunk_prefix = chunk(pl.tile_prefix, together ? work_prefix + work_own : work_prefix);
    pl.chunk_own = chunk(pl.tile_own, together ? work_prefix + work_own : pl.lone ? work_own : work_own / 4);
    if (pl.lone || (pl.tile_own && C.kv_heads * tiles > 128))
        pl.chunk_own = (int32_t)((B.max_len + step - 1) / step * step);
    // (Own parts of many rows, whole / cut so that 256 workgroups share them: 3000 tokens of 16 heads, 192 tiles of rows, 95 / 113 us; 1000 of 40 heads on 8, 160
    // tiles, 42 / 61; 2048 of 16 on 8, 128 tiles, 71 / 63.  3400 tokens of 32 on 8 behind a prefix of 300: 79 with the prefix ahead, 141 joined.)
    // Own items take the prefix ahead of their own keys where that costs less than to join two parts: prompts that fill the chip (their rows' sums would go
    // through memory in fp32), and parts so few and short that a step of twice as many wavefronts is cheaper than a second launch (some 5 us), prefix or not.  At
    // two steps it is no longer: 513 keys of 32 heads of 128 take 10.4 us in one launch of 32 workgroups, 10.3 cut into chunks and joined (caches cold: 15.9,
    // 14.4).
    const int64_t all = (int64_t)B.n_prefix + B.max_len, items = C.kv_heads * tiles;
    pl.few = longest <= 32 && !pl.tile_prefix && items <= 512 && all <= ATT_FEW_WAVES / ATT_WAVES * step && C.dim <= 128;
    pl.ahead = B.n_prefix > 0 && (pl.few || (pl.tile_own && items > 128));
    if (pl.ahead)
        pl.tiles_prefix = 0;
    if (pl.ahead || pl.few)
        pl.chunk_own = (int32_t)((all + 15 + step - 1) / step * step);
    pl.chunks_prefix = pl.ahead ? 0 : (B.n_prefix + pl.chunk_prefix - 1) / pl.chunk_prefix;
    pl.chunks_own = pl.ahead ? 1 : (B.max_len + pl.chunk_own - 1) / pl.chunk_own;
    return pl;
}

size_t attend_floats(const griffin_kv_cache &C, const griffin_kv_batch &B, const SeqTable &seqs, int32_t n_heads)
{
    const AttPlan pl = attend_plan(C, B, seqs, n_heads);
    const size_t slots = (size_t)seqs.cu[seqs.n] * n_heads * (pl.chunks_prefix + pl.chunks_own);
    return pl.chunks_prefix + pl.chunks_own < 2 ? 0 : slots * (C.dim + 2);
}

template <bool BF16, int DB, int NTP, int NTO, bool LONE>
static int go_rows(const AttendParams &p, hipStream_t st)
{
    const int32_t wgs = p.wgs_prefix + (LONE ? (p.items_own + ATT_WAVES - 1) / ATT_WAVES : p.items_own);
    if (p.dim == DB)
        hipLaunchKernelGGL((attend_rows_kernel<BF16, DB, true, NTP, NTO, LONE>), dim3(wgs), dim3(ATT_WAVES * 64), 0, st, p);
    else
        hipLaunchKernelGGL((attend_rows_kernel<BF16, DB, false, NTP, NTO, LONE>), dim3(wgs), dim3(ATT_WAVES * 64), 0, st, p);
    return check_launch("attend_rows_kernel");
}

template <bool BF16, int DB, bool FULL>
static int go_few(const AttendParams &p, hipStream_t st)
{
    constexpr int bytes = att_lds_floats<DB, ATT_FEW_WAVES>() * sizeof(float);
    RAISE_LDS_LIMIT((attend_few_kernel<BF16, DB, FULL>), bytes);
    hipLaunchKernelGGL((attend_few_kernel<BF16, DB, FULL>), dim3(p.items_own), dim3(ATT_FEW_WAVES * 64), bytes, st, p);
    return check_launch("attend_few_kernel");
}

template <bool BF16, int DB, bool LONE>
static int launch_rows(const AttendParams &p, int ntp, int nto, hipStream_t st)
{
    if constexpr (DB <= 128) {
        if (nto == 2)
            return go_rows<BF16, DB, 2, 2, LONE>(p, st);
        if (ntp == 2)
            return go_rows<BF16, DB, 2, 1, LONE>(p, st);
    }
    return go_rows<BF16, DB, 1, 1, LONE>(p, st);
}

template <bool BF16, int DB>
static int attend_typed(AttendParams &p, const AttPlan &pl, hipStream_t st)
{
    int rc = GRIFFIN_OK;
    const int32_t wgs_prefix = p.kv_heads * pl.tiles_prefix * pl.chunks_prefix, wgs_own = p.kv_heads * pl.tiles_own * pl.chunks_own;
    const int32_t tiled = (pl.tile_prefix ? wgs_prefix : 0) + (pl.tile_own ? wgs_own : 0), others = wgs_prefix + wgs_own - tiled;
    if constexpr (BF16)
        if (tiled > 0) {
            p.wgs_prefix = pl.tile_prefix ? wgs_prefix : 0;
            rc = launch_attend_tiles(p, tiled, st);
        }
    if (rc == GRIFFIN_OK && others > 0) {
        p.wgs_prefix = pl.tile_prefix ? 0 : wgs_prefix;
        p.items_own = pl.tile_own ? 0 : wgs_own;
        const int ntp = p.wgs_prefix > 0 ? pl.ntp : 1, nto = p.items_own > 0 ? pl.nto : 1;
        if constexpr (DB <= 128)
            if (pl.few)
                return p.dim == DB ? go_few<BF16, DB, true>(p, st) : go_few<BF16, DB, false>(p, st);
        rc = pl.lone ? launch_rows<BF16, DB, true>(p, ntp, nto, st) : launch_rows<BF16, DB, false>(p, ntp, nto, st);
    }
    if (rc != GRIFFIN_OK || !p.part)
        return rc;
    const int64_t rows = (int64_t)p.seqs.cu[p.seqs.n] * p.n_heads;
    // A wavefront has 16 chunks of features on their way at a time (dim 128); of few rows with more, four share a row.  (One / four wavefronts a row, the whole call:
    // 256 rows of 60 chunks 34.4 / 31.4 us, 512 of 33 21.3 / 20.1, 32 of 32 10.3 / 9.9; 512 of 18 13.2 / 14.1, 1280 of 33 28.7 / 31.6.)
    if (rows <= 512 && pl.chunks_prefix + pl.chunks_own > 24)
        hipLaunchKernelGGL((attend_join_kernel<BF16, DB, 4>), dim3((uint32_t)rows), dim3(256), 0, st, p);
    else
        hipLaunchKernelGGL((attend_join_kernel<BF16, DB, 1>), dim3((uint32_t)((rows + 3) / 4)), dim3(256), 0, st, p);
    return check_launch("attend_join_kernel");
}

template <bool BF16>
static int attend_width(AttendParams &p, const AttPlan &pl, hipStream_t st)
{
    if (p.dim <= 64)
        return attend_typed<BF16, 64>(p, pl, st);
    return p.dim <= 128 ? attend_typed<BF16, 128>(p, pl, st) : attend_typed<BF16, 256>(p, pl, st);
}

static AttDiv divide_by(int32_t d) { return {(uint32_t)d, d > 1 ? (uint32_t)(((uint64_t)1 << 32) / d) + 1 : 0}; }

int launch_attend(const AttendJob &job, const SeqTable &seqs, hipStream_t st)
{
    const griffin_kv_cache &C = job.C;
    const griffin_kv_batch &B = job.B;
    const AttPlan pl = attend_plan(C, B, seqs, job.n_heads);
    const int64_t wgs = (int64_t)C.kv_heads * ((int64_t)pl.tiles_prefix * pl.chunks_prefix + (int64_t)pl.tiles_own * pl.chunks_own);
    // a launch holds fewer than 2^32 threads, and quotients are exact while dividend times divisor is below 2^32
    const int64_t rows = (int64_t)seqs.cu[seqs.n] * job.n_heads, limit = (int64_t)1 << 32;
    if (wgs >= 1 << 23 || rows >= 1 << 24 || wgs * C.kv_heads >= limit || wgs * std::max(pl.chunks_prefix, pl.chunks_own) >= limit ||
        rows * job.n_heads >= limit)
        return GRIFFIN_EUNSUPPORTED;
    AttendParams p = {};
    p.q = job.q; p.K = C.K; p.V = C.V; p.out = job.out;
    if (pl.chunks_prefix + pl.chunks_own > 1) {
        p.part = job.ws;
        p.part_ml = (float2 *)(job.ws + (size_t)seqs.cu[seqs.n] * job.n_heads * (pl.chunks_prefix + pl.chunks_own) * C.dim);
    }
    p.lens = B.lens; p.pages = B.pages; p.prefix_pages = B.prefix_pages;
    p.ldq = job.ldq; p.hsq = job.hsq; p.ldo = job.ldo; p.hso = job.hso;
    p.page_stride = C.page_stride; p.head_stride = C.head_stride; p.token_stride = C.token_stride; p.ld_pages = B.ld_pages;
    p.page_stride16 = (uint32_t)(C.page_stride / (C.dtype == GRIFFIN_BF16 ? 8 : 4));
    p.scale2 = job.scale * 1.4426950408889634f;
    p.tokens = seqs.cu[seqs.n];
    p.n_heads = job.n_heads; p.kv_heads = C.kv_heads; p.group = job.n_heads / C.kv_heads; p.dim = C.dim;
    p.page_shift = __builtin_ctz(C.page_size);
    p.last_page = (int32_t)(C.n_pages - 1);
    p.max_len = B.max_len; p.n_prefix = B.n_prefix;
    p.ahead = pl.ahead ? B.n_prefix : 0;
    p.chunk_prefix = pl.chunk_prefix; p.chunk_own = pl.chunk_own;
    p.chunks_prefix = pl.chunks_prefix; p.chunks_own = pl.chunks_own; p.tiles_prefix = pl.tiles_prefix;
    p.seqs = seqs;
    const auto tiles_of = [&](int b) { return (int32_t)(((int64_t)(seqs.cu[b + 1] - seqs.cu[b]) * p.group + pl.rows_own - 1) / pl.rows_own); };
    for (int b = 0; b < seqs.n; ++b)
        p.order[b] = (uint8_t)b;
    if (pl.tile_own)
        std::sort(p.order, p.order + seqs.n, [&](uint8_t a, uint8_t b) { return tiles_of(a) != tiles_of(b) ? tiles_of(a) > tiles_of(b) : a < b; });
    for (int b = 0; b < seqs.n; ++b)
        p.tiles_own[b + 1] = p.tiles_own[b] + tiles_of(p.order[b]);
    int32_t each = seqs.n > 1 ? seqs.cu[1] : 0, tiles_each = seqs.n > 1 ? p.tiles_own[1] : 0;
    for (int b = 1; b < seqs.n; ++b) {
        each = seqs.cu[b + 1] - seqs.cu[b] == seqs.cu[1] ? each : 0;
        tiles_each = p.tiles_own[b + 1] - p.tiles_own[b] == p.tiles_own[1] ? tiles_each : 0;
    }
    p.each = divide_by((int64_t)p.tokens * each < (int64_t)1 << 32 ? each : 0);
    p.tiles_each = divide_by((int64_t)pl.tiles_own * tiles_each < (int64_t)1 << 32 ? tiles_each : 0);
    p.by_heads = divide_by(p.n_heads); p.by_kv_heads = divide_by(p.kv_heads); p.by_group = divide_by(p.group);
    p.by_chunks_prefix = divide_by(pl.chunks_prefix > 0 ? pl.chunks_prefix : 1); p.by_chunks_own = divide_by(pl.chunks_own);
    return C.dtype == GRIFFIN_BF16 ? attend_width<true>(p, pl, st) : attend_width<false>(p, pl, st);
}

}  // namespace griffin
