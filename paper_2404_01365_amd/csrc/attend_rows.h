// A few rows of an attention against a range of keys, by the wavefronts of a workgroup or by one alone (attend.hip, and attend_tile.hip for own parts beside a
// prefix that it takes).
//
// A wavefront streams keys on its own, global memory -> registers -> matrix cores, no LDS.  Scores are formed transposed, S^T = K Q^T, with
// keys as the rows of the A operand: the result's column, lane & 15, is the query row, so m, l and the factors are a lane's own.  The result's
// rows are keys 4 (lane >> 4) .. + 3 of a tile of 16, and exactly these, as they stand, are the k positions that lane has to hold in the B operand of
// O^T = V^T P^T, if V's A operand takes its keys in the same order.  That operand wants consecutive keys of one feature where memory has
// consecutive features of one key: a lane loads the 8 x 8 block (keys x features) whose transpose is its share of eight A operands (row r of operand e:
// feature 8 r + e) and turns it with 32 byte permutes.
#pragma once

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
    float m[NT];
    att_f32x4 l[NT];             // bf16: the row's sum in every element (att_add_weights); fp32: element 0, of the lane's own keys
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
                    s[n][i] = att_mfma(f.k[i][c], r.q[n][c], s[n][i]);
                else
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        s[n][i] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(f.k[i][c][e]), __uint_as_float(r.q[n][c][e]), s[n][i], 0, 0, 0);
            }
}

// Scores to weights: the rows' maximum carried on, sum and o scaled to the new one, the sum carried on in fp32 (bf16: with the second product)
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
        if constexpr (BF16)
            r.l[n] *= f;
        else
            r.l[n][0] = r.l[n][0] * f + l;
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
        for (int n = 0; n < NT; ++n)
            att_add_weights(r.l[n], w[n]);
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
                    r.o[n][c * S::VD + e] = att_mfma(a, w[n], r.o[n][c * S::VD + e]);
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
    if (it.slot0 >= 0)
        return it.slot0 + row - it.first;
    const int32_t token = p.by_group(row), head = it.hk * p.group + row - token * p.group;
    return ((int64_t)(it.token0 + token) * p.n_heads + head) * (p.chunks_prefix + p.chunks_own) + it.split;
}

// Features d .. d + 7 of a row: the sums themselves for the join, or the output
template <bool BF16, bool FULL>
__device__ __forceinline__ void att_store8(const AttendParams &p, const AttendItem &it, int32_t row, int d, float (&x)[8], float l)
{
    if (!FULL && d >= p.dim)
        return;
    if (p.part && !it.alone) {
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

// What the wavefronts have summed comes together and is stored.  S says which features a lane's sums are: element i of o[n][c S::VD + e] is feature
// (c 16 + 4 (lane >> 4) + i) S::VD + e of row 16 n + (lane & 15).
template <bool BF16, class S, int DB, bool FULL, int NT, int WAVES>
__device__ __forceinline__ void att_finish(const AttendParams &p, float *lds, const AttendItem &it, const float (&m_of)[NT], const float (&sum)[NT],
                                           const att_f32x4 (&o)[NT][S::NO])
{
    const int32_t rows = it.rows, first = it.first;
    const int lane = threadIdx.x & 63, wave = WAVES == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if constexpr (WAVES == 1) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int32_t row = first + 16 * n + (lane & 15);
            if (row >= rows)
                continue;
            if (p.part && !it.alone && lane < 16)
                p.part_ml[att_slot(p, it, row)] = make_float2(m_of[n], sum[n]);
#pragma unroll
            for (int c = 0; c < S::NC; ++c)
#pragma unroll
                for (int h = 0; h < S::VD / 2; ++h) {      // eight consecutive features of the lane's run of 4 VD
                    float x[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        x[j] = o[n][c * S::VD + (h * 8 + j) % S::VD][(h * 8 + j) / S::VD];
                    att_store8<BF16, FULL>(p, it, row, (c * 16 + (lane >> 4) * 4) * S::VD + h * 8, x, sum[n]);
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
                            x[j] = o[n][(part * CW + c) * S::VD + (h * 4 + j) % S::VD][(h * 4 + j) / S::VD];
                        *(att_f32x4 *)(mine + (c * 16 + (lane >> 4) * 4) * S::VD + h * 4) = x;
                    }
                if (lane < 16) {
                    ml[wave * 32 + lane] = m_of[n];
                    ml[wave * 32 + 16 + lane] = sum[n];
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
                if (p.part && !it.alone && part == 0 && d == 0)
                    p.part_ml[att_slot(p, it, row)] = make_float2(m, l);
                att_store8<BF16, FULL>(p, it, row, part * W + d, x, l);
            }
        }
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
        r.l[n] = att_f32x4{0, 0, 0, 0};
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
    float sum[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n)
        sum[n] = BF16 ? r.l[n][0] : lane_groups_sum(r.l[n][0]);
    att_finish<BF16, S, DB, FULL, NT, WAVES>(p, lds, it, r.m, sum, r.o);
}

// floats of LDS in which WAVES wavefronts' sums come together
template <int DB, int WAVES>
constexpr int att_lds_floats() { return WAVES * 16 * ((DB < 128 ? DB : 128) + 4) + WAVES * 32; }

}  // namespace griffin
