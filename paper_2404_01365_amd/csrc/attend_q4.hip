// Attention over a cache in 4 bits (griffin_attention_q4).  The mathematics and the arrangement of scores and sums are those of attend_rows.h; a wavefront streams codes
// from memory into its registers, makes fp16 values of them there, and feeds the matrix cores with those.
//
// A code is four bits of a word: masked into the last bits of an fp16 it is an integer, and one multiply-add makes the value of it, two at a time.
// Keys (A operand of S^T = K Q^T): lane & 15 is the key, lane >> 4 says which quarter of its features the lane holds; the order of a word's features in the
// operand is that in which they come out, and queries are laid out alike.  Values (A operand of O^T = V^T P^T): the lane holds the codes of eight keys for VD
// neighbouring features; a byte permute puts two keys' codes of two features side by side, so the turn from rows of features to pairs of keys costs nothing beside
// the unpacking.
#include <algorithm>

#include "attend_rows.h"
#include "q4.h"

namespace griffin {

typedef __attribute__((ext_vector_type(8))) _Float16 q4_f16x8;

__device__ __forceinline__ att_f32x4 q4_mfma(att_u32x4 a, att_u32x4 b, att_f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(q4_f16x8, a), __builtin_bit_cast(q4_f16x8, b), c, 0, 0, 0);
}

struct AttendQ4Params : AttendParams {
    Q4Shape s;
};

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

// A step's two tiles of 16 keys: their pages' numbers (looked up a step ahead of their use) and places, and the lane's place in a tile.
template <bool F32, int DB>
struct Q4Stage {
    using S = Q4Att<F32, DB>;
    const char *K, *V;                       // of the kv head
    uint32_t at_k, at_kp[S::NP], at_v[4][S::NC], at_vp[4][S::NC];       // of values: keys 4 (lane >> 4) + j
    int32_t page[2];
    uint64_t codes[2], pairs[2];

    __device__ __forceinline__ Q4Stage(const AttendQ4Params &p, int hk, int lane)
    {
        K = (const char *)p.K + (uint64_t)hk * p.s.head_bytes;
        V = (const char *)p.V + (uint64_t)hk * p.s.head_bytes;
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

    __device__ __forceinline__ void look_up(const AttendQ4Params &p, const AttendItem &it, int32_t key0)
    {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            page[i] = att_look_up(p, it, key0 + 16 * i);
    }

    __device__ __forceinline__ void place(const AttendQ4Params &p, const AttendItem &it, int32_t key0)
    {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            int32_t key = key0 + 16 * i;
            key -= key < it.hole_end ? 0 : it.hole_end;
            const uint32_t in = key & ((1 << p.page_shift) - 1);
            const uint64_t block = (uint64_t)att_page(__builtin_amdgcn_readfirstlane(page[i]), p.last_page) * (uint32_t)p.kv_heads * p.s.head_bytes;
            codes[i] = block + in * p.s.row_bytes;
            pairs[i] = block + p.s.pairs_at + in * p.s.groups * 4;
        }
    }

    __device__ __forceinline__ void load_keys(Q4Keys<F32, DB> &f) const
    {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const char *at = K + codes[i] + at_k;
            if constexpr (S::NW == 2)
                *(uint2 *)f.k[i] = *(const uint2 *)at;
            else
#pragma unroll
                for (int w = 0; w < S::NW; w += 4)
                    *(att_u32x4 *)(f.k[i] + w) = *(const att_u32x4 *)(at + w * 4);
#pragma unroll
            for (int j = 0; j < S::NP; ++j)
                f.pair[i][j] = *(const uint32_t *)(K + pairs[i] + at_kp[j]);
        }
    }

    __device__ __forceinline__ void load_vals(Q4Vals<F32, DB> &f) const
    {
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int c = 0; c < S::NC; ++c) {
                const char *at = V + codes[j >> 2] + at_v[j & 3][c];
                f.v[j][c] = S::VD == 4 ? *(const uint16_t *)at : *(const uint32_t *)at;
                f.pair[j][c] = *(const uint32_t *)(V + pairs[j >> 2] + at_vp[j & 3][c]);
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

// Scores to weights, cut to fp16 (fp32: and what that leaves, once more): the rows' reference carried on, moved only when scores outgrow it by more than 8 (base 2), so
// that weights are up to 2^8 times its.  Sums are of the weights as they are multiplied, by a product with ones: what cutting takes off all of them cancels.
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
        // 2^7 times the weights, up to 2^15: fp16 keeps their bits down to 2^-21 of the reference's, and 2^-31 of it below.  The quotient does not see it.
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
                if constexpr (F32)
                    w[n][1][2 * i + e / 2] = q4_word(__builtin_bit_cast(q4_pair, __builtin_amdgcn_cvt_pkrtz(x[e] - (float)v[0], x[e + 1] - (float)v[1])));
            }
        }
        constexpr uint32_t ONES = 0x3C003C00u;
#pragma unroll
        for (int h = 0; h < S::NF; ++h)
            r.l[n] = q4_mfma(att_u32x4{ONES, ONES, ONES, ONES}, w[n][h], r.l[n]);
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

// ... of the keys from `key` on of one step
template <bool F32, int DB, int NT>
__device__ __forceinline__ void q4_add_odd(const AttendQ4Params &p, const AttendItem &it, Q4Rows<F32, DB, NT> &r, int32_t key)
{
    using S = Q4Att<F32, DB>;
    const int32_t stop = key + S::KS < it.end ? key + S::KS : it.end;
    for (; key < stop; ++key) {
        const int32_t from = key - (key < it.hole_end ? 0 : it.hole_end);
        const uint32_t page = att_page(__builtin_amdgcn_readfirstlane(att_look_up(p, it, key)), p.last_page), in = from & ((1 << p.page_shift) - 1);
        const char *at = (const char *)p.V + ((uint64_t)page * (uint32_t)p.kv_heads + it.hk) * p.s.head_bytes + p.s.pairs_at + in * p.s.groups * 4;
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

// A row's queries in the order of the codes' pairs, scaled so that the largest lies in [128, 256)
template <bool F32, int DB, int NT>
__device__ __forceinline__ void q4_load_row(const AttendQ4Params &p, Q4Rows<F32, DB, NT> &r, int n, int64_t at, int lane)
{
    using S = Q4Att<F32, DB>;
    float x[S::NW][8], top = 0;
#pragma unroll
    for (int w = 0; w < S::NW; ++w) {
        const int d = ((lane >> 4) * S::NW + w) * 8;
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
    r.scale2[n] = ldexpf(p.scale2, -up);
#pragma unroll
    for (int w = 0; w < S::NW; ++w)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float a = ldexpf(x[w][j], up), b = ldexpf(x[w][j + 4], up);
            const q4_pair v = {(_Float16)a, (_Float16)b};
            r.q[n][0][w][j] = q4_word(v);
            if constexpr (F32) {
                const q4_pair rest = {(_Float16)(a - (float)v[0]), (_Float16)(b - (float)v[1])};
                r.q[n][1][w][j] = q4_word(rest);
            }
        }
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
    Q4Stage<F32, DB> in(p, it.hk, lane);
    in.look_up(p, it, key0);
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
        q4_load_row<F32, DB, NT>(p, r, n, (int64_t)(it.token0 + token) * p.ldq + (int64_t)head * p.hsq, lane);
        r.m[n] = -INFINITY;
        r.l[n] = att_f32x4{0, 0, 0, 0};
#pragma unroll
        for (int c = 0; c < S::NO; ++c)
            r.o[n][c] = att_f32x4{0, 0, 0, 0};
    }
    bool odd = false;
    if (key0 < end) {
        Q4Keys<F32, DB> fk;
        Q4Vals<F32, DB> fv;
        in.place(p, it, key0);
        in.load_keys(fk);
        in.load_vals(fv);
        in.look_up(p, it, key0 + STRIDE);
        for (; key0 < end; key0 += STRIDE) {
            att_f32x4 s[NT][2];
            att_u32x4 w[NT][S::NF];
            q4_scores<F32, DB, NT>(s, fk, r);
            __builtin_amdgcn_sched_barrier(0);
            const bool more = key0 + STRIDE < end;
            if (more) {
                in.place(p, it, key0 + STRIDE);
                in.load_keys(fk);
                in.look_up(p, it, key0 + 2 * STRIDE);
            }
            __builtin_amdgcn_sched_barrier(0);
            if (key0 + S::KS > least || it.touches_hole(key0, S::KS)) {
                q4_mask<F32, DB, NT>(s, r, it, key0, lane);
                odd |= q4_clear<F32, DB>(fv, it, key0, lane);
            }
            q4_softmax<F32, DB, NT>(s, w, r);
            q4_weigh<F32, DB, NT>(w, fv, r);
            __builtin_amdgcn_sched_barrier(0);
            if (more)
                in.load_vals(fv);
        }
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

// LONE: own items go a wavefront each
template <bool F32, int DB, int NTP, int NTO, bool LONE>
__global__ __launch_bounds__(ATT_WAVES * 64, DB > 128 || F32 ? 1 : 2) void attend_q4_kernel(AttendQ4Params p)
{
    __shared__ __align__(16) float lds[att_lds_floats<DB, ATT_WAVES>()];
    AttendItem it;
    if ((int32_t)blockIdx.x < p.wgs_prefix) {
        att_prefix_item<16 * NTP>(p, blockIdx.x, it);
        attend_q4<F32, DB, NTP, ATT_WAVES>(p, lds, it);
        return;
    }
    int32_t id = blockIdx.x - p.wgs_prefix;
    if (LONE) {
        id = id * ATT_WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        if (id >= p.items_own)
            return;
    }
    if (att_own_item<16 * NTO, false>(p, id, it))
        attend_q4<F32, DB, NTO, LONE ? 1 : ATT_WAVES>(p, lds, it);
}

// Parts so short and few that one launch does them: twice as many wavefronts an item instead of chunks, nothing to join
template <bool F32, int DB>
__global__ __launch_bounds__(ATT_FEW_WAVES * 64) void attend_q4_few_kernel(AttendQ4Params p)
{
    extern __shared__ __align__(16) float q4_few_lds[];
    AttendItem it;
    if (att_own_item<16, false>(p, blockIdx.x, it))
        attend_q4<F32, DB, 1, ATT_FEW_WAVES>(p, q4_few_lds, it);
}

// ------------------------------------------------------------------ host side
static int q4_widest(const griffin_kv_cache_q4 &C) { return C.dim > 128 || (C.dtype == GRIFFIN_F32 && C.dim > 64) ? 1 : 2; }

static AttPlan attend_q4_plan(const griffin_kv_cache_q4 &C, const griffin_kv_batch &B, const SeqTable &seqs, int32_t n_heads)
{
    AttPlan pl = {};
    const int widest = q4_widest(C);                       // tiles of 16 rows that the registers hold
    const int32_t group = n_heads / C.kv_heads;
    const int64_t rows = (int64_t)seqs.cu[seqs.n] * group;
    int64_t longest = 0;
    for (int b = 0; b < seqs.n; ++b)
        longest = std::max(longest, (int64_t)(seqs.cu[b + 1] - seqs.cu[b]) * group);
    pl.nto = longest <= 16 ? 1 : widest;
    pl.ntp = rows <= 16 ? 1 : widest;
    if (pl.nto == widest)                                  // compiled pairs: (1, 1), (2, 1), (2, 2)
        pl.ntp = widest;
    pl.rows_own = 16 * pl.nto;
    pl.rows_prefix = 16 * pl.ntp;
    int64_t tiles = 0;
    for (int b = 0; b < seqs.n; ++b)
        tiles += ((int64_t)(seqs.cu[b + 1] - seqs.cu[b]) * group + pl.rows_own - 1) / pl.rows_own;
    pl.tiles_own = (int32_t)tiles;
    pl.tiles_prefix = B.n_prefix > 0 ? (int32_t)((rows + pl.rows_prefix - 1) / pl.rows_prefix) : 0;
    pl.lone = C.kv_heads * tiles >= 1024 && B.max_len <= 256;
    const int64_t step = ATT_WAVES * 32;
    const int64_t work_prefix = C.kv_heads * (int64_t)pl.tiles_prefix * B.n_prefix, work_own = C.kv_heads * tiles * B.max_len;
    const auto chunk = [&](int64_t work, int32_t keys) {   // no longer than the part: up to 2^30 keys and a quantum
        const int64_t even = std::min((work + 511) / 512, (int64_t)keys);
        return (int32_t)((std::max(even, (int64_t)1) + step - 1) / step * step);
    };
    const int64_t work = work_prefix + work_own;
    pl.chunk_prefix = chunk(pl.lone ? work_prefix : work, B.n_prefix);
    pl.chunk_own = pl.lone ? (int32_t)((B.max_len + step - 1) / step * step) : chunk(work, B.max_len);
    const int64_t all = (int64_t)B.n_prefix + B.max_len;
    pl.few = longest <= 16 && C.kv_heads * tiles <= 512 && all <= ATT_FEW_WAVES / ATT_WAVES * step && C.dim <= 128;
    pl.ahead = B.n_prefix > 0 && pl.few;
    if (pl.ahead)
        pl.tiles_prefix = 0;
    if (pl.few)
        pl.chunk_own = (int32_t)((all + 15 + step - 1) / step * step);
    pl.chunks_prefix = pl.ahead ? 0 : (B.n_prefix + pl.chunk_prefix - 1) / pl.chunk_prefix;
    pl.chunks_own = pl.ahead ? 1 : (B.max_len + pl.chunk_own - 1) / pl.chunk_own;
    return pl;
}

size_t attend_q4_floats(const griffin_kv_cache_q4 &C, const griffin_kv_batch &B, const SeqTable &seqs, int32_t n_heads)
{
    if (!attend_takes(seqs, n_heads))
        return 0;
    const AttPlan pl = attend_q4_plan(C, B, seqs, n_heads);
    const size_t slots = (size_t)seqs.cu[seqs.n] * n_heads * (pl.chunks_prefix + pl.chunks_own);
    return pl.chunks_prefix + pl.chunks_own < 2 ? 0 : slots * (C.dim + 2);
}

template <bool F32, int DB, int NTP, int NTO>
static int go_rows(const AttendQ4Params &p, bool lone, hipStream_t st)
{
    const int32_t wgs = p.wgs_prefix + (lone ? (p.items_own + ATT_WAVES - 1) / ATT_WAVES : p.items_own);
    if (lone)
        hipLaunchKernelGGL((attend_q4_kernel<F32, DB, NTP, NTO, true>), dim3(wgs), dim3(ATT_WAVES * 64), 0, st, p);
    else
        hipLaunchKernelGGL((attend_q4_kernel<F32, DB, NTP, NTO, false>), dim3(wgs), dim3(ATT_WAVES * 64), 0, st, p);
    return check_launch("attend_q4_kernel");
}

template <bool F32, int DB>
static int attend_typed(AttendQ4Params &p, const AttPlan &pl, hipStream_t st)
{
    p.wgs_prefix = p.kv_heads * pl.tiles_prefix * pl.chunks_prefix;
    p.items_own = p.kv_heads * pl.tiles_own * pl.chunks_own;
    if constexpr (DB <= 128)
        if (pl.few) {
            constexpr int bytes = att_lds_floats<DB, ATT_FEW_WAVES>() * sizeof(float);
            RAISE_LDS_LIMIT((attend_q4_few_kernel<F32, DB>), bytes);
            hipLaunchKernelGGL((attend_q4_few_kernel<F32, DB>), dim3(p.items_own), dim3(ATT_FEW_WAVES * 64), bytes, st, p);
            return check_launch("attend_q4_few_kernel");
        }
    int rc;
    if constexpr (DB <= 64 || (DB <= 128 && !F32)) {
        if (pl.nto == 2)
            rc = go_rows<F32, DB, 2, 2>(p, pl.lone, st);
        else if (pl.ntp == 2)
            rc = go_rows<F32, DB, 2, 1>(p, pl.lone, st);
        else
            rc = go_rows<F32, DB, 1, 1>(p, pl.lone, st);
    } else
        rc = go_rows<F32, DB, 1, 1>(p, pl.lone, st);
    return rc == GRIFFIN_OK && p.part ? launch_attend_join(p, !F32, st) : rc;
}

template <bool F32>
static int attend_width(AttendQ4Params &p, const AttPlan &pl, hipStream_t st)
{
    if (p.dim <= 64)
        return attend_typed<F32, 64>(p, pl, st);
    return p.dim <= 128 ? attend_typed<F32, 128>(p, pl, st) : attend_typed<F32, 256>(p, pl, st);
}

int launch_attend_q4(const AttendQ4Job &job, const SeqTable &seqs, hipStream_t st)
{
    const griffin_kv_cache_q4 &C = job.C;
    if (!attend_takes(seqs, job.n_heads))
        return GRIFFIN_EUNSUPPORTED;
    const AttPlan pl = attend_q4_plan(C, job.B, seqs, job.n_heads);
    if (!att_launch_fits(pl, C.kv_heads))
        return GRIFFIN_EUNSUPPORTED;
    AttendQ4Params p = {};
    p.q = job.q; p.K = C.K; p.V = C.V; p.out = job.out;
    p.ldq = job.ldq; p.hsq = job.hsq; p.ldo = job.ldo; p.hso = job.hso;
    att_set_up(p, pl, job.B, seqs, job.n_heads, C.kv_heads, C.dim, C.page_size, C.n_pages, job.scale, job.ws);
    p.s = q4_shape(C);
    return C.dtype == GRIFFIN_BF16 ? attend_width<false>(p, pl, st) : attend_width<true>(p, pl, st);
}

}  // namespace griffin
