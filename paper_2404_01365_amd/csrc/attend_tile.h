// Attention of many rows: what the kernels over caches of bf16 (attend_tile.hip) and in 4 bits (attend_q4_tile.hip) share.  F, the format, says
//   WAVES                    of a workgroup
//   Params, Rows, Stage      a launch's arguments, a wavefront's rows (TileRows), and a step's keys and values on their way (attend_tile.hip describes one)
//   LIFT                     weights are 2^LIFT times what they stand for, numerator and denominator alike
//   product, add_weights     a product of the matrix cores, and one with ones
//   weights                  two weights rounded into a word
//   scale2                   of a row's scores
//   load_row                 a row's queries
//   add_odd                  infinite and NaN values that were made zero in the steps of [key, most), added to the rows that see them
//   order                    the features of o as they are stored: element i of o[n][e] is feature 16 e + 4 (lane >> 4) + i
//   own_item, own_rows       the id-th own part of a few rows (false: no row needs it), and the work on it, by a workgroup or a wavefront
#pragma once

#include "attend_rows.h"

namespace griffin {

typedef __attribute__((ext_vector_type(4))) short att_s16x4;
typedef __attribute__((address_space(3))) att_s16x4 lds_s16x4;       // LDS is addressed by 32-bit offsets
typedef __attribute__((address_space(3))) att_u32x4 lds_u32x4;

template <int DB>
struct TileShape {
    static constexpr int NQ = DB / 32;                        // 32-feature pieces of a key
    static constexpr int NO = DB / 16;                        // tiles of 16 features of the output
    static constexpr int KEYS = att_tile_keys(DB);            // of a step
    static constexpr int KT = KEYS / 16;                      // tiles of 16 keys of a step
    static constexpr int NT = DB > 128 ? 1 : 2;               // tiles of 16 rows of a wavefront
    static constexpr int ROW = DB * 2;                        // bytes of a value's row
    static constexpr int BYTES = KEYS * ROW;            // of a step's keys, and of its values
};

template <int DB>
struct TileRows {
    using S = TileShape<DB>;
    att_u32x4 q[S::NT][S::NQ];
    int32_t end[S::NT];
    float m[S::NT];
    att_f32x4 l[S::NT];                                       // the row's sum in every element (att_add_weights)
    att_f32x4 o[S::NT][S::NO];
};

// which 32-byte piece of a value's row lies in the place of piece 0: rows whose places would share banks differ in it
template <int DB>
__device__ __forceinline__ int tile_turn(int row) { return DB >= 128 ? row & 7 : (row >> 1) & 3; }

// A operand of V^T: features 16 e .. + 15 of the keys of tiles 2h and 2h + 1, in the order in which the lanes hold their scores.  `at` is the
// lane's place for e = 0 (tile_vals_at); the others' differ from it in the bits of the turned pieces.
template <int DB>
__device__ __forceinline__ uint32_t tile_vals_at(uint32_t lds)
{
    using S = TileShape<DB>;
    const int lane = threadIdx.x & 63, row = (lane >> 4) * 4 + ((lane >> 2) & 3);
    return lds + row * S::ROW + tile_turn<DB>(row) * 32 + (lane & 3) * 8;
}

template <int DB>
__device__ __forceinline__ att_u32x4 tile_vals(uint32_t at, int e, int h)
{
    using S = TileShape<DB>;
    typedef __attribute__((ext_vector_type(2))) uint32_t pair_t;
    const uint32_t x = at ^ e * 32;
    const pair_t lo = __builtin_bit_cast(pair_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(uintptr_t)(x + 2 * h * 16 * S::ROW)));
    const pair_t hi = __builtin_bit_cast(pair_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(uintptr_t)(x + (2 * h + 1) * 16 * S::ROW)));
    return att_u32x4{lo.x, lo.y, hi.x, hi.y};
}

// O^T += V^T P^T
template <class F, int DB>
__device__ __forceinline__ void tile_weigh(uint32_t vals, const att_u32x4 (&w)[TileShape<DB>::NT][TileShape<DB>::KT / 2], typename F::Rows &r)
{
    using S = TileShape<DB>;
    constexpr int H = S::KT / 2, G = 4 / H;                   // operands of G tiles of features are read while those before are multiplied
    att_u32x4 a[2][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        a[0][i] = tile_vals<DB>(vals, i % G, i / G);
#pragma unroll
    for (int h = 0; h < H; ++h)                               // while the first operands are on their way
#pragma unroll
        for (int n = 0; n < S::NT; ++n)
            F::add_weights(r.l[n], w[n][h]);
#pragma unroll
    for (int e = 0; e < S::NO; e += G) {
        const int now = e / G & 1;
        __builtin_amdgcn_sched_barrier(0);
        if (e + G < S::NO)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                a[now ^ 1][i] = tile_vals<DB>(vals, e + G + i % G, i / G);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
#pragma unroll
            for (int n = 0; n < S::NT; ++n)
                r.o[n][e + i % G] = F::product(a[now][i], w[n][i / G], r.o[n][e + i % G]);
        }
    }
    __builtin_amdgcn_sched_barrier(0);
}

template <int DB>
using TileScores = att_f32x4[TileShape<DB>::NT][TileShape<DB>::KT];

// S^T = K Q^T
template <class F, int DB>
__device__ __forceinline__ void tile_scores(uint32_t keys, TileScores<DB> &s, const typename F::Rows &r)
{
    using S = TileShape<DB>;
    // two pieces of two tiles of keys are read while those before are multiplied: sums that follow each other are different ones
    constexpr int STEPS = S::KT / 2 * S::NQ / 2;
    const uint32_t at = keys + (threadIdx.x & 63) * 16;
    const auto read = [&](int f, int i) {
        const int t = f / (S::NQ / 2) * 2 + (i & 1), c = f % (S::NQ / 2) * 2 + (i >> 1);
        return *(const lds_u32x4 *)(uintptr_t)(at + (t * S::NQ + c) * 1024);
    };
    att_u32x4 a[2][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        a[0][i] = read(0, i);
#pragma unroll
    for (int f = 0; f < STEPS; ++f) {
        __builtin_amdgcn_sched_barrier(0);
        if (f + 1 < STEPS)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                a[f + 1 & 1][i] = read(f + 1, i);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int n = 0; n < S::NT; ++n) {
                const int t = f / (S::NQ / 2) * 2 + (i & 1), c = f % (S::NQ / 2) * 2 + (i >> 1);
                s[n][t] = F::product(a[f & 1][i], r.q[n][c], c == 0 ? att_f32x4{0, 0, 0, 0} : s[n][t]);
            }
    }
    __builtin_amdgcn_sched_barrier(0);
}

// Scores to weights of 16 bits; the rows' reference carried on, sum and o scaled when it moves
template <class F, int DB>
__device__ __forceinline__ void tile_softmax(bool masked, TileScores<DB> &s, att_u32x4 (&w)[TileShape<DB>::NT][TileShape<DB>::KT / 2], typename F::Rows &r,
                                             const typename F::Params &p, const AttendItem &it, int32_t key0)
{
    using S = TileShape<DB>;
    const int lane = threadIdx.x & 63;
    if (masked)
#pragma unroll
        for (int n = 0; n < S::NT; ++n)
#pragma unroll
            for (int t = 0; t < S::KT; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int32_t key = key0 + 16 * t + (lane >> 4) * 4 + e;
                    s[n][t][e] = key < r.end[n] && !it.missing(key) ? s[n][t][e] : -INFINITY;
                }
    float top[S::NT];
    bool grown = false;
#pragma unroll
    for (int n = 0; n < S::NT; ++n) {
        top[n] = -INFINITY;
#pragma unroll
        for (int t = 0; t < S::KT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                top[n] = fmaxf(top[n], s[n][t][e]);
        top[n] *= F::scale2(p, r, n);
        grown |= top[n] > r.m[n] + 8.0f;
    }
    if (__any(grown))
#pragma unroll
        for (int n = 0; n < S::NT; ++n) {
            const float m = fmaxf(r.m[n], lane_groups_max(top[n]));
            const float f = m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(r.m[n] - m);        // nothing seen yet: nothing to scale
            r.m[n] = m;
            r.l[n] *= f;
#pragma unroll
            for (int e = 0; e < S::NO; ++e)
                r.o[n][e] *= f;
        }
#pragma unroll
    for (int n = 0; n < S::NT; ++n) {
        const float base = (r.m[n] == -INFINITY ? 0.0f : r.m[n]) - F::LIFT;
#pragma unroll
        for (int t = 0; t < S::KT; ++t) {
            float x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
                x[e] = __builtin_amdgcn_exp2f(s[n][t][e] * F::scale2(p, r, n) - base);
            w[n][t / 2][t % 2 * 2] = F::weights(x[0], x[1]);
            w[n][t / 2][t % 2 * 2 + 1] = F::weights(x[2], x[3]);
        }
    }
}

// OWN: who takes own parts.  TILES: they are tiles, too.  ROWS, EACH: they are of a few rows, and a workgroup, or each wavefront, takes one as attend_rows.h has it
// behind the tiles, which saves a launch.
enum TileOwn { OWN_TILES, OWN_ROWS, OWN_EACH };

template <class F, int DB, bool FULL, TileOwn OWN>
__global__ __launch_bounds__(64 * F::WAVES, 2) void attend_tile_kernel(typename F::Params p)
{
    using S = TileShape<DB>;
    using Stage = typename F::Stage;
    extern __shared__ __align__(1024) char tile_lds[];        // two steps of keys and values
    const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)tile_lds;
    AttendItem it;
    if ((int32_t)blockIdx.x < p.wgs_prefix)
        att_prefix_item<16 * S::NT * F::WAVES>(p, blockIdx.x, it);
    else if constexpr (OWN == OWN_TILES) {
        if (!att_own_item<16 * S::NT * F::WAVES, true>(p, blockIdx.x - p.wgs_prefix, it))
            return;
    } else {
        int32_t id = blockIdx.x - p.wgs_prefix;
        if (OWN == OWN_EACH)
            id = id * F::WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        if (id < p.items_own && F::own_item(p, id, it))
            F::template own_rows<OWN == OWN_EACH ? 1 : F::WAVES>(p, (float *)tile_lds, it);
        return;
    }
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int32_t first = it.first + wave * 16 * S::NT;
    const auto sees = [&](int32_t row) {                      // where the keys that a row sees end
        const int32_t to = it.own + p.by_group(row) + 1;
        return it.own < 0 || to > it.end ? it.end : to;
    };
    // rows behind the last repeat it and are not stored
    const auto of = [&](int n) { return first + 16 * n + (lane & 15) < it.rows ? first + 16 * n + (lane & 15) : it.rows - 1; };
    typename F::Rows r;
#pragma unroll
    for (int n = 0; n < S::NT; ++n) {
        const int32_t row = of(n);
        r.end[n] = sees(row);
        const int32_t token = p.by_group(row), head = it.hk * p.group + row - token * p.group;
        F::load_row(p, r, n, (int64_t)(it.token0 + token) * p.ldq + (int64_t)head * p.hsq, lane);
        r.m[n] = -INFINITY;
        r.l[n] = att_f32x4{0, 0, 0, 0};
#pragma unroll
        for (int e = 0; e < S::NO; ++e)
            r.o[n][e] = att_f32x4{0, 0, 0, 0};
    }
    // keys that all rows of the wavefront see, and that any sees (none: it has no rows)
    const int32_t least = first < it.rows ? sees(first) : it.begin;
    const int32_t most = first < it.rows ? sees(first + 16 * S::NT < it.rows ? first + 16 * S::NT - 1 : it.rows - 1) : it.begin;
    // steps from the one that begins at `clear` on have keys that some row of the workgroup does not see.  A first row that ends before this chunk begins: all of
    // its steps, and none of the chunk before, whose workgroup adds what is infinite there.
    const int32_t alike = sees(it.first) > it.begin ? sees(it.first) - it.begin : 0;
    const int32_t clear = it.begin + alike / S::KEYS * S::KEYS;
    // Loads are two steps ahead of their use: a step's work is shorter than a read from memory under load takes.  Two stages take turns; step i
    // loads step i + 2's, looks up i + 4's pages, and stores i + 1's in the other room.
    Stage even(p, it, wave, lane), odds(p, it, wave, lane);
    bool odd = false;
    uint32_t room = 0;
    const auto store = [&](Stage &in, int32_t key0) {
        if (key0 >= clear || it.touches_hole(key0, S::KEYS))
            odd |= in.clear(it, key0, wave, lane);
        in.store(lds + room, lds + 2 * S::BYTES + room, wave, lane);
    };
    const auto step = [&](Stage &now, Stage &other, int32_t key0) {
        if (key0 + 2 * S::KEYS < it.end) {
            now.load(p, wave, lane);
            now.look_up(p, it, key0 + 4 * S::KEYS, wave);
        }
        if (key0 < most) {
            TileScores<DB> s;
            att_u32x4 w[S::NT][S::KT / 2];
            tile_scores<F, DB>(lds + room, s, r);
            tile_softmax<F, DB>(key0 + S::KEYS > least || it.touches_hole(key0, S::KEYS), s, w, r, p, it, key0);
            tile_weigh<F, DB>(tile_vals_at<DB>(lds + 2 * S::BYTES + room), w, r);
        }
        room ^= S::BYTES;
        if (key0 + S::KEYS < it.end) {
            store(other, key0 + S::KEYS);
            other.place(p, it, key0 + 3 * S::KEYS, wave);
        }
        __syncthreads();
    };
    even.look_up(p, it, it.begin, wave);
    odds.look_up(p, it, it.begin + S::KEYS, wave);
    even.place(p, it, it.begin, wave);
    odds.place(p, it, it.begin + S::KEYS, wave);
    even.load(p, wave, lane);
    even.look_up(p, it, it.begin + 2 * S::KEYS, wave);
    if (it.begin + S::KEYS < it.end)
        odds.load(p, wave, lane);
    odds.look_up(p, it, it.begin + 3 * S::KEYS, wave);
    store(even, it.begin);
    even.place(p, it, it.begin + 2 * S::KEYS, wave);
    __syncthreads();
    for (int32_t key0 = it.begin; key0 < it.end; key0 += 2 * S::KEYS) {
        step(even, odds, key0);
        if (key0 + S::KEYS >= it.end)
            break;
        step(odds, even, key0 + S::KEYS);
    }
    if (__syncthreads_or(odd)) {
        const int32_t at_hole = it.hole / S::KEYS * S::KEYS;                 // the step with the hole, if it comes before
        if (it.touches_hole(at_hole, S::KEYS) && at_hole < clear)
            F::add_odd(p, it, r, at_hole, at_hole + S::KEYS < it.end ? at_hole + S::KEYS : it.end);
        F::add_odd(p, it, r, clear, most);
    }
    F::order(r);
#pragma unroll
    for (int n = 0; n < S::NT; ++n) {
        const float l = r.l[n][0];
        if (first + 16 * n + (lane & 15) >= it.rows)
            continue;
        const int32_t row = of(n), of_group = p.by_group(row), token = it.token0 + of_group, head = it.hk * p.group + row - of_group * p.group;
        if (p.part) {
            const int64_t slot = ((int64_t)token * p.n_heads + head) * (p.chunks_prefix + p.chunks_own) + it.split;
            if (lane < 16)
                p.part_ml[slot] = make_float2(r.m[n], l);
            float *at = p.part + slot * p.dim + (lane >> 4) * 4;
#pragma unroll
            for (int e = 0; e < S::NO; ++e)
                if (FULL || e * 16 + (lane >> 4) * 4 < p.dim)
                    *(att_f32x4 *)(at + e * 16) = r.o[n][e];
        } else {
            const float f = l == 0.0f ? 0.0f : 1.0f / l;      // a row without keys: zeros
            uint16_t *at = (uint16_t *)p.out + (int64_t)token * p.ldo + (int64_t)head * p.hso + (lane >> 4) * 4;
#pragma unroll
            for (int e = 0; e < S::NO; ++e)
                if (FULL || e * 16 + (lane >> 4) * 4 < p.dim)
                    *(uint2 *)(at + e * 16) = make_uint2(f32x2_to_bf16x2(r.o[n][e][0] * f, r.o[n][e][1] * f),
                                                         f32x2_to_bf16x2(r.o[n][e][2] * f, r.o[n][e][3] * f));
        }
    }
}

template <class F, int DB, bool FULL, TileOwn OWN>
static int go_tiles(const typename F::Params &p, int32_t wgs, hipStream_t st)
{
    constexpr int rooms = 4 * TileShape<DB>::BYTES, sums = OWN == OWN_ROWS ? att_lds_floats<DB, F::WAVES>() * 4 : 0, bytes = rooms > sums ? rooms : sums;
    RAISE_LDS_LIMIT((attend_tile_kernel<F, DB, FULL, OWN>), bytes);
    hipLaunchKernelGGL((attend_tile_kernel<F, DB, FULL, OWN>), dim3(wgs), dim3(64 * F::WAVES), bytes, st, p);
    return check_launch("attend_tile_kernel");
}

template <class F, int DB, bool FULL>
static int go_tiles_and_rows(const typename F::Params &p, int32_t wgs, bool each, hipStream_t st)
{
    if constexpr (DB <= 128) {
        if (each)
            return go_tiles<F, DB, FULL, OWN_EACH>(p, wgs + (p.items_own + F::WAVES - 1) / F::WAVES, st);
        if (p.items_own > 0)
            return go_tiles<F, DB, FULL, OWN_ROWS>(p, wgs + p.items_own, st);
    }
    return go_tiles<F, DB, FULL, OWN_TILES>(p, wgs, st);
}

}  // namespace griffin
