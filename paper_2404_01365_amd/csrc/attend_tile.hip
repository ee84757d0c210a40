// Attention of many rows (bf16): prompts, and a prefix that more than 64 rows share.  The mathematics and the arrangement of scores
// and sums are those of attend_rows.h; here eight wavefronts of 32 rows each (16 of heads wider than 128) take the same keys, which go through LDS
// 64 at a time (32 of the wider heads), two steps' worth of room, so that a step's loads travel while the step before is computed.
//
// Keys lie in LDS in the order of the A operands (a lane's 16 bytes side by side: reads without bank conflicts).  Values lie as in memory, a row a
// key; V^T's operand is read with ds_read_b64_tr_b16, by which 16 lanes fetch four rows' 16 features and get a feature's four keys each.  The 32-byte
// pieces of a row are exchanged by the row's number so that those rows fall into different banks.
//
// The rows' reference maximum moves only when scores outgrow it by more than 8 (base 2): weights then are up to 2^8 (their rounding to bf16 is
// relative, and cancels from what a dominating one weighs, as the sum is of rounded ones, too), and o is scaled a few times instead of at every step.
//
// Bound by the matrix cores and what stands between the two products.  A step of 64 keys for 32 rows of 128 features is 64 products of 16x16x32 a wavefront and four with ones
// for the sums, two wavefronts a SIMD: at 8.25 ns each when they are fed without a pause 1.12 us, and some 0.5 us of weights (exponentials, maxima, rounding) for
// both.  The two hardly overlap, though they come from different wavefronts: two products and eight multiply-adds of two wavefronts take 49 ns together, 33 and 20
// apart.  So some 1.6 us is what this arrangement can reach, and 2.0 is measured; what the rest goes into is not known.  Prompts of 2048, 1117, 604 and 381 tokens of 32
// heads on 8, 49 GFLOP that are seen: 74 us = 660 TFLOP/s of them, caches cold 89.  Tried and slower on these, 88 to 117 us: the halves of a workgroup in turn, one multiplying while the other forms weights; products and
// weights of neighbouring tiles interleaved within a wavefront; four wavefronts of 64 rows.
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
    static constexpr int PIECES = BYTES / (16 * 64 * ATT_TILE_WAVES);      // 16-byte pieces of either that a thread brings in
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

// A step's keys and values on their way: page numbers looked up (they come from memory, so two steps ahead), made places, loaded into registers, stored in
// LDS.  A wavefront brings in pieces of the same tiles of 16 keys of both: of keys a piece of 32 features in the order of the A operands, of values whole rows.
template <int DB, bool FULL>
struct TileStage {
    using S = TileShape<DB>;
    const char *K, *V;                       // of the kv head
    uint32_t stride, at_k, at_v;             // bytes from key to key; the lane's place in a tile
    int32_t page[S::PIECES];
    uint64_t base[S::PIECES];
    att_u32x4 k[S::PIECES], v[S::PIECES];

    static __device__ __forceinline__ int tile_of(int wave, int i) { return (wave + ATT_TILE_WAVES * i) / S::NQ; }
    static __device__ __forceinline__ int row_of(int wave, int lane) { return (wave * 64 / (DB / 8) + lane / (DB / 8)) & 15; }
    static_assert(64 / (DB / 8) * S::NQ == 16 && 64 * ATT_TILE_WAVES / (DB / 8) % 16 == 0, "tile_of holds for keys and values, row_of for all pieces");

    __device__ __forceinline__ TileStage(const AttendParams &p, const AttendItem &it, int wave, int lane)
    {
        K = (const char *)p.K + it.hk * p.head_stride * 2;
        V = (const char *)p.V + it.hk * p.head_stride * 2;
        stride = (uint32_t)p.token_stride * 2;
        at_k = (lane & 15) * stride + (wave % S::NQ * 32 + (lane >> 4) * 8) * 2;
        at_v = row_of(wave, lane) * stride + lane % (DB / 8) * 16;
    }

    __device__ __forceinline__ void look_up(const AttendParams &p, const AttendItem &it, int32_t key0, int wave)
    {
#pragma unroll
        for (int i = 0; i < S::PIECES; ++i)
            page[i] = att_look_up(p, it, key0 + 16 * tile_of(wave, i));
    }

    __device__ __forceinline__ void place(const AttendParams &p, const AttendItem &it, int32_t key0, int wave)
    {
#pragma unroll
        for (int i = 0; i < S::PIECES; ++i)
            base[i] = att_place<2>(p, it, page[i], key0 + 16 * tile_of(wave, i));
    }

    __device__ __forceinline__ void load(const AttendParams &p, int wave, int lane)
    {
#pragma unroll
        for (int i = 0; i < S::PIECES; ++i) {
            // the piece's features are the same in every round of ATT_TILE_WAVES pieces.  Keys' features from dim on are zero, as the queries' are;
            // values' end in outputs that are not stored
            if (FULL || wave % S::NQ * 32 + (lane >> 4) * 8 < p.dim)
                k[i] = *(const att_u32x4 *)(K + base[i] + at_k);
            else
                k[i] = att_u32x4{0, 0, 0, 0};
            if (FULL || lane % (DB / 8) * 8 < p.dim)
                v[i] = *(const att_u32x4 *)(V + base[i] + at_v);
            else
                v[i] = att_u32x4{0, 0, 0, 0};
        }
    }
    static_assert(ATT_TILE_WAVES % S::NQ == 0, "a wavefront's pieces of keys have the same features");

    // values behind the last key or in the hole, and infinite and NaN ones, as zeros; true if there were any of these
    __device__ __forceinline__ bool clear(const AttendItem &it, int32_t key0, int wave, int lane)
    {
        uint32_t kept = ~0u;
#pragma unroll
        for (int i = 0; i < S::PIECES; ++i) {
            const int32_t key = key0 + 16 * tile_of(wave, i) + row_of(wave, lane);
            const bool in = key < it.end && !it.missing(key);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t m = att_finite_mask(v[i][j]);
                v[i][j] = in ? v[i][j] & m : 0;
                kept &= in ? m : ~0u;
            }
        }
        return kept != ~0u;
    }

    __device__ __forceinline__ void store(uint32_t keys, uint32_t vals, int wave, int lane) const
    {
#pragma unroll
        for (int i = 0; i < S::PIECES; ++i) {
            const int row = tile_of(wave, i) * 16 + row_of(wave, lane);
            *(lds_u32x4 *)(uintptr_t)(keys + (wave + ATT_TILE_WAVES * i) * 1024 + lane * 16) = k[i];
            *(lds_u32x4 *)(uintptr_t)(vals + row * S::ROW + (lane % (DB / 8) ^ tile_turn<DB>(row) << 1) * 16) = v[i];
        }
    }
};

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

// In steps in which rows differ in the keys that they see, or in which keys end, infinite and NaN values of keys that a row does not see must not reach
// it, as 0 x Inf would: there they are stored as zeros, and what was made zero is added at the end to the rows that do see it.
template <int DB, bool FULL>
__device__ __forceinline__ void tile_add_infinite(const AttendParams &p, const AttendItem &it, TileRows<DB> &r, int32_t key, int32_t most)
{
    using S = TileShape<DB>;
    const int d = (threadIdx.x >> 4 & 3) * 4;
    for (; key < most; ++key) {
        const uint16_t *at = (const uint16_t *)((const char *)((const uint16_t *)p.V + it.hk * p.head_stride) +
                                                att_place<2>(p, it, att_look_up(p, it, key), key)) + d;
#pragma unroll
        for (int e = 0; e < S::NO; ++e) {
            __builtin_amdgcn_sched_barrier(0);
            const uint2 x = FULL || e * 16 + d < p.dim ? *(const uint2 *)(at + e * 16) : make_uint2(0, 0);
            const uint32_t odd[2] = {x.x & ~att_finite_mask(x.x), x.y & ~att_finite_mask(x.y)};
#pragma unroll
            for (int n = 0; n < S::NT; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    r.o[n][e][i] += key < r.end[n] && !it.missing(key) ? (i & 1 ? bf16_hi(odd[i / 2]) : bf16_lo(odd[i / 2])) : 0.0f;
        }
    }
}

// O^T += V^T P^T
template <int DB>
__device__ __forceinline__ void tile_weigh(uint32_t vals, const att_u32x4 (&w)[TileShape<DB>::NT][TileShape<DB>::KT / 2], TileRows<DB> &r)
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
            att_add_weights(r.l[n], w[n][h]);
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
                r.o[n][e + i % G] = att_mfma(a[now][i], w[n][i / G], r.o[n][e + i % G]);
        }
    }
    __builtin_amdgcn_sched_barrier(0);
}

template <int DB>
using TileScores = att_f32x4[TileShape<DB>::NT][TileShape<DB>::KT];

// S^T = K Q^T
template <int DB>
__device__ __forceinline__ void tile_scores(uint32_t keys, TileScores<DB> &s, const TileRows<DB> &r)
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
                s[n][t] = att_mfma(a[f & 1][i], r.q[n][c], c == 0 ? att_f32x4{0, 0, 0, 0} : s[n][t]);
            }
    }
    __builtin_amdgcn_sched_barrier(0);
}

// Scores to weights in bf16; the rows' reference carried on, sum and o scaled when it moves
template <int DB>
__device__ __forceinline__ void tile_softmax(bool masked, TileScores<DB> &s, att_u32x4 (&w)[TileShape<DB>::NT][TileShape<DB>::KT / 2], TileRows<DB> &r,
                                             float scale2, const AttendItem &it, int32_t key0)
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
        top[n] *= scale2;
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
        const float base = r.m[n] == -INFINITY ? 0.0f : r.m[n];
#pragma unroll
        for (int t = 0; t < S::KT; ++t) {
            float x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
                x[e] = __builtin_amdgcn_exp2f(s[n][t][e] * scale2 - base);
            w[n][t / 2][t % 2 * 2] = f32x2_to_bf16x2(x[0], x[1]);
            w[n][t / 2][t % 2 * 2 + 1] = f32x2_to_bf16x2(x[2], x[3]);
        }
    }
}

// OWN: who takes own parts.  TILES: they are tiles, too.  ROWS, EACH: they are of a few rows, and a workgroup, or each wavefront, takes one as attend_rows.h has it
// behind the tiles, which saves a launch.
enum TileOwn { OWN_TILES, OWN_ROWS, OWN_EACH };

template <int DB, bool FULL, TileOwn OWN>
__global__ __launch_bounds__(64 * ATT_TILE_WAVES) void attend_tile_kernel(AttendParams p)
{
    using S = TileShape<DB>;
    extern __shared__ __align__(1024) char tile_lds[];        // two steps of keys and values
    const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)tile_lds;
    AttendItem it;
    if ((int32_t)blockIdx.x < p.wgs_prefix)
        att_prefix_item<att_tile_rows(DB)>(p, blockIdx.x, it);
    else if constexpr (OWN == OWN_TILES) {
        if (!att_own_item<att_tile_rows(DB), true>(p, blockIdx.x - p.wgs_prefix, it))
            return;
    } else {
        int32_t id = blockIdx.x - p.wgs_prefix;
        if (OWN == OWN_EACH)
            id = id * ATT_TILE_WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        if (id < p.items_own && att_own_item<16, false>(p, id, it))
            attend_rows<true, DB, FULL, 1, OWN == OWN_EACH ? 1 : ATT_TILE_WAVES>(p, (float *)tile_lds, it);
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
    TileRows<DB> r;
#pragma unroll
    for (int n = 0; n < S::NT; ++n) {
        const int32_t row = of(n);
        r.end[n] = sees(row);
        const int32_t token = p.by_group(row), head = it.hk * p.group + row - token * p.group;
        const char *at = (const char *)p.q + ((int64_t)(it.token0 + token) * p.ldq + (int64_t)head * p.hsq) * 2 +
                         (lane >> 4) * 16;
#pragma unroll
        for (int s = 0; s < S::NQ; ++s) {
            if (FULL || s * 32 + (lane >> 4) * 8 < p.dim)
                r.q[n][s] = *(const att_u32x4 *)(at + s * 64);
            else
                r.q[n][s] = att_u32x4{0, 0, 0, 0};
        }
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
    TileStage<DB, FULL> even(p, it, wave, lane), odds(p, it, wave, lane);
    bool odd = false;
    uint32_t room = 0;
    const auto store = [&](TileStage<DB, FULL> &in, int32_t key0) {
        if (key0 >= clear || it.touches_hole(key0, S::KEYS))
            odd |= in.clear(it, key0, wave, lane);
        in.store(lds + room, lds + 2 * S::BYTES + room, wave, lane);
    };
    const auto step = [&](TileStage<DB, FULL> &now, TileStage<DB, FULL> &other, int32_t key0) {
        if (key0 + 2 * S::KEYS < it.end) {
            now.load(p, wave, lane);
            now.look_up(p, it, key0 + 4 * S::KEYS, wave);
        }
        if (key0 < most) {
            TileScores<DB> s;
            att_u32x4 w[S::NT][S::KT / 2];
            tile_scores<DB>(lds + room, s, r);
            tile_softmax<DB>(key0 + S::KEYS > least || it.touches_hole(key0, S::KEYS), s, w, r, p.scale2, it, key0);
            tile_weigh<DB>(tile_vals_at<DB>(lds + 2 * S::BYTES + room), w, r);
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
            tile_add_infinite<DB, FULL>(p, it, r, at_hole, at_hole + S::KEYS < it.end ? at_hole + S::KEYS : it.end);
        tile_add_infinite<DB, FULL>(p, it, r, clear, most);
    }
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

template <int DB, TileOwn OWN>
static int go_tiles(const AttendParams &p, int32_t wgs, hipStream_t st)
{
    constexpr int rooms = 4 * TileShape<DB>::BYTES, sums = OWN == OWN_ROWS ? att_lds_floats<DB, ATT_TILE_WAVES>() * 4 : 0, bytes = rooms > sums ? rooms : sums;
    if (p.dim == DB) {
        RAISE_LDS_LIMIT((attend_tile_kernel<DB, true, OWN>), bytes);
        hipLaunchKernelGGL((attend_tile_kernel<DB, true, OWN>), dim3(wgs), dim3(64 * ATT_TILE_WAVES), bytes, st, p);
    } else {
        RAISE_LDS_LIMIT((attend_tile_kernel<DB, false, OWN>), bytes);
        hipLaunchKernelGGL((attend_tile_kernel<DB, false, OWN>), dim3(wgs), dim3(64 * ATT_TILE_WAVES), bytes, st, p);
    }
    return check_launch("attend_tile_kernel");
}

template <int DB>
static int go_tiles_and_rows(const AttendParams &p, int32_t wgs, bool each, hipStream_t st)
{
    if (each)
        return go_tiles<DB, OWN_EACH>(p, wgs + (p.items_own + ATT_TILE_WAVES - 1) / ATT_TILE_WAVES, st);
    return p.items_own > 0 ? go_tiles<DB, OWN_ROWS>(p, wgs + p.items_own, st) : go_tiles<DB, OWN_TILES>(p, wgs, st);
}

int launch_attend_tiles(const AttendParams &p, int32_t wgs, bool each, hipStream_t st)
{
    if (p.dim <= 64)
        return go_tiles_and_rows<64>(p, wgs, each, st);
    return p.dim <= 128 ? go_tiles_and_rows<128>(p, wgs, each, st) : go_tiles<256, OWN_TILES>(p, wgs, st);
}

}  // namespace griffin
