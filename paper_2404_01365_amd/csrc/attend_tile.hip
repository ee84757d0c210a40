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
#include "attend_tile.h"

namespace griffin {

// A step's keys and values on their way: page numbers looked up (they come from memory, so two steps ahead), made places, loaded into registers, stored in
// LDS.  A wavefront brings in pieces of the same tiles of 16 keys of both: of keys a piece of 32 features in the order of the A operands, of values whole rows.
template <int DB, bool FULL>
struct TileStage {
    using S = TileShape<DB>;
    static constexpr int PIECES = S::BYTES / (16 * 64 * ATT_TILE_WAVES);       // 16-byte pieces of either that a thread brings in
    const char *K, *V;                       // of the kv head
    uint32_t stride, at_k, at_v;             // bytes from key to key; the lane's place in a tile
    int32_t page[PIECES];
    uint64_t base[PIECES];
    att_u32x4 k[PIECES], v[PIECES];

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
        for (int i = 0; i < PIECES; ++i)
            page[i] = att_look_up(p, it, key0 + 16 * tile_of(wave, i));
    }

    __device__ __forceinline__ void place(const AttendParams &p, const AttendItem &it, int32_t key0, int wave)
    {
#pragma unroll
        for (int i = 0; i < PIECES; ++i)
            base[i] = att_place<2>(p, it, page[i], key0 + 16 * tile_of(wave, i));
    }

    __device__ __forceinline__ void load(const AttendParams &p, int wave, int lane)
    {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
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
        for (int i = 0; i < PIECES; ++i) {
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
        for (int i = 0; i < PIECES; ++i) {
            const int row = tile_of(wave, i) * 16 + row_of(wave, lane);
            *(lds_u32x4 *)(uintptr_t)(keys + (wave + ATT_TILE_WAVES * i) * 1024 + lane * 16) = k[i];
            *(lds_u32x4 *)(uintptr_t)(vals + row * S::ROW + (lane % (DB / 8) ^ tile_turn<DB>(row) << 1) * 16) = v[i];
        }
    }
};

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

template <int DB, bool FULL>
struct TileBf16 {
    using S = TileShape<DB>;
    using Params = AttendParams;
    using Rows = TileRows<DB>;
    using Stage = TileStage<DB, FULL>;
    static constexpr int WAVES = ATT_TILE_WAVES;
    static constexpr float LIFT = 0;

    static __device__ __forceinline__ att_f32x4 product(att_u32x4 a, att_u32x4 b, att_f32x4 c) { return att_mfma(a, b, c); }
    static __device__ __forceinline__ void add_weights(att_f32x4 &l, att_u32x4 w) { att_add_weights(l, w); }
    static __device__ __forceinline__ uint32_t weights(float a, float b) { return f32x2_to_bf16x2(a, b); }
    static __device__ __forceinline__ float scale2(const AttendParams &p, const Rows &, int) { return p.scale2; }
    static __device__ __forceinline__ void load_row(const AttendParams &p, Rows &r, int n, int64_t row, int lane)
    {
        const char *at = (const char *)p.q + row * 2 + (lane >> 4) * 16;
#pragma unroll
        for (int s = 0; s < S::NQ; ++s) {
            if (FULL || s * 32 + (lane >> 4) * 8 < p.dim)
                r.q[n][s] = *(const att_u32x4 *)(at + s * 64);
            else
                r.q[n][s] = att_u32x4{0, 0, 0, 0};
        }
    }
    static __device__ __forceinline__ void add_odd(const AttendParams &p, const AttendItem &it, Rows &r, int32_t key, int32_t most)
    {
        tile_add_infinite<DB, FULL>(p, it, r, key, most);
    }
    static __device__ __forceinline__ void order(Rows &) {}
    static __device__ __forceinline__ bool own_item(const AttendParams &p, int32_t id, AttendItem &it) { return att_own_item<16, false>(p, id, it); }
    template <int WAVES>
    static __device__ __forceinline__ void own_rows(const AttendParams &p, float *lds, const AttendItem &it)
    {
        attend_rows<true, DB, FULL, 1, WAVES>(p, lds, it);
    }
};

template <int DB>
static int go(const AttendParams &p, int32_t wgs, bool each, hipStream_t st)
{
    return p.dim == DB ? go_tiles_and_rows<TileBf16<DB, true>, DB, true>(p, wgs, each, st) : go_tiles_and_rows<TileBf16<DB, false>, DB, false>(p, wgs, each, st);
}

int launch_attend_tiles(const AttendParams &p, int32_t wgs, bool each, hipStream_t st)
{
    if (p.dim <= 64)
        return go<64>(p, wgs, each, st);
    return p.dim <= 128 ? go<128>(p, wgs, each, st) : go<256>(p, wgs, each, st);
}

}  // namespace griffin
