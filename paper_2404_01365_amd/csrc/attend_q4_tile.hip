// Attention of many rows over a cache in 4 bits: attend_tile.h with codes that become fp16 on their way into LDS, once for all 256 rows of a workgroup (128 of heads wider
// than 128).  Four wavefronts bring in a step's keys, four its values, 16 tokens each: a lane loads 32 features of a token, which is one group or half of one.  Keys: what
// a lane has unpacked are its own 16 bytes of as many A operands as it loaded words, queries being laid out alike.  Values go into LDS in the order in which pairs come out of a word,
// features 0, 4, 1, 5, 2, 6, 3, 7 of every eight; that order is undone once, where the output leaves.
#include "attend_q4.h"
#include "attend_tile.h"

namespace griffin {

template <int DB>
struct Q4TileStage {
    using S = TileShape<DB>;
    static constexpr int W = S::NQ < 4 ? S::NQ : 4;           // words that a lane brings in
    static constexpr int PARTS = S::NQ / W;                   // ... of a token's, by as many wavefronts
    static_assert(S::KT * PARTS * 2 == ATT_TILE_WAVES, "a tile of 16 tokens a wavefront, of keys and of values");
    const char *pool;                        // of the kv head: keys, or values
    uint32_t at, at_pair, to;                // the lane's place in a tile, and in a step's room
    int32_t page;
    uint64_t codes, pairs;
    uint32_t w[W], pair;

    static __device__ __forceinline__ bool is_key(int wave) { return wave < ATT_TILE_WAVES / 2; }
    static __device__ __forceinline__ int tile_of(int wave) { return wave % (ATT_TILE_WAVES / 2) / PARTS; }

    __device__ __forceinline__ Q4TileStage(const AttendQ4Params &p, const AttendItem &it, int wave, int lane)
    {
        const int part = wave % PARTS, tile = tile_of(wave);
        pool = (const char *)(is_key(wave) ? p.K : p.V) + (uint64_t)it.hk * p.s.head_bytes;
        const int token = is_key(wave) ? lane & 15 : lane >> 2, row = tile * 16 + token;
        const int word = is_key(wave) ? (lane >> 4) * S::NQ + part * W : (part * 4 + (lane & 3)) * W;
        // features from dim on meet queries that are zero, or end in outputs that are not stored: some of the row's own will do
        const int f = word * 8 < p.dim ? word * 8 : 0;
        at = token * p.s.row_bytes + f / 2;
        at_pair = (token * p.s.groups + (f >> p.s.group_shift)) * 4;
        to = is_key(wave) ? (tile * S::NQ + part * W) * 1024 + lane * 16 : row * S::ROW + (word ^ tile_turn<DB>(row) << 1) * 16;
    }

    __device__ __forceinline__ void look_up(const AttendQ4Params &p, const AttendItem &it, int32_t key0, int wave)
    {
        page = att_look_up(p, it, key0 + 16 * tile_of(wave));
    }

    __device__ __forceinline__ void place(const AttendQ4Params &p, const AttendItem &it, int32_t key0, int wave)
    {
        int32_t key = key0 + 16 * tile_of(wave);
        key -= key < it.hole_end ? 0 : it.hole_end;
        const uint32_t in = key & ((1 << p.page_shift) - 1);
        const uint64_t block = (uint64_t)att_page(__builtin_amdgcn_readfirstlane(page), p.last_page) * (uint32_t)p.kv_heads * p.s.head_bytes;
        codes = block + in * p.s.row_bytes;
        pairs = block + p.s.pairs_at + in * p.s.groups * 4;
    }

    __device__ __forceinline__ void load(const AttendQ4Params &, int, int)
    {
        if constexpr (W == 2)
            *(uint2 *)w = *(const uint2 *)(pool + codes + at);
        else
            *(att_u32x4 *)w = *(const att_u32x4 *)(pool + codes + at);
        pair = *(const uint32_t *)(pool + pairs + at_pair);
    }

    // values behind the last key or in the hole, and groups of NaN, as zeros; true if there were any of these
    __device__ __forceinline__ bool clear(const AttendItem &it, int32_t key0, int wave, int lane)
    {
        if (is_key(wave))
            return false;
        const int32_t key = key0 + 16 * tile_of(wave) + (lane >> 2);
        const bool in = key < it.end && !it.missing(key), odd = q4_odd(pair);
        pair = in && !odd ? pair : 0;
        return in && odd;
    }

    __device__ __forceinline__ void store(uint32_t keys, uint32_t vals, int wave, int) const
    {
        const q4_pair scale = q4_scales(pair), middle = q4_middles(pair);
        const uint32_t room = is_key(wave) ? keys : vals;
#pragma unroll
        for (int i = 0; i < W; ++i) {
            att_u32x4 x;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                x[j] = q4_word(q4_value_pair(w[i] >> 4 * j, scale, middle));
            // keys: another operand, 1 KB on.  Values: the next 16 bytes, whose number's bits below the turn's or among them change
            *(lds_u32x4 *)(uintptr_t)(room + (is_key(wave) ? to + i * 1024 : to ^ i * 16)) = x;
        }
    }
};

template <int DB>
struct Q4TileRows : TileRows<DB> {
    float scale[TileShape<DB>::NT];
};

template <int DB>
struct TileQ4 {
    using S = TileShape<DB>;
    using Params = AttendQ4Params;
    using Rows = Q4TileRows<DB>;
    using Stage = Q4TileStage<DB>;
    static constexpr float LIFT = 7;                          // as in attend_q4.h

    static __device__ __forceinline__ att_f32x4 product(att_u32x4 a, att_u32x4 b, att_f32x4 c) { return q4_mfma(a, b, c); }
    static __device__ __forceinline__ void add_weights(att_f32x4 &l, att_u32x4 w) { l = q4_mfma(att_u32x4{Q4_ONES, Q4_ONES, Q4_ONES, Q4_ONES}, w, l); }
    static __device__ __forceinline__ uint32_t weights(float a, float b) { return q4_word(__builtin_bit_cast(q4_pair, __builtin_amdgcn_cvt_pkrtz(a, b))); }
    static __device__ __forceinline__ float scale2(const AttendQ4Params &, const Rows &r, int n) { return r.scale[n]; }
    static __device__ __forceinline__ void load_row(const AttendQ4Params &p, Rows &r, int n, int64_t row, int lane)
    {
        att_u32x4 q[1][S::NQ];
        r.scale[n] = q4_load_row<false, S::NQ>(p, q, row, lane);
#pragma unroll
        for (int w = 0; w < S::NQ; ++w)
            r.q[n][w] = q[0][w];
    }
    static __device__ __forceinline__ void add_odd(const AttendQ4Params &p, const AttendItem &it, Rows &r, int32_t key, int32_t most)
    {
        for (; key < most; ++key) {
            const char *at = (const char *)p.V + q4_pairs_of(p, it, key);
#pragma unroll
            for (int e = 0; e < S::NO; ++e) {                 // all four elements are of one eight of features
                const int d = e * 16 + (threadIdx.x >> 5 & 1) * 8;
                const bool odd = d < p.dim && q4_odd(*(const uint32_t *)(at + (d < p.dim ? d >> p.s.group_shift : 0) * 4));
#pragma unroll
                for (int n = 0; n < S::NT; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        r.o[n][e][i] = odd && key < r.end[n] && !it.missing(key) ? __builtin_nanf("") : r.o[n][e][i];
            }
        }
    }
    // Lanes l and l ^ 16 have features 0, 4, 1, 5 and 2, 6, 3, 7 of eight: each gives away two, and has four in a row
    static __device__ __forceinline__ void order(Rows &r)
    {
        const bool first = (threadIdx.x & 16) == 0;
#pragma unroll
        for (int n = 0; n < S::NT; ++n)
#pragma unroll
            for (int e = 0; e < S::NO; ++e) {
                const att_f32x4 v = r.o[n][e];
                const float a = __shfl_xor(first ? v[1] : v[0], 16), b = __shfl_xor(first ? v[3] : v[2], 16);
                r.o[n][e] = first ? att_f32x4{v[0], v[2], a, b} : att_f32x4{a, b, v[1], v[3]};
            }
    }
    static __device__ __forceinline__ bool own_item(const AttendQ4Params &p, int32_t id, AttendItem &it) { return q4_own_item<16>(p, id, it); }
    template <int WAVES>
    static __device__ __forceinline__ void own_rows(const AttendQ4Params &p, float *lds, const AttendItem &it)
    {
        attend_q4<false, DB, 1, WAVES>(p, lds, it);
    }
};

int launch_attend_q4_tiles(const AttendQ4Params &p, int32_t wgs, bool each, hipStream_t st)
{
    if (p.dim <= 64)
        return go_tiles_and_rows<TileQ4<64>, 64, false>(p, wgs, each, st);
    return p.dim <= 128 ? go_tiles_and_rows<TileQ4<128>, 128, false>(p, wgs, each, st) : go_tiles_and_rows<TileQ4<256>, 256, false>(p, wgs, each, st);
}

}  // namespace griffin
