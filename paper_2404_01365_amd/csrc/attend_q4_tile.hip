// Attention of many rows over a cache in 4 bits: attend_tile.h with codes that become fp16 on their way into LDS, once for all 128 rows of a workgroup (64 of heads wider than 128).
// Each of its four wavefronts brings in 16 tokens of a step's keys and values: a lane loads 32 features of a token, which is one group or half of one.  Keys: what a lane has
// unpacked are its own 16 bytes of as many A operands as it loaded words, queries being laid out alike.  Values go into LDS in the order in which pairs come out of a word, features 0, 4,
// 1, 5, 2, 6, 3, 7 of every eight; that order is undone once, where the output leaves.
//
// Bound by the matrix cores, reads from LDS and what stands between the two products, some 1.1, 0.9 and 1.0 us for 64 keys of 256 rows, of which two workgroups a CU, each at a place of its own,
// overlap a part: 1.9 us.  (One workgroup of eight wavefronts a CU, whose barriers keep them in step: a prompt of 1000 tokens of 32 heads on 8 48 instead of 35 us, of 2048 72 instead of 65,
// packed prompts of 2048, 1117, 604 and 381 tokens 77.6 instead of 75.0, 2800 tokens of 16 heads 93 instead of 82; 4 x 300 behind 2048 shared 79 instead of 85.)
#include "attend_q4.h"
#include "attend_tile.h"

namespace griffin {

template <int DB>
struct Q4TileStage {
    using S = TileShape<DB>;
    static constexpr int W = S::NQ < 4 ? S::NQ : 4;           // words that a lane brings in
    static constexpr int PARTS = S::NQ / W;                   // ... of a token's, by as many wavefronts
    static_assert(S::KT * PARTS == Q4_TILE_WAVES, "a wavefront brings in a tile of 16 tokens, or half of it, of keys and of values");
    uint32_t at[2], at_pair[2], to[2];       // of keys, of values: the lane's place in a tile, and in a step's room
    Q4Tile tile;
    uint32_t w[2][W], pair[2];

    static __device__ __forceinline__ int tile_of(int wave) { return wave / PARTS; }

    __device__ __forceinline__ Q4TileStage(const AttendQ4Params &p, const AttendItem &, int wave, int lane)
    {
        const int part = wave % PARTS;
#pragma unroll
        for (int v = 0; v < 2; ++v) {
            const int token = v ? lane >> 2 : lane & 15, row = tile_of(wave) * 16 + token;
            const int word = v ? (part * 4 + (lane & 3)) * W : (lane >> 4) * S::NQ + part * W;
            // features from dim on meet queries that are zero, or end in outputs that are not stored: some of the row's own will do
            const int f = word * 8 < p.dim ? word * 8 : 0;
            at[v] = token * p.s.row_bytes + f / 2;
            at_pair[v] = (token * p.s.groups + (f >> p.s.group_shift)) * 4;
            to[v] = v ? row * S::ROW + (word ^ tile_turn<DB>(row) << 1) * 16 : (tile_of(wave) * S::NQ + part * W) * 1024 + lane * 16;
        }
    }

    __device__ __forceinline__ void look_up(const AttendQ4Params &p, const AttendItem &it, int32_t key0, int wave) { tile.look_up(p, it, key0 + 16 * tile_of(wave)); }

    __device__ __forceinline__ void place(const AttendQ4Params &p, const AttendItem &it, int32_t key0, int wave) { tile.set(p, it, key0 + 16 * tile_of(wave)); }

    __device__ __forceinline__ void load(const AttendQ4Params &, int, int)
    {
#pragma unroll
        for (int v = 0; v < 2; ++v) {
            const __amdgpu_buffer_rsrc_t pool = v ? tile.V : tile.K;
            if constexpr (W == 2)
                *(q4_u32x2 *)w[v] = __builtin_amdgcn_raw_buffer_load_b64(pool, at[v], tile.codes, 0);
            else
                *(att_u32x4 *)w[v] = __builtin_amdgcn_raw_buffer_load_b128(pool, at[v], tile.codes, 0);
            pair[v] = __builtin_amdgcn_raw_buffer_load_b32(pool, at_pair[v], tile.pairs, 0);
        }
    }

    // values behind the last key or in the hole, and groups of NaN, as zeros; true if there were any of these
    __device__ __forceinline__ bool clear(const AttendItem &it, int32_t key0, int wave, int lane)
    {
        const int32_t key = key0 + 16 * tile_of(wave) + (lane >> 2);
        const bool in = key < it.end && !it.missing(key), odd = q4_odd(pair[1]);
        pair[1] = in && !odd ? pair[1] : 0;
        return in && odd;
    }

    __device__ __forceinline__ void store(uint32_t keys, uint32_t vals, int, int) const
    {
#pragma unroll
        for (int v = 0; v < 2; ++v) {
            const q4_pair scale = q4_scales(pair[v]), middle = q4_middles(pair[v]);
#pragma unroll
            for (int i = 0; i < W; ++i) {
                att_u32x4 x;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    x[j] = q4_word(q4_value_pair(w[v][i] >> 4 * j, scale, middle));
                // keys: another operand, 1 KB on.  Values: the next 16 bytes, whose number's bits are below the turn's or among them
                *(lds_u32x4 *)(uintptr_t)(v ? vals + (to[v] ^ i * 16) : keys + to[v] + i * 1024) = x;
            }
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
    static constexpr int WAVES = Q4_TILE_WAVES;
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
