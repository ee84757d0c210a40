// Attention of many rows (bf16): prompts, and a prefix that more than 64 rows share.  The mathematics and the arrangement of scores
// and sums are those of attend.hip; here eight wavefronts of 32 rows each (16 of heads wider than 128) take the same keys, which go through LDS
// 64 at a time, two steps' worth of room, so that a step's loads travel while the step before is computed.
//
// Keys lie in LDS in the order of the A operands (a lane's 16 bytes side by side: reads without bank conflicts).  Values lie as in memory, a row a
// key; V^T's operand is read with ds_read_b64_tr_b16, by which 16 lanes fetch four rows' 16 features and get a feature's four keys each.  The 32-byte
// pieces of a row are exchanged by the row's number so that those rows fall into different banks.
//
// The rows' reference maximum moves only when scores outgrow it by more than 8 (base 2): weights then are up to 2^8 (their rounding to bf16 is
// relative), and o is scaled a few times instead of at every step.
#include "attend.h"

namespace griffin {

typedef __attribute__((ext_vector_type(4))) short att_s16x4;
typedef __attribute__((address_space(3))) att_s16x4 lds_s16x4;

template <int DB>
struct TileShape {
    static constexpr int NQ = DB / 32;                        // 32-feature pieces of a key
    static constexpr int NO = DB / 16;                        // tiles of 16 features of the output
    static constexpr int KT = ATT_TILE_KEYS / 16;             // tiles of 16 keys of a step
    static constexpr int NT = DB > 128 ? 1 : 2;               // tiles of 16 rows of a wavefront
    static constexpr int ROW = DB * 2;                        // bytes of a value's row
    static constexpr int BYTES = ATT_TILE_KEYS * ROW;         // of a step's keys, and of its values
    static constexpr int PIECES = BYTES / (16 * 64 * ATT_TILE_WAVES);      // 16-byte pieces of either that a thread brings in
};

template <int DB>
struct TileRows {
    using S = TileShape<DB>;
    att_u32x4 q[S::NT][S::NQ];
    int32_t end[S::NT];
    float m[S::NT], l[S::NT];
    att_f32x4 o[S::NT][S::NO];
};

// which 32-byte piece of a value's row lies in the place of piece 0: rows whose places would share banks differ in it
template <int DB>
__device__ __forceinline__ int tile_turn(int row) { return DB >= 128 ? row & 7 : (row >> 1) & 3; }

template <int DB, bool FULL>
__device__ __forceinline__ void tile_load(att_u32x4 (&k)[TileShape<DB>::PIECES], att_u32x4 (&v)[TileShape<DB>::PIECES], const AttendParams &p,
                                          const AttendItem &it, int32_t key0)
{
    using S = TileShape<DB>;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const char *Kh = (const char *)p.K + it.hk * p.head_stride * 2, *Vh = (const char *)p.V + it.hk * p.head_stride * 2;
#pragma unroll
    for (int i = 0; i < S::PIECES; ++i) {
        const int f = wave + ATT_TILE_WAVES * i, t = f / S::NQ, s = f % S::NQ;
        const AttTile tile = att_tile(p, it.pages, key0 + 16 * t, it.end);
        const int row = (lane & 15) < tile.rows ? (lane & 15) : tile.rows, d = s * 32 + (lane >> 4) * 8;
        if (FULL || d < p.dim)
            k[i] = *(const att_u32x4 *)(Kh + (tile.base + row * p.token_stride + d) * 2);
        else
            k[i] = att_u32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int i = 0; i < S::PIECES; ++i) {
        const int first = (wave * 64 + 64 * ATT_TILE_WAVES * i) / (DB / 8), row = first + lane / (DB / 8), d = lane % (DB / 8) * 8;
        const AttTile tile = att_tile(p, it.pages, key0 + (first & ~15), it.end);
        const int at = (row & 15) < tile.rows ? (row & 15) : tile.rows;
        v[i] = *(const att_u32x4 *)(Vh + (tile.base + at * p.token_stride + (FULL || d < p.dim ? d : 0)) * 2);
    }
}

template <int DB>
__device__ __forceinline__ void tile_store(char *lds, const att_u32x4 (&k)[TileShape<DB>::PIECES], const att_u32x4 (&v)[TileShape<DB>::PIECES])
{
    using S = TileShape<DB>;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int i = 0; i < S::PIECES; ++i) {
        *(att_u32x4 *)(lds + (wave + ATT_TILE_WAVES * i) * 1024 + lane * 16) = k[i];
        const int row = (wave * 64 + 64 * ATT_TILE_WAVES * i) / (DB / 8) + lane / (DB / 8), piece = lane % (DB / 8);
        *(att_u32x4 *)(lds + S::BYTES + row * S::ROW + (piece ^ tile_turn<DB>(row) << 1) * 16) = v[i];
    }
}

// A operand of V^T: features 16 e .. + 15 of the keys of tiles 2h and 2h + 1, in the order in which the lanes hold their scores
template <int DB>
__device__ __forceinline__ att_u32x4 tile_vals(const char *vals, int e, int h)
{
    using S = TileShape<DB>;
    const int lane = threadIdx.x & 63, row = (lane >> 4) * 4 + ((lane >> 2) & 3);
    const char *at = vals + row * S::ROW + (e ^ tile_turn<DB>(row)) * 32 + (lane & 3) * 8;
    typedef __attribute__((ext_vector_type(2))) uint32_t pair_t;
    const pair_t lo = __builtin_bit_cast(pair_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(at + 2 * h * 16 * S::ROW)));
    const pair_t hi = __builtin_bit_cast(pair_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(at + (2 * h + 1) * 16 * S::ROW)));
    return att_u32x4{lo.x, lo.y, hi.x, hi.y};
}

__device__ __forceinline__ att_f32x4 att_mfma(att_u32x4 a, att_u32x4 b, att_f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(att_bf16x8, a), __builtin_bit_cast(att_bf16x8, b), c, 0, 0, 0);
}

// A step in which rows differ in the keys that they see, or in which keys end: infinite and NaN values of keys that a row does not see must not
// reach it, as 0 x Inf would.  A product of all values with zeros is NaN if there are any.  If so, they are counted per row that sees them and by sign
// in a product of ones, the sums they are in become infinite or NaN, and `true` says that the product to come has to take them as zeros.
template <int DB>
__device__ __forceinline__ bool tile_take_infinite(const char *vals, TileRows<DB> &r, int32_t key0)
{
    using S = TileShape<DB>;
    const att_u32x4 zero = {0, 0, 0, 0};
    att_f32x4 sum = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < S::NO; ++e)
#pragma unroll
        for (int h = 0; h < S::KT / 2; ++h)
            sum = att_mfma(tile_vals<DB>(vals, e, h), zero, sum);
    if (!__any(sum[0] != sum[0] || sum[1] != sum[1] || sum[2] != sum[2] || sum[3] != sum[3]))
        return false;
    const int lane = threadIdx.x & 63;
    for (int minus = 0; minus < 2; ++minus)
#pragma unroll
        for (int e = 0; e < S::NO; ++e)
#pragma unroll
            for (int n = 0; n < S::NT; ++n) {
                __builtin_amdgcn_sched_barrier(0);            // one at a time: this is not where registers are to go
                att_f32x4 count = {0, 0, 0, 0};
                for (int h = 0; h < S::KT / 2; ++h) {
                    att_u32x4 a = tile_vals<DB>(vals, e, h), seen;
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        a[w] = att_infinite<true>(a[w], minus);
                        const int32_t key = key0 + h * 32 + (w >> 1) * 16 + (lane >> 4) * 4 + (w & 1) * 2;
                        seen[w] = (key < r.end[n] ? 0x3F80u : 0) | (key + 1 < r.end[n] ? 0x3F800000u : 0);
                    }
                    count = att_mfma(a, seen, count);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    r.o[n][e][i] += count[i] > 0 ? (minus ? -INFINITY : INFINITY) : 0.0f;
            }
    return true;
}

template <int DB, bool CLEAN>
__device__ __forceinline__ void tile_weigh(const char *vals, const att_u32x4 (&w)[TileShape<DB>::NT][TileShape<DB>::KT / 2], TileRows<DB> &r)
{
    using S = TileShape<DB>;
#pragma unroll
    for (int e = 0; e < S::NO; ++e)
#pragma unroll
        for (int h = 0; h < S::KT / 2; ++h) {
            att_u32x4 a = tile_vals<DB>(vals, e, h);
            if (CLEAN)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    a[i] = att_finite_or_0<true>(a[i]);
#pragma unroll
            for (int n = 0; n < S::NT; ++n)
                r.o[n][e] = att_mfma(a, w[n][h], r.o[n][e]);
        }
}

// Keys key0 .. key0 + 63, in LDS, for the wavefront's rows.  MASKED: some rows do not see some of them.
template <int DB, bool MASKED>
__device__ __forceinline__ void tile_step(const char *lds, TileRows<DB> &r, float scale2, int32_t key0)
{
    using S = TileShape<DB>;
    const int lane = threadIdx.x & 63;
    att_f32x4 s[S::NT][S::KT];
#pragma unroll
    for (int t = 0; t < S::KT; ++t) {
#pragma unroll
        for (int n = 0; n < S::NT; ++n)
            s[n][t] = att_f32x4{0, 0, 0, 0};
#pragma unroll
        for (int c = 0; c < S::NQ; ++c) {
            const att_u32x4 a = *(const att_u32x4 *)(lds + (t * S::NQ + c) * 1024 + lane * 16);
#pragma unroll
            for (int n = 0; n < S::NT; ++n)
                s[n][t] = att_mfma(a, r.q[n][c], s[n][t]);
        }
    }
    float top[S::NT];
    bool grown = false;
#pragma unroll
    for (int n = 0; n < S::NT; ++n) {
        top[n] = -INFINITY;
#pragma unroll
        for (int t = 0; t < S::KT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (MASKED && key0 + 16 * t + (lane >> 4) * 4 + e >= r.end[n])
                    s[n][t][e] = -INFINITY;
                top[n] = fmaxf(top[n], s[n][t][e]);
            }
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
    att_u32x4 w[S::NT][S::KT / 2];
#pragma unroll
    for (int n = 0; n < S::NT; ++n) {
        const float base = r.m[n] == -INFINITY ? 0.0f : r.m[n];
        float l[S::KT];
#pragma unroll
        for (int t = 0; t < S::KT; ++t) {
            float x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
                x[e] = __builtin_amdgcn_exp2f(s[n][t][e] * scale2 - base);
            l[t] = (x[0] + x[1]) + (x[2] + x[3]);
            w[n][t / 2][t % 2 * 2] = f32x2_to_bf16x2(x[0], x[1]);
            w[n][t / 2][t % 2 * 2 + 1] = f32x2_to_bf16x2(x[2], x[3]);
        }
        r.l[n] += (l[0] + l[1]) + (l[2] + l[3]);
    }
    if (MASKED && tile_take_infinite<DB>(lds + S::BYTES, r, key0))
        tile_weigh<DB, true>(lds + S::BYTES, w, r);
    else
        tile_weigh<DB, false>(lds + S::BYTES, w, r);
}

template <int DB, bool FULL>
__global__ __launch_bounds__(64 * ATT_TILE_WAVES) void attend_tile_kernel(AttendParams p)
{
    using S = TileShape<DB>;
    extern __shared__ __align__(16) char tile_lds[];          // two steps of keys and values
    AttendItem it;
    if (!att_item<att_tile_rows(DB), att_tile_rows(DB), true>(p, blockIdx.x, it))
        return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    TileRows<DB> r;
    int32_t token[S::NT], head[S::NT], least = it.end, most = it.begin;       // keys that all rows of the wavefront see, and that any sees
    const int32_t first = it.first + wave * 16 * S::NT;
#pragma unroll
    for (int n = 0; n < S::NT; ++n) {
        int32_t row = first + 16 * n + (lane & 15);
        const bool in = row < it.rows;                        // rows behind the last repeat it and are not stored
        row = in ? row : it.rows - 1;
        token[n] = it.token0 + row / p.group;
        head[n] = it.hk * p.group + row % p.group;
        r.end[n] = it.own < 0 || it.own + row / p.group + 1 > it.end ? it.end : it.own + row / p.group + 1;
        least = r.end[n] < least ? r.end[n] : least;
        most = in && r.end[n] > most ? r.end[n] : most;
        const char *at = (const char *)p.q + ((int64_t)token[n] * p.ldq + (int64_t)head[n] * p.hsq) * 2 + (lane >> 4) * 16;
#pragma unroll
        for (int s = 0; s < S::NQ; ++s) {
            if (FULL || s * 32 + (lane >> 4) * 8 < p.dim)
                r.q[n][s] = *(const att_u32x4 *)(at + s * 64);
            else
                r.q[n][s] = att_u32x4{0, 0, 0, 0};
        }
        r.m[n] = -INFINITY;
        r.l[n] = 0;
#pragma unroll
        for (int e = 0; e < S::NO; ++e)
            r.o[n][e] = att_f32x4{0, 0, 0, 0};
    }
    att_u32x4 k[S::PIECES], v[S::PIECES];
    tile_load<DB, FULL>(k, v, p, it, it.begin);
    tile_store<DB>(tile_lds, k, v);
    __syncthreads();
    int room = 0;
    for (int32_t key0 = it.begin; key0 < it.end; key0 += ATT_TILE_KEYS) {
        const bool more = key0 + ATT_TILE_KEYS < it.end;
        if (more)
            tile_load<DB, FULL>(k, v, p, it, key0 + ATT_TILE_KEYS);
        if (__any(key0 < most) && __all(key0 + ATT_TILE_KEYS <= least))
            tile_step<DB, false>(tile_lds + room * 2 * S::BYTES, r, p.scale2, key0);
        else if (__any(key0 < most))
            tile_step<DB, true>(tile_lds + room * 2 * S::BYTES, r, p.scale2, key0);
        room ^= 1;
        if (more)
            tile_store<DB>(tile_lds + room * 2 * S::BYTES, k, v);
        __syncthreads();
    }
#pragma unroll
    for (int n = 0; n < S::NT; ++n) {
        const float l = lane_groups_sum(r.l[n]);
        if (first + 16 * n + (lane & 15) >= it.rows)
            continue;
        const int64_t slot = ((int64_t)token[n] * p.n_heads + head[n]) * (p.chunks_prefix + p.chunks_own) + it.split;
        const float f = p.part ? 1.0f : (l == 0.0f ? 0.0f : 1.0f / l);        // a row without keys: zeros
        if (p.part && lane < 16)
            p.part_ml[slot] = make_float2(r.m[n], l);
#pragma unroll
        for (int e = 0; e < S::NO; ++e) {
            const int d = e * 16 + (lane >> 4) * 4;
            if (!FULL && d >= p.dim)
                continue;
            const att_f32x4 x = r.o[n][e] * f;
            if (p.part)
                *(att_f32x4 *)(p.part + slot * p.dim + d) = x;
            else
                *(uint2 *)((uint16_t *)p.out + (int64_t)token[n] * p.ldo + (int64_t)head[n] * p.hso + d) =
                    make_uint2(f32x2_to_bf16x2(x[0], x[1]), f32x2_to_bf16x2(x[2], x[3]));
        }
    }
}

template <int DB>
static int go_tiles(const AttendParams &p, int32_t wgs, hipStream_t st)
{
    constexpr int bytes = 4 * TileShape<DB>::BYTES;
    if (p.dim == DB) {
        RAISE_LDS_LIMIT((attend_tile_kernel<DB, true>), bytes);
        hipLaunchKernelGGL((attend_tile_kernel<DB, true>), dim3(wgs), dim3(64 * ATT_TILE_WAVES), bytes, st, p);
    } else {
        RAISE_LDS_LIMIT((attend_tile_kernel<DB, false>), bytes);
        hipLaunchKernelGGL((attend_tile_kernel<DB, false>), dim3(wgs), dim3(64 * ATT_TILE_WAVES), bytes, st, p);
    }
    return check_launch("attend_tile_kernel");
}

int launch_attend_tiles(const AttendParams &p, int32_t wgs, hipStream_t st)
{
    if (p.dim <= 64)
        return go_tiles<64>(p, wgs, st);
    return p.dim <= 128 ? go_tiles<128>(p, wgs, st) : go_tiles<256>(p, wgs, st);
}

}  // namespace griffin
