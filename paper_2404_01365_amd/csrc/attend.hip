// Attention of a step's new tokens over the prefix that all sequences share and over each sequence's own pages
// (griffin_attention): o = sum_k softmax_k(scale q.k) v_k.
//
// One pass over the keys with the running maximum m and sum l of the softmax: a step forms the scores of a few keys, takes
// m' = max(m, scores), scales o and l by 2^(m - m') and adds the step's weights and weighted values (exponents to base 2, the factor
// log2(e) goes into the scale).  A row is a token and a head; the rows of all heads that share a kv head go together, and in the prefix those of all
// sequences, so that keys and values are read once for 16 to 256 rows.
//
// A few rows take their keys straight from memory (attend_rows.h), many through LDS (attend_tile.hip).
//
// Long key ranges are cut into chunks for as many workgroups as fill the chip; each leaves its rows' o, m and l, and a second kernel joins them.
//
// Bound by bytes while few rows share a key, with the latency of a step's loads on top: a part that one step covers is two launches' latency, 4.5 us of it the join's.
// Measured: 64 continuations of 1024 shared tokens and 1 to 120 of their own, 40 heads of 128, 102 MB, 32 us warm = 3.2 TB/s, caches cold 57 us = 1.8; 8 sequences behind 30000 shared
// keys of 8 heads of 128, four query heads each, 125 MB, 31 us = 4.0 TB/s, cold 64 = 2.0; one row of 513 keys of 32 heads 8.3 us and the join.
// The products of 16 rows a key are a twentieth of the matrix cores' rate when keys arrive at a copy's, of 64 rows a quarter: the arrangement is made for loads.
#include <algorithm>

#include "attend_rows.h"

namespace griffin {

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
    bool beside;                        // ... in the launch of the prefix's tiles
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
    // 46 / 62; one sequence of 64 rows 16.6 / 14.2.)  So does a prefix beside them, in their launch (2 x 100 tokens of 32 heads on 8 behind 300 shared 23 / 35, behind 2048 31 / 51; 5 x 1 and
    // 33 tokens 15 / 22, 19 / 27), and one of more rows than that where there is enough to multiply: its workgroups are fewer and larger.  (8 kv heads of 128, us there / here: 80 rows of 8192 keys 24.4 / 21.2, of 32768 40.0 / 43.0; 192 rows of 2048 keys 28 / 18, of 8192 34.8 / 31.4, of 32768
    // 55 / 81; 448 rows of 2048 keys 34 / 26, of 8192 43 / 54.)
    pl.tile_own = bf16 && longest > 64;
    pl.tile_prefix = bf16 && (pl.tile_own || (rows > 64 && (double)rows * B.n_prefix * C.kv_heads * C.dim >= 0x1p31));
    // Own parts of a few rows go in the launch of those tiles, if the tiles' share of registers is enough for them.  (In a launch of their own, 48 of 5 to 700 keys
    // behind 32768: 74 us, not 67; 20 of 50: 43, not 40.)
    pl.beside = pl.tile_prefix && !pl.tile_own && C.dim <= 128;
    // Where a wavefront has the registers it takes two tiles of 16 rows, and so reads keys half as often.  (Own parts, two / one: 16 of 48 rows and 2000 keys 35 / 57 us, 16
    // of 64 rows and 1000 keys 26.8 / 25.6, one of 64 rows and 4000 keys 17.6 / 14.4; up to 32 rows the same.  A prefix: 64 rows of 30000 keys 34 / 47, 48 of 16384 23 / 28, 64
    // of 2048 12.7 / 14.0, 80 of 2048 15.1 / 13.6.)
    pl.nto = longest <= 32 || pl.beside ? 1 : widest;
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
    // keys 23 / 30 / 32, 32 rows of 30000 31 / 35 / 41; fewer, 256: 3 % slower to 7 % faster.  Tiles, 256 / 512: 192 rows of 32768 keys 71 / 85, a prompt of 2048 63 / 70;
    // heads of 256, 256 / 512: 15.7 / 18.4.)  Own parts behind tiles of the prefix are cut finer: the longest is known here, most are shorter
    // (48 of 5 to 700 keys, 512 / 1024 / 2048 workgroups of four wavefronts' keys: 68 / 73 / 67 us).  Own parts of many rows are one chunk if they fill the chip.
    const int64_t step = ATT_WAVES * (bf16 ? 32 : 16);
    const int64_t work_prefix = C.kv_heads * (int64_t)pl.tiles_prefix * B.n_prefix, work_own = C.kv_heads * tiles * B.max_len;
    const auto chunk = [&](bool tile, int64_t work, int32_t keys) {        // no longer than the part: up to 2^30 keys and a quantum
        const int64_t quantum = tile ? tile_keys : pl.beside ? ATT_FEW_WAVES / ATT_WAVES * step : step, wgs = tile || pl.lone || C.dim > 128 ? 256 : 512;
        const int64_t even = std::min((work + wgs - 1) / wgs, (int64_t)keys);
        return (int32_t)((std::max(even, (int64_t)1) + quantum - 1) / quantum * quantum);
    };
    const bool together = pl.tile_prefix == pl.tile_own && !pl.lone;
    pl.chunk_prefix = chunk(pl.tile_prefix, together ? work_prefix + work_own : work_prefix, B.n_prefix);
    pl.chunk_own = chunk(pl.tile_own, together ? work_prefix + work_own : pl.lone ? work_own : work_own / 4, B.max_len);
    if (pl.lone || (pl.tile_own && C.kv_heads * tiles > 128))
        pl.chunk_own = (int32_t)((B.max_len + step - 1) / step * step);
    // (Own parts of many rows, whole / cut so that 256 workgroups share them: 3000 tokens of 16 heads, 192 tiles of rows, 95 / 113 us; 1000 of 40 heads on 8, 160
    // tiles, 42 / 61; 2048 of 16 on 8, 128 tiles, 71 / 63.  Behind own tokens in the cache: 1100 of 32 on 8 behind 1000 73 / 106, behind 30000 898 / 1043;
    // three times 400 behind 8000, 8000 and 0 251 / 216.)
    // Own items take the prefix ahead of their own keys where that costs less than to join two parts: parts so few and short that a step of twice as many
    // wavefronts is cheaper than a second launch (some 5 us), prefix or not, and own tiles that fill the chip (their rows' sums would go through memory in fp32),
    // unless the prefix is read much oftener for it: tiles of a sequence's rows are not full, those of the prefix are.  With three of four tiles' rows there it pays
    // whatever the prefix, else up to 16384 keys more in all.  (Prefix ahead / joined, 32 heads on 8.  3400 tokens behind 300, 2048, 8192 and 32768: 131 / 193, 224 /
    // 277, 578 / 601, 1996 / 1975; four times 300 behind 32768: 970 / 1168.  20 times 20 behind 300, 1024, 2048, 32768: 18 / 32, 33 / 41, 55 / 47, 698 / 295; 47 times a
    // token and one of 17 tokens behind 64, 300, 1024, 32768: 37 / 39, 48 / 40, 75 / 45, 1366 / 84.  64 heads on 8, 17 times 9 behind 300, 1024, 8192: 19 / 28, 33 / 32, 181 /
    // 71.)
    // At two steps one launch is no longer cheaper: 513 keys of 32 heads of 128 take 10.4 us in one launch of 32 workgroups, 10.3 cut into chunks and joined (caches
    // cold: 15.9, 14.4).
    const int64_t all = (int64_t)B.n_prefix + B.max_len, items = C.kv_heads * tiles;
    pl.few = longest <= 32 && !pl.tile_prefix && items <= 512 && all <= ATT_FEW_WAVES / ATT_WAVES * step && C.dim <= 128;
    const int64_t beyond = tiles - (rows + pl.rows_own - 1) / pl.rows_own;      // tiles more than all rows in a row would take
    pl.ahead = B.n_prefix > 0 && (pl.few || (pl.tile_own && items > 128 && (4 * beyond <= tiles || beyond * B.n_prefix <= 16384)));
    if (pl.ahead)
        pl.tiles_prefix = 0;
    if (pl.ahead || pl.few)
        pl.chunk_own = (int32_t)((all + 15 + step - 1) / step * step);
    pl.chunks_prefix = pl.ahead ? 0 : (B.n_prefix + pl.chunk_prefix - 1) / pl.chunk_prefix;
    pl.chunks_own = pl.ahead ? 1 : (B.max_len + pl.chunk_own - 1) / pl.chunk_own;
    return pl;
}

// Rows that are planned for: a launch holds fewer than 2^32 threads, and quotients are exact while dividend times divisor is below 2^32.  With at most 2^30 keys the
// plan's products then stay below 2^52.
static bool attend_takes(const SeqTable &seqs, int32_t n_heads)
{
    const int64_t rows = (int64_t)seqs.cu[seqs.n] * n_heads;
    return rows < 1 << 24 && rows * n_heads < (int64_t)1 << 32;
}

size_t attend_floats(const griffin_kv_cache &C, const griffin_kv_batch &B, const SeqTable &seqs, int32_t n_heads)
{
    if (!attend_takes(seqs, n_heads))
        return 0;
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
            p.wgs_prefix = wgs_prefix;
            p.items_own = pl.beside ? wgs_own : 0;
            rc = launch_attend_tiles(p, tiled, pl.beside && pl.lone, st);
        }
    if (rc == GRIFFIN_OK && others > 0 && !pl.beside) {
        p.wgs_prefix = pl.tile_prefix ? 0 : wgs_prefix;
        p.items_own = wgs_own;
        const int ntp = p.wgs_prefix > 0 ? pl.ntp : 1, nto = pl.nto;
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
    if (!attend_takes(seqs, job.n_heads))
        return GRIFFIN_EUNSUPPORTED;
    const AttPlan pl = attend_plan(C, B, seqs, job.n_heads);
    const int64_t wgs = (int64_t)C.kv_heads * ((int64_t)pl.tiles_prefix * pl.chunks_prefix + (int64_t)pl.tiles_own * pl.chunks_own), limit = (int64_t)1 << 32;
    if (wgs >= 1 << 23 || wgs * C.kv_heads >= limit || wgs * std::max(pl.chunks_prefix, pl.chunks_own) >= limit)
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
