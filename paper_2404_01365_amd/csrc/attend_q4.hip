// Attention over a cache in 4 bits (griffin_attention_q4): a few rows straight from memory (attend_q4.h), many through LDS (attend_q4_tile.hip).
#include <algorithm>

#include "attend_q4.h"

namespace griffin {

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
    const bool bf16 = C.dtype == GRIFFIN_BF16;
    const int widest = q4_widest(C);                       // tiles of 16 rows that the registers hold
    const int32_t group = n_heads / C.kv_heads;
    const int64_t rows = (int64_t)seqs.cu[seqs.n] * group;
    int64_t longest = 0;
    for (int b = 0; b < seqs.n; ++b)
        longest = std::max(longest, (int64_t)(seqs.cu[b + 1] - seqs.cu[b]) * group);
    pl.tile_own = bf16 && longest > 64;
    pl.tile_prefix = bf16 && (pl.tile_own || (rows > 64 && (double)rows * B.n_prefix * C.kv_heads * C.dim >= 0x1p31));
    pl.beside = pl.tile_prefix && !pl.tile_own && C.dim <= 128;
    pl.nto = longest <= 16 || pl.beside ? 1 : widest;
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
    pl.lone = !pl.tile_own && C.kv_heads * tiles >= 1024 && B.max_len <= 256;
    const int64_t step = ATT_WAVES * 32;
    const int64_t work_prefix = C.kv_heads * (int64_t)pl.tiles_prefix * B.n_prefix, work_own = C.kv_heads * tiles * B.max_len;
    const auto chunk = [&](bool tile, int64_t work, int32_t keys, int64_t wgs) {   // no longer than the part: up to 2^30 keys and a quantum
        const int64_t quantum = tile ? att_tile_keys(C.dim) : pl.beside ? ATT_FEW_WAVES / ATT_WAVES * step : step;
        const int64_t even = std::min((work + wgs - 1) / wgs, (int64_t)keys);
        return (int32_t)((std::max(even, (int64_t)1) + quantum - 1) / quantum * quantum);
    };
    const bool together = pl.tile_prefix == pl.tile_own && !pl.lone;
    const int64_t wgs_rows = C.dim > 128 ? 512 : 512;
    pl.chunk_prefix = chunk(pl.tile_prefix, together && pl.tile_own ? work_prefix + work_own : work_prefix, B.n_prefix, pl.tile_prefix ? 256 : 512);
    pl.chunk_own = chunk(pl.tile_own, together && pl.tile_own ? work_prefix + work_own : work_own, B.max_len, pl.tile_own ? 256 : pl.beside ? 1024 : wgs_rows);
    if (pl.lone || (pl.tile_own && C.kv_heads * tiles > 128))
        pl.chunk_own = (int32_t)((B.max_len + step - 1) / step * step);
    const int64_t all = (int64_t)B.n_prefix + B.max_len, items = C.kv_heads * tiles;
    pl.few = longest <= 16 && !pl.tile_prefix && items <= 512 && all <= ATT_FEW_WAVES / ATT_WAVES * step && C.dim <= 128;
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
    int rc = GRIFFIN_OK;
    const int32_t wgs_prefix = p.kv_heads * pl.tiles_prefix * pl.chunks_prefix, wgs_own = p.kv_heads * pl.tiles_own * pl.chunks_own;
    const int32_t tiled = (pl.tile_prefix ? wgs_prefix : 0) + (pl.tile_own ? wgs_own : 0), others = wgs_prefix + wgs_own - tiled;
    if constexpr (!F32)
        if (tiled > 0) {
            p.wgs_prefix = wgs_prefix;
            p.items_own = pl.beside ? wgs_own : 0;
            rc = launch_attend_q4_tiles(p, tiled, pl.beside && pl.lone, st);
        }
    if (rc == GRIFFIN_OK && others > 0 && !pl.beside) {
        p.wgs_prefix = pl.tile_prefix ? 0 : wgs_prefix;
        p.items_own = wgs_own;
        if constexpr (DB <= 128)
            if (pl.few) {
                constexpr int bytes = att_lds_floats<DB, ATT_FEW_WAVES>() * sizeof(float);
                RAISE_LDS_LIMIT((attend_q4_few_kernel<F32, DB>), bytes);
                hipLaunchKernelGGL((attend_q4_few_kernel<F32, DB>), dim3(p.items_own), dim3(ATT_FEW_WAVES * 64), bytes, st, p);
                return check_launch("attend_q4_few_kernel");
            }
        const int ntp = p.wgs_prefix > 0 ? pl.ntp : 1, nto = pl.nto;
        if constexpr (DB <= 64 || (DB <= 128 && !F32)) {
            if (nto == 2)
                rc = go_rows<F32, DB, 2, 2>(p, pl.lone, st);
            else if (ntp == 2)
                rc = go_rows<F32, DB, 2, 1>(p, pl.lone, st);
            else
                rc = go_rows<F32, DB, 1, 1>(p, pl.lone, st);
        } else
            rc = go_rows<F32, DB, 1, 1>(p, pl.lone, st);
    }
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
