// Attention over a cache in 4 bits (griffin_attention_q4): a few rows straight from memory (attend_q4.h), many through LDS (attend_q4_tile.hip).
#include <algorithm>

#include "attend_join.h"
#include "attend_q4.h"

namespace griffin {

// LONE: own items go a wavefront each
template <bool F32, int DB, int NTP, int NTO, bool LONE>
__global__ __launch_bounds__(ATT_WAVES * 64, DB > 128 && F32 ? 1 : 2) void attend_q4_kernel(AttendQ4Params p)
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
    if (LONE ? att_own_item<16 * NTO, false>(p, id, it) : q4_own_item<16 * NTO>(p, id, it))
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

// where the join finds a row's chunks
__device__ __forceinline__ AttParts att_parts(const AttendQ4Params &p, int32_t row, int32_t token, int32_t head)
{
    if (p.deal < 0)
        return att_parts((const AttendParams &)p, row, token, head);
    const int b = att_sequence(token, p.each, p.seqs.cu, p.seqs.n);
    const int32_t first = p.seqs.cu[b], held = p.lens[b] < 0 ? 0 : (p.lens[b] < p.max_len ? p.lens[b] : p.max_len);
    const int32_t seen = held + token - first + 1 < p.max_len ? held + token - first + 1 : p.max_len;
    const int4 cut = p.cuts[b];
    if (p.chunks_prefix == 0 && cut.y == 1)                // the part's own workgroup has left the output
        return {0, 0, 0, 0, 0};
    const int32_t hk = p.by_group(head), in = (token - first) * p.group + head - hk * p.group, tile = in / p.rows_own;
    const int64_t slot = ((int64_t)(cut.x + tile * cut.y) * p.kv_heads + hk) * p.rows_own + in - tile * p.rows_own;
    return {(int64_t)row * p.chunks_prefix, p.slots_own + slot, p.chunks_prefix, (seen + cut.z - 1) / cut.z, p.kv_heads * p.rows_own};
}

// ------------------------------------------------------------------ host side
struct Q4Plan : AttPlan {
    int32_t deal;                       // as in AttendQ4Params
    int64_t parts;                      // own parts of a kv head at most, where the device cuts them
    int32_t quantum;
    int64_t slots_own;                  // slots before theirs
    size_t floats;                      // of workspace
};

// All rules go by sizes alone; figures are for 8 kv heads of 128 and four query heads each unless they say otherwise, us a call.
static Q4Plan attend_q4_plan(const griffin_kv_cache_q4 &C, const griffin_kv_batch &B, const SeqTable &seqs, int32_t n_heads)
{
    Q4Plan pl = {};
    const bool bf16 = C.dtype == GRIFFIN_BF16;
    const int widest = C.dim > 128 || (!bf16 && C.dim > 64) ? 1 : 2;         // tiles of 16 rows that the registers hold
    const int32_t group = n_heads / C.kv_heads;
    const int64_t rows = (int64_t)seqs.cu[seqs.n] * group;
    int64_t longest = 0;
    for (int b = 0; b < seqs.n; ++b)
        longest = std::max(longest, (int64_t)(seqs.cu[b + 1] - seqs.cu[b]) * group);
    // Own parts of more than 64 rows go through LDS, 128 rows a workgroup.  (16 sequences of 200 to 2000 keys, there / here: 48 rows each 34 / 32, 80 rows 37 / 39, 128 rows 42 / 43, 192 rows 60 / 58,
    // two of 3000 to 4000 keys and 64 to 192 rows the same within 6 %; 20 times 80 rows behind 300 shared keys, which they then take ahead of their own, 18 / 32.)  So does a
    // prefix of more rows than that where there is enough to multiply.  (80 rows of 16384 keys 31 / 28, of 32768 37 / 46; 128 rows of 4096 28 / 18, of 16384 34 / 31, of 32768 44 / 44; 192 of 8192 32 / 34,
    // of 16384 40 / 54; 320 rows of 1024 26 / 22, of 4096 30 / 32, of 8192 38 / 49.)
    pl.tile_own = bf16 && longest > 64;
    pl.tile_prefix = bf16 && (pl.tile_own || (rows > 64 && (double)rows * B.n_prefix * C.kv_heads * C.dim > 0x1p31));
    pl.beside = pl.tile_prefix && !pl.tile_own && C.dim <= 128;
    // A wavefront takes two tiles of 16 rows where it has the registers and the rows: codes are unpacked once for both.  (Own parts, two / one: 16 of 20 rows and 500 to 4000
    // keys 26 / 32, 32 of 32 rows and 100 to 1000 keys 24.3 / 24.9; two of 48 rows and 4000 keys 18.9 / 17.6.)
    pl.nto = longest <= 16 || pl.beside ? 1 : widest;
    pl.ntp = rows <= 16 ? 1 : widest;
    if (!pl.tile_own && !pl.tile_prefix && pl.nto == widest)        // compiled pairs: (1, 1), (2, 1), (2, 2)
        pl.ntp = widest;
    pl.rows_own = pl.tile_own ? q4_tile_rows(C.dim) : 16 * pl.nto;
    pl.rows_prefix = pl.tile_prefix ? q4_tile_rows(C.dim) : 16 * pl.ntp;
    int64_t tiles = 0;
    for (int b = 0; b < seqs.n; ++b)
        tiles += ((int64_t)(seqs.cu[b + 1] - seqs.cu[b]) * group + pl.rows_own - 1) / pl.rows_own;
    pl.tiles_own = (int32_t)tiles;
    pl.tiles_prefix = B.n_prefix > 0 ? (int32_t)((rows + pl.rows_prefix - 1) / pl.rows_prefix) : 0;
    const int64_t step = ATT_WAVES * 32, all = (int64_t)B.n_prefix + B.max_len, items = C.kv_heads * tiles;
    // Own parts that fill the chip as they are go a wavefront each, and parts so few and short that a step of twice as many wavefronts is cheaper than a second launch take the
    // prefix, too, all in one launch: rules of the 16-bit cache (attend.hip), whose parts are as many steps long.  (A wavefront each / cut by the device, 32 kv heads of 128: 100 of 5 to 120 keys 17 / 25,
    // 40 of 5 to 250 16.6 / 19.2, 128 of 100 to 255 36 / 49, 200 of 5 to 60 behind 1000 42 / 77; 200 of 5 to 250, 8 heads of 64, 13.5 / 19.5.  One launch / not: one of 250 keys 8.0 / 11.8, 16 of three tokens
    // behind 200 8.5 / 12.6, 64 of 10 to 250 12.3 / 12.2, 16 of them of 32 kv heads 12.1 / 11.6.  Both end earlier than they could: 100 of 200 to 500 a wavefront each 45 / 54, one of 500 in one launch 9.5 / 11.9, but 64
    // of 260 to 500 16.2 / 15.0.)
    pl.lone = !pl.tile_own && items >= 1024 && B.max_len <= 256;
    pl.few = longest <= 16 && !pl.tile_prefix && items <= 512 && all <= ATT_FEW_WAVES / ATT_WAVES * step && C.dim <= 128;
    const int64_t work_prefix = C.kv_heads * (int64_t)pl.tiles_prefix * B.n_prefix;
    const auto chunk = [&](int64_t quantum, int64_t work, int32_t keys) {    // for 256 workgroups; no longer than the part: up to 2^30 keys and a quantum
        const int64_t even = std::min((work + 255) / 256, (int64_t)keys);
        return (int32_t)((std::max(even, (int64_t)1) + quantum - 1) / quantum * quantum);
    };
    // Tiles' chunks, the least for which no more than 512 workgroups a round share the prefix and, of tiles, own parts: two a CU.  (One round, 320 rows of 32768 keys, 256 / 384 /
    // 512 / 768 workgroups: 92 / 84 / 75 / 83; 192 rows of them 64 / 63 / 65 / 67; 200 behind 8000 own, 384 / 512 / 1024, 67 / 54 / 65.)  Several rounds of shorter chunks where one would be far
    // from full: a round takes some 1.9 us for 64 keys of 128 features, a chunk's sums go out and in again at some 4 TB/s.
    // (One round / several: 800 tokens on 30000 own keys 539 / 440, 1100 on them 1018 / 705, 700 and 1100 behind 30000 shared 749 / 397, 1027 / 607, 16 heads of 256 on 8, 700 on 16000, 414 / 344.)
    // A round that is begun for no more than one workgroup a CU takes 0.65 of a full one's time, and fewer rounds than a chunk a tile takes there cannot be.  (Beyond 512 tiles, whole / in more rounds:
    // 2100, 2500 and 3000 tokens on 30000 own keys, 528 to 752 tiles, 1714 / 1283, 1725 / 1435, 1759 / 1763, on 16000 926 / 742, 945 / 844, 985 / 1033, on 4000 268 / 314, 291 / 336, 352 / 416, 880 tiles on
    // 120000 9078 / 7854; 4100 and 5000 tokens on 30000, 1032 and 1256 tiles, 3004 / 2704, 2913 / 3102.)  More than 512 tiles of a prefix and of own parts together stay whole: the model, which takes all
    // for as long as the longest, does not tell them apart.  (Whole / cut: 64 of 40 tokens behind 2000 and 32768 shared 171 / 165, 1857 / 1527, 200 of 17 behind 8000 623 / 677, 256 of 20 behind 3000 390 / 444.)
    constexpr double STEP = 1.9 / (64 * 128);
    const auto rounds_of = [](int64_t wgs) { return wgs <= 512 ? 1.0 : (double)(wgs / 512) + (wgs % 512 > 256 ? 1.0 : wgs % 512 > 0 ? 0.65 : 0.0); };
    double least = 0;                                      // us, of the chunks that were chosen
    const auto tile_chunk = [&]() {
        const int64_t quantum = att_tile_keys(C.dim), heads = C.kv_heads, own = pl.tile_own ? tiles : 0;
        const int64_t most = (std::max((int64_t)B.n_prefix, own > 0 ? (int64_t)B.max_len : 0) + quantum - 1) / quantum;
        const int64_t all_tiles = heads * (pl.tiles_prefix + own), first = std::max((all_tiles + 511) / 512, (int64_t)1);
        int64_t best = most;
        least = 0;
        if (all_tiles > 512 && pl.tiles_prefix > 0 && own > 0)
            return (int32_t)(most * quantum);
        for (int64_t rounds = first; rounds < first + 8; ++rounds) {
            int64_t lo = 1, hi = most;
            while (lo < hi) {
                const int64_t mid = (lo + hi) / 2, keys = mid * quantum;
                if (heads * (pl.tiles_prefix * ((B.n_prefix + keys - 1) / keys) + own * ((B.max_len + keys - 1) / keys)) <= 512 * rounds) hi = mid;
                else lo = mid + 1;
            }
            const double taken = lo == most ? rounds_of(all_tiles) : (double)rounds;
            const double cost = taken * (lo * quantum) * C.dim * STEP + (double)rows * heads * ((most + lo - 1) / lo) * (C.dim + 2) * 2e-6;
            if (rounds == first || cost < 0.9 * least) {
                best = lo;
                least = cost;
            }
        }
        return (int32_t)(best * quantum);
    };
    // The prefix: a workgroup a CU, two steps each at least of heads wider than 128.  (128 / 256 / 512 workgroups: 32 rows of 16384 keys 21 / 17 / 22, of 32768 31 / 22 / 25, 64 rows of 32768
    // 48 / 32 / 31, 16 rows of 4096 11.8 / 13.3 / 13.0, 64 rows of 4096 16.0 / 15.5 / 19.8.  16 heads of 256, 5 rows of 1999: 15.9 /
    // 22.0 / 21.7, which is two steps, one and one.)
    pl.chunk_prefix = pl.tile_prefix ? tile_chunk()
                                     : chunk(C.dim > 128 ? 2 * step : step, work_prefix, B.n_prefix);
    // Own tiles of many rows are one chunk where that is quicker than to share the chip evenly and join: they take some 1.7 us for 64 keys of 128 features, and cut into 512 parts 2.4 items / 512 and
    // some 20 us for sums that go through memory.  (Whole / cut: prompts of 300, 400 and 512 tokens 16.9 / 23.6, 18.9 / 26.9, 21.9 / 28.9, 512 behind 1000 and 8000 own 46 / 39,
    // 213 / 100, 1000 alone and behind 8000 35 / 49, 226 / 189, 200 behind 8000 205 / 54, four times 60 behind 2048 shared 59 / 31.)  Whole ones take the prefix, too, ahead of their own keys,
    // unless it is read much oftener for it: the rule of the 16-bit cache.
    const int64_t beyond = tiles - (rows + pl.rows_own - 1) / pl.rows_own;   // tiles more than all rows in a row would take
    bool whole = pl.tile_own && (double)all * C.dim * (363.0 - items) <= 3.5e7;
    if (whole && items > 363 && B.n_prefix == 0) {         // rounds that are far from full.  (Whole / cut: 1500 tokens on 30000 own keys 1030 / 816, of 64 features 722 / 498.)
        tile_chunk();
        whole = 0.9 * rounds_of(items) * STEP * (double)all * C.dim <= least;
    }
    pl.ahead = B.n_prefix > 0 && (pl.few || (whole && (4 * beyond <= tiles || beyond * B.n_prefix <= 16384)));
    if (pl.ahead || pl.few)
        pl.chunk_own = (int32_t)((all + 15 + step - 1) / step * step);
    else if (pl.tile_own && !(whole && B.n_prefix == 0))
        pl.chunk_own = tile_chunk();
    else
        pl.chunk_own = (int32_t)((B.max_len + step - 1) / step * step);
    if (pl.ahead)
        pl.tiles_prefix = 0;
    pl.chunks_prefix = pl.ahead ? 0 : (B.n_prefix + pl.chunk_prefix - 1) / pl.chunk_prefix;
    pl.chunks_own = pl.ahead ? 1 : (B.max_len + pl.chunk_own - 1) / pl.chunk_own;
    // Other own parts of a few rows, longer than a step, are cut by the device, which counts quanta in 32 bits: into 512 parts and more, behind tiles of the prefix 256.  (256 / 512 / 1024: 32
    // sequences of 500 to 8000 keys 63 / 52 / 53, 64 of 100 to 4000 60 / 51 / 55, four of 500 to 30000 33 / 25 / 27, 16 of 20 rows and 500 to 4000 31 / 26 / 33, 8 of 100 to 4000 of 16 heads of 256 43 / 40 / 45;
    // 48 of 5 to 700 behind 32768 66 / 66 / 69, 16 of five tokens there 79 / 81 / 82.  Cut by max_len instead, the best number of workgroups for each: 57, 58, 27, 33.)
    // Parts are whole steps of a workgroup, beside tiles two: those of up to 256 keys, often all that a sequence has, stay in one piece.  (Two steps / one: 48 of 5 to 700 behind 32768 62.4 / 60.6, of
    // 100 to 250 57.4 / 58.1, 16 of five tokens and 5 to 700 74.0 / 73.9, 17 of 130 to 255 behind 65536 51.0 / 51.4, 40 of two and 5 to 2000 behind 16384 63.0 / 59.3, 100 of 5 to 1000 there 73.7 / 73.9.)
    pl.quantum = (int32_t)(pl.beside ? ATT_FEW_WAVES / ATT_WAVES * step : step);
    pl.deal = -1;
    if (!pl.tile_own && !pl.few && !pl.lone && B.max_len > pl.quantum && tiles * ((B.max_len + (int64_t)pl.quantum - 1) / pl.quantum) < (int64_t)1 << 31) {
        pl.deal = pl.beside ? 8 : 9;
        pl.parts = (((int64_t)1 << pl.deal) / C.kv_heads) + tiles;
        pl.chunks_own = 0;
    }
    const int64_t row_heads = (int64_t)seqs.cu[seqs.n] * n_heads;
    pl.slots_own = (row_heads * pl.chunks_prefix + 1) / 2 * 2;
    if (pl.deal >= 0)
        pl.floats = (size_t)(pl.slots_own + pl.parts * C.kv_heads * pl.rows_own) * (C.dim + 2) + 4 * seqs.n;
    else if (pl.chunks_prefix + pl.chunks_own > 1)
        pl.floats = (size_t)row_heads * (pl.chunks_prefix + pl.chunks_own) * (C.dim + 2);
    return pl;
}

size_t attend_q4_floats(const griffin_kv_cache_q4 &C, const griffin_kv_batch &B, const SeqTable &seqs, int32_t n_heads)
{
    return attend_takes(seqs, n_heads) ? attend_q4_plan(C, B, seqs, n_heads).floats : 0;
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
static int attend_typed(AttendQ4Params &p, const Q4Plan &pl, hipStream_t st)
{
    int rc = GRIFFIN_OK;
    const int32_t wgs_prefix = p.kv_heads * pl.tiles_prefix * pl.chunks_prefix, wgs_own = p.kv_heads * (int32_t)(pl.deal < 0 ? (int64_t)pl.tiles_own * pl.chunks_own : pl.parts);
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
    return rc == GRIFFIN_OK && p.part ? launch_attend_join(p, !F32, pl.chunks_prefix + (pl.deal < 0 ? pl.chunks_own : (1 << pl.deal) / p.kv_heads / pl.tiles_own), st) : rc;
}

template <bool F32>
static int attend_width(AttendQ4Params &p, const Q4Plan &pl, hipStream_t st)
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
    const Q4Plan pl = attend_q4_plan(C, job.B, seqs, job.n_heads);
    if (!att_launch_fits(pl, C.kv_heads) || (pl.deal >= 0 && (pl.parts * C.kv_heads >= 1 << 23 || pl.parts * C.kv_heads * C.kv_heads >= (int64_t)1 << 32)))
        return GRIFFIN_EUNSUPPORTED;
    AttendQ4Params p = {};
    p.q = job.q; p.K = C.K; p.V = C.V; p.out = job.out;
    p.ldq = job.ldq; p.hsq = job.hsq; p.ldo = job.ldo; p.hso = job.hso;
    att_set_up(p, pl, job.B, seqs, job.n_heads, C.kv_heads, C.dim, C.page_size, C.n_pages, job.scale, job.ws);
    p.s = q4_shape(C);
    p.deal = pl.deal; p.quantum = pl.quantum; p.rows_own = pl.rows_own; p.slots_own = pl.slots_own;
    if (pl.deal >= 0) {
        const int64_t slots = pl.slots_own + pl.parts * C.kv_heads * pl.rows_own;
        p.part = job.ws;
        p.part_ml = (float2 *)(job.ws + slots * C.dim);
        p.cuts = (int4 *)(p.part_ml + slots);              // an even number of slots: 16 bytes
    }
    return C.dtype == GRIFFIN_BF16 ? attend_width<false>(p, pl, st) : attend_width<true>(p, pl, st);
}

}  // namespace griffin
