// What the two attention kernels share: attend.hip (a few rows, keys straight into registers) and attend_tile.hip (many rows,
// keys through LDS).
#pragma once

#include "layer.h"

namespace griffin {

typedef __attribute__((ext_vector_type(4))) float att_f32x4;
typedef __attribute__((ext_vector_type(8))) __bf16 att_bf16x8;
typedef __attribute__((ext_vector_type(4))) uint32_t att_u32x4;

constexpr int ATT_WAVES = 4;            // of a workgroup of attend.hip
constexpr int ATT_TILE_WAVES = 8;       // ... of attend_tile.hip
constexpr int ATT_TILE_KEYS = 64;       // its step

struct AttendParams {
    const void *q, *K, *V;
    void *out;
    float *part;             // [tokens][n_heads][chunks][dim] unscaled sums, or NULL: one chunk, written to `out`
    float2 *part_ml;         // [tokens][n_heads][chunks] maximum (base 2) and sum
    const int32_t *lens, *pages, *prefix_pages;
    int64_t ldq, hsq, ldo, hso, page_stride, head_stride, token_stride, ld_pages;
    uint32_t page_stride16;  // page_stride in 16 bytes (of bf16)
    float scale2;            // scale log2(e)
    int32_t n_heads, kv_heads, group, dim, page_shift, last_page, max_len, n_prefix;
    // keys a chunk (a multiple of a workgroup's step), chunks, and tiles of rows of the prefix
    int32_t chunk_prefix, chunk_own, chunks_prefix, chunks_own, tiles_prefix;
    int32_t wgs_prefix;      // workgroups of this launch that take the prefix, ahead of those that take own parts
    SeqTable seqs;
    int32_t tiles_own[GRIFFIN_MAX_SEQS + 1];                  // tiles of rows of the sequences before
};

// A workgroup's share: rows first .. of the `rows` rows whose tokens begin at token0 (row = token * group + member of the group), against keys
// [begin, end) of a list of pages, for kv head hk.  own: the position of token0 among its sequence's own tokens; -1: every row sees every key.
struct AttendItem {
    const int32_t *pages;
    int32_t begin, end, own, hk, token0, rows, first, split;
};

// maximum over the lanes l, l ^ 16, l ^ 32, l ^ 48
__device__ __forceinline__ float lane_groups_max(float v)
{
    typedef __attribute__((ext_vector_type(2))) uint32_t pair_t;
    pair_t r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(r.x), __uint_as_float(r.y));
    r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r.x), __uint_as_float(r.y));
}

// a page's number, kept in the pools
__device__ __forceinline__ int64_t att_page(int32_t page, int32_t last_page) { return page < 0 ? 0 : (page > last_page ? last_page : page); }

// where the tiles of a step lie: tile t's page and its first slot there, kept in range of the keys that there are
struct AttTile {
    int64_t base;                // elements from the head's begin
    int32_t rows;                // its valid slots less one
};

__device__ __forceinline__ AttTile att_tile(const AttendParams &p, const int32_t *pages, int32_t key0, int32_t end)
{
    const int32_t last = (end - 1) & ~15;
    key0 = key0 < last ? key0 : last;
    key0 = __builtin_amdgcn_readfirstlane(key0);
    AttTile t;
    t.base = page_of(pages, key0 >> p.page_shift, p.last_page) * p.page_stride + (int64_t)(key0 & ((1 << p.page_shift) - 1)) * p.token_stride;
    t.rows = end - 1 - key0 < 15 ? end - 1 - key0 : 15;
    return t;
}

// All bits of the two bf16 in a word that are neither infinite nor NaN (an exponent of all ones)
__device__ __forceinline__ uint32_t att_finite_mask(uint32_t w)
{
    return ((w & 0x7F80u) == 0x7F80u ? 0 : 0xFFFFu) | ((w & 0x7F800000u) == 0x7F800000u ? 0 : 0xFFFF0000u);
}

// The item of workgroup `id`; false: no row needs it.  Workgroups go [tile of ROWS rows][chunk][kv head], the prefix's first; TOP: own tiles from
// the last to the first, those that see the most keys ahead
template <int ROWS_PREFIX, int ROWS_OWN, bool TOP>
__device__ __forceinline__ bool att_item(const AttendParams &p, int32_t id, AttendItem &it)
{
    if (id < p.wgs_prefix) {
        const int chunk = id / p.kv_heads % p.chunks_prefix, tile = id / p.kv_heads / p.chunks_prefix;
        it.hk = id % p.kv_heads;
        it.pages = p.prefix_pages;
        it.begin = chunk * p.chunk_prefix;
        it.end = it.begin + p.chunk_prefix < p.n_prefix ? it.begin + p.chunk_prefix : p.n_prefix;
        it.own = -1;
        it.token0 = 0;
        it.rows = p.seqs.cu[p.seqs.n] * p.group;
        it.first = tile * ROWS_PREFIX;
        it.split = chunk;
        return true;
    }
    id -= p.wgs_prefix;
    const int chunk = id / p.kv_heads % p.chunks_own;
    int tile = id / p.kv_heads / p.chunks_own;
    if (TOP)
        tile = p.tiles_own[p.seqs.n] - 1 - tile;
    it.hk = id % p.kv_heads;
    int b = 0, hi = p.seqs.n - 1;                          // the last sequence whose tiles begin at or before this one
    while (b < hi) {
        const int mid = (b + hi + 1) / 2;
        if (p.tiles_own[mid] <= tile) b = mid;
        else hi = mid - 1;
    }
    it.token0 = p.seqs.cu[b];
    it.rows = (p.seqs.cu[b + 1] - p.seqs.cu[b]) * p.group;
    it.first = (tile - p.tiles_own[b]) * ROWS_OWN;
    it.own = p.lens[b] < 0 ? 0 : (p.lens[b] < p.max_len ? p.lens[b] : p.max_len);
    const int32_t last = it.first + ROWS_OWN < it.rows ? it.first + ROWS_OWN - 1 : it.rows - 1;       // the tile's last row sees the most keys
    const int32_t end = it.own + last / p.group + 1 < p.max_len ? it.own + last / p.group + 1 : p.max_len;
    it.pages = p.pages + (int64_t)b * p.ld_pages;
    it.begin = chunk * p.chunk_own;
    it.end = it.begin + p.chunk_own < end ? it.begin + p.chunk_own : end;
    it.split = p.chunks_prefix + chunk;
    return it.begin < it.end;                              // else no row reads this chunk's partial sums
}

// launches the `wgs` workgroups of p on tiles of att_tile_rows(dim) rows; bf16 only
int launch_attend_tiles(const AttendParams &p, int32_t wgs, hipStream_t st);
constexpr int att_tile_rows(int32_t dim) { return 16 * ATT_TILE_WAVES * (dim > 128 ? 1 : 2); }

}  // namespace griffin
