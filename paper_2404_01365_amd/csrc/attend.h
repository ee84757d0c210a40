// What the attention's kernels share: those of a few rows (attend_rows.h, keys straight into registers) and of many (attend_tile.hip,
// keys through LDS).
#pragma once

#include "layer.h"

namespace griffin {

typedef __attribute__((ext_vector_type(4))) float att_f32x4;
typedef __attribute__((ext_vector_type(8))) __bf16 att_bf16x8;
typedef __attribute__((ext_vector_type(4))) uint32_t att_u32x4;

__device__ __forceinline__ att_f32x4 att_mfma(att_u32x4 a, att_u32x4 b, att_f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(att_bf16x8, a), __builtin_bit_cast(att_bf16x8, b), c, 0, 0, 0);
}

// l += the sum over keys of bf16 weights in a B operand, by a product with ones: every element of a column's lanes holds that row's sum.  The softmax's sum is
// one of the weights as they are multiplied, rounded to bf16, and not as they were before: what a weight is off by then is in numerator and denominator alike, so
// that weights add up to one and a row that one key dominates is as exact as its value, also where that key's weight is no power of two.  (Computed on the host for 513
// normal scores and references that lag by up to 2^8, relative to the output: deviation 6, 0.7e-3 instead of 1.5e-3; 1.5, 1.6e-3 either way.)
__device__ __forceinline__ void att_add_weights(att_f32x4 &l, att_u32x4 w)
{
    constexpr uint32_t ONES = 0x3F803F80u;
    l = att_mfma(att_u32x4{ONES, ONES, ONES, ONES}, w, l);
}

constexpr int ATT_WAVES = 4;            // of a workgroup of attend_rows_kernel
constexpr int ATT_FEW_WAVES = 8;        // ... of attend_few_kernel, and of own parts beside tiles
constexpr int ATT_TILE_WAVES = 8;       // ... of attend_tile.hip
constexpr int att_tile_keys(int32_t dim) { return dim > 128 ? 32 : 64; }      // its step

// Division by a number that the host knows, exact while the dividend times it is below 2^32
struct AttDiv {
    uint32_t by, mul;

    __device__ __forceinline__ int32_t operator()(int32_t x) const { return by == 1 ? x : (int32_t)__umulhi((uint32_t)x, mul); }
};

struct AttendParams {
    const void *q, *K, *V;
    void *out;
    float *part;             // [tokens][n_heads][chunks][dim] unscaled sums, or NULL: one chunk, written to `out`
    float2 *part_ml;         // [tokens][n_heads][chunks] maximum (base 2) and sum
    const int32_t *lens, *pages, *prefix_pages;
    int64_t ldq, hsq, ldo, hso, page_stride, head_stride, token_stride, ld_pages;
    uint32_t page_stride16;  // page_stride in 16 bytes
    float scale2;            // scale log2(e)
    int32_t tokens, n_heads, kv_heads, group, dim, page_shift, last_page, max_len, n_prefix;
    AttDiv by_heads, by_kv_heads, by_group, by_chunks_prefix, by_chunks_own;
    // keys a chunk (a multiple of a workgroup's step), chunks, and tiles of rows of the prefix
    int32_t chunk_prefix, chunk_own, chunks_prefix, chunks_own, tiles_prefix;
    int32_t ahead;           // tokens of the prefix that own items take ahead of their own: all (then there are no items of the prefix) or 0
    int32_t wgs_prefix;      // workgroups of this launch that take the prefix, ahead of those that take own parts
    int32_t items_own;       // own items of this launch
    AttDiv each, tiles_each;                                  // new tokens, and tiles of rows, of every sequence where they are equally many, else by 0
    SeqTable seqs;
    int32_t tiles_own[GRIFFIN_MAX_SEQS + 1];                  // tiles of rows of the sequences before; where attend_tile.hip takes own parts:
    uint8_t order[GRIFFIN_MAX_SEQS];                          // ... in this order, the sequences with most tiles first
};

// A workgroup's share: rows first .. of the `rows` rows whose tokens begin at token0 (row = token * group + member of the group), against keys
// [begin, end) of a list of pages, for kv head hk.  own: the position of token0 among its sequence's own tokens; -1: every row sees every key.
struct AttendItem {
    const int32_t *pages;
    int32_t last_entry;      // of the list that may be read
    int32_t begin, end, own, hk, token0, rows, first, split;
    // Where own items take the prefix, too, they count its keys first and their own from the next multiple of 16 on: keys from hole to hole_end are none,
    // and `own`, `begin` and `end` are counted like that.  Else both are 0.
    int32_t hole, hole_end;

    __device__ __forceinline__ bool missing(int32_t key) const { return key >= hole && key < hole_end; }
    __device__ __forceinline__ bool touches_hole(int32_t key0, int32_t keys) const { return hole < hole_end && key0 < hole_end && key0 + keys > hole; }
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
__device__ __forceinline__ uint32_t att_page(int32_t page, int32_t last_page) { return page < 0 ? 0 : (page > last_page ? last_page : page); }

// The number of the page that holds a tile of 16 keys.  Keys behind the last one are read like others (the table's entry, clamped into the pools: some memory of
// theirs), get no weight, and their values are made zero before they are multiplied by it.  By the vector memory path: a wait for a scalar load is one for all
// that is asked of LDS behind it, too.
__device__ __forceinline__ int32_t att_look_up(const AttendParams &p, const AttendItem &it, int32_t key)
{
    const bool ahead = key < it.hole_end;
    const int32_t last = ahead ? (it.hole - 1) >> p.page_shift : it.last_entry;
    int32_t at = (ahead ? key : key - it.hole_end) >> p.page_shift;
    at = at < last ? at : last;
    asm volatile("" : "+v"(at));
    return (ahead ? p.prefix_pages : it.pages)[at];
}

// where that tile begins, in bytes from the kv head's begin
template <int ES>
__device__ __forceinline__ uint64_t att_place(const AttendParams &p, const AttendItem &it, int32_t page, int32_t key)
{
    key -= key < it.hole_end ? 0 : it.hole_end;
    return (uint64_t)att_page(__builtin_amdgcn_readfirstlane(page), p.last_page) * p.page_stride16 * 16 +
           (uint64_t)(uint32_t)(key & ((1 << p.page_shift) - 1)) * ((uint32_t)p.token_stride * ES);
}

// All bits of the two bf16 in a word that are neither infinite nor NaN (an exponent of all ones)
__device__ __forceinline__ uint32_t att_finite_mask(uint32_t w)
{
    typedef __attribute__((ext_vector_type(2))) uint16_t pair_t;
    const pair_t missing = __builtin_bit_cast(pair_t, ~w & 0x7F807F80u);      // 0: all ones
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_min(missing, pair_t{1, 1}) * pair_t{0xFFFF, 0xFFFF});
}

// The sequence that `at` falls to, of `per` (tokens or tiles of rows) each or, with per 0, by the sums in `first`
__device__ __forceinline__ int att_sequence(int32_t at, const AttDiv &per, const int32_t *first, int n)
{
    if (per.by > 0)
        return per(at);
    int b = 0, hi = n - 1;                                    // the last sequence that begins at or before `at`
    while (b < hi) {
        const int mid = (b + hi + 1) / 2;
        if (first[mid] <= at) b = mid;
        else hi = mid - 1;
    }
    return b;
}

// Prefix item `id` of [tile of ROWS rows][chunk][kv head]
template <int ROWS>
__device__ __forceinline__ void att_prefix_item(const AttendParams &p, int32_t id, AttendItem &it)
{
    const int32_t of_heads = p.by_kv_heads(id), tile = p.by_chunks_prefix(of_heads), chunk = of_heads - tile * p.chunks_prefix;
    it.hk = id - of_heads * p.kv_heads;
    it.pages = p.prefix_pages;
    it.last_entry = (p.n_prefix - 1) >> p.page_shift;
    it.begin = chunk * p.chunk_prefix;
    it.end = it.begin + p.chunk_prefix < p.n_prefix ? it.begin + p.chunk_prefix : p.n_prefix;
    it.own = -1;
    it.token0 = 0;
    it.rows = p.tokens * p.group;
    it.first = tile * ROWS;
    it.split = chunk;
    it.hole = it.hole_end = 0;
}

// Tiles of rows in falling order of their number within a sequence, so that those that see the most keys are begun first: the `id`-th one.  With tiles
// T_0 >= T_1 >= .. of the sequences in p.order and S_m = T_0 + .. + T_(m-1), m sequences have a tile t for t in [T_m, T_(m-1)), and S_m - m t
// tiles have number t or more.
__device__ __forceinline__ void att_top_tile(const AttendParams &p, int32_t id, int &b, int32_t &tile)
{
    int lo = 1, hi = p.seqs.n;                                // the least m with id < S_m - m T_m (T_n = 0)
    while (lo < hi) {
        const int mid = (lo + hi) / 2;
        const int32_t below = mid < p.seqs.n ? p.tiles_own[mid + 1] - p.tiles_own[mid] : 0;
        if (id < p.tiles_own[mid] - mid * below) hi = mid;
        else lo = mid + 1;
    }
    tile = (p.tiles_own[lo] - 1 - id) / lo;
    b = p.order[id - (p.tiles_own[lo] - lo * (tile + 1))];
}

// Own item `id` of [tile of ROWS rows][chunk][kv head]; TOP: tiles as att_top_tile has them.  false: no row needs it.
template <int ROWS, bool TOP>
__device__ __forceinline__ bool att_own_item(const AttendParams &p, int32_t id, AttendItem &it)
{
    const int32_t of_heads = p.by_kv_heads(id), of_chunks = p.by_chunks_own(of_heads), chunk = of_heads - of_chunks * p.chunks_own;
    int b;
    int32_t tile;
    if (TOP)
        att_top_tile(p, of_chunks, b, tile);
    else {
        b = att_sequence(of_chunks, p.tiles_each, p.tiles_own, p.seqs.n);
        tile = of_chunks - p.tiles_own[b];
    }
    it.hk = id - of_heads * p.kv_heads;
    const int32_t len = p.lens[b];
    it.pages = p.pages + (int64_t)b * p.ld_pages;
    it.last_entry = (p.max_len - 1) >> p.page_shift;
    it.token0 = p.seqs.cu[b];
    it.rows = (p.seqs.cu[b + 1] - p.seqs.cu[b]) * p.group;
    it.first = tile * ROWS;
    it.own = len < 0 ? 0 : (len < p.max_len ? len : p.max_len);
    const int32_t last = it.first + ROWS < it.rows ? it.first + ROWS - 1 : it.rows - 1;               // the tile's last row sees the most keys
    it.hole = p.ahead;
    it.hole_end = (p.ahead + 15) & ~15;
    const int32_t end = it.hole_end + (it.own + p.by_group(last) + 1 < p.max_len ? it.own + p.by_group(last) + 1 : p.max_len);
    it.own += it.hole_end;
    it.begin = chunk * p.chunk_own;
    it.end = it.begin + p.chunk_own < end ? it.begin + p.chunk_own : end;
    it.split = p.chunks_prefix + chunk;
    return it.begin < it.end;                                 // else no row reads this chunk's partial sums
}

// launches the `wgs` workgroups of p on tiles of att_tile_rows(dim) rows, and behind them p.items_own own items of 16 rows, a workgroup each or, `each`, a
// wavefront each (dim <= 128); bf16 only
int launch_attend_tiles(const AttendParams &p, int32_t wgs, bool each, hipStream_t st);
constexpr int att_tile_rows(int32_t dim) { return 16 * ATT_TILE_WAVES * (dim > 128 ? 1 : 2); }

}  // namespace griffin
