// A step's keys and values into their pages, the keys rotated on the way, the queries rotated beside them (griffin_kv_append).
// Moves every element once: bytes bound for prompts, one launch's latency for a token a sequence.  A thread takes eight features where their alignment
// lets it, with both halves of the rotated pairs, so that nothing is read twice; sines and cosines come from tables (they are a program's own, and exact for any
// position).  Measured: 4150 packed prompt tokens of 32 heads, q, k and v, 205 MB, 45 us = 4.5 TB/s, caches cold 54 us = 3.8 (a large copy reaches
// 4.9); a token for each of 16 sequences 4.7 us, a launch's own.
#include "layer.h"

namespace griffin {

struct AppendParams {
    const void *k, *v, *q;
    void *q_out, *K, *V;
    int64_t ldk, hsk, ldv, hsv, ldq, hsq, ldo, hso, page_stride, head_stride, token_stride, ld_pages;
    const int32_t *lens, *pages;
    const float *cos, *sin;
    int64_t n_pos;
    int32_t n_heads, kv_heads, dim, half, pieces, page_shift, last_page, max_len, n_prefix;
    int32_t items, items_rot, items_copy, blocks;     // a token's work; of a rotated and of a copied head; workgroups a token
    int32_t token0;                                   // this launch's first token
    int32_t each;                                     // new tokens of every sequence where they are equally many, else 0
    SeqTable seqs;
};

template <bool BF16, int N>
struct Vec {
    uint32_t w[BF16 ? (N + 1) / 2 : N];
};

// N consecutive elements, aligned to as many (8: 16 bytes of bf16, 32 of fp32)
template <bool BF16, int N>
__device__ __forceinline__ void load_n(const void *p, int64_t i, float (&v)[N])
{
    if (N == 1) {
        v[0] = load_scalar<BF16>(p, i);
        return;
    }
    if (BF16) {
        Vec<true, N> t;
        __builtin_memcpy(&t, __builtin_assume_aligned((const uint16_t *)p + i, 2 * N), sizeof t);
#pragma unroll
        for (int j = 0; j < N; ++j)
            v[j] = j & 1 ? bf16_hi(t.w[j / 2]) : bf16_lo(t.w[j / 2]);
    } else
        __builtin_memcpy(v, __builtin_assume_aligned((const float *)p + i, N >= 4 ? 16 : 4 * N), sizeof v);
}

template <bool BF16, int N>
__device__ __forceinline__ void store_n(void *p, int64_t i, const float (&v)[N])
{
    if (N == 1) {
        store_scalar<BF16>(p, i, v[0]);
        return;
    }
    if (BF16) {
        Vec<true, N> t;
#pragma unroll
        for (int j = 0; j < N / 2; ++j)
            t.w[j] = f32x2_to_bf16x2(v[2 * j], v[2 * j + 1]);
        __builtin_memcpy(__builtin_assume_aligned((uint16_t *)p + i, 2 * N), &t, sizeof t);
    } else
        __builtin_memcpy(__builtin_assume_aligned((float *)p + i, N >= 4 ? 16 : 4 * N), v, sizeof v);
}

// A thread's item of a rotated head is, for halves, N pairs (N features of the first half and those that belong to them) or N features
// behind the rotated ones; for pairs, N consecutive features.  Of a copied head (values): N = 8 features.
template <bool BF16, bool PAIRS, int N>
__global__ __launch_bounds__(256) void kv_append_kernel(AppendParams p)
{
    const int token = p.token0 + blockIdx.x / p.blocks;
    const int item = (blockIdx.x % p.blocks) * 256 + threadIdx.x;
    int b = 0;
    if (p.each > 0)
        b = token / p.each;
    else {
        int hi = p.seqs.n - 1;             // the last sequence that begins at or before the token
        while (b < hi) {
            const int mid = (b + hi + 1) / 2;
            if (p.seqs.cu[mid] <= token) b = mid;
            else hi = mid - 1;
        }
    }
    const int32_t held = p.lens[b] < 0 ? 0 : p.lens[b];
    const int64_t slot = (int64_t)held + token - p.seqs.cu[b];
    if (item >= p.items)
        return;
    const int64_t pos = slot + p.n_prefix < p.n_pos ? slot + p.n_prefix : p.n_pos - 1;
    const bool room = slot < p.max_len;    // else no slot: only the query is of use
    int64_t at = 0;
    if (room)
        at = page_of(p.pages + (int64_t)b * p.ld_pages, (int32_t)(slot >> p.page_shift), p.last_page) * p.page_stride +
             (slot & ((1 << p.page_shift) - 1)) * p.token_stride;

    const int rotated = (p.n_heads + p.kv_heads) * p.items_rot;
    if (item >= rotated) {                 // a value: copied
        const int head = (item - rotated) / p.items_copy, e = (item - rotated) % p.items_copy * 8;
        float x[8];
        load_n<BF16, 8>(p.v, token * p.ldv + head * p.hsv + e, x);
        if (room)
            store_n<BF16, 8>(p.V, at + head * p.head_stride + e, x);
        return;
    }
    const int head = item / p.items_rot, i = item % p.items_rot;
    const bool is_q = head < p.n_heads;
    const void *src = is_q ? p.q : p.k;
    void *dst = is_q ? p.q_out : p.K;
    const int64_t from = is_q ? token * p.ldq + head * p.hsq : token * p.ldk + (head - p.n_heads) * p.hsk;
    const int64_t to = is_q ? token * p.ldo + head * p.hso : at + (head - p.n_heads) * p.head_stride;
    const float *cs = p.cos + pos * p.half, *sn = p.sin + pos * p.half;
    if (!is_q && !room)
        return;
    if constexpr (PAIRS) {
        const int e = i * N;
        float x[N];
        load_n<BF16, N>(src, from + e, x);
        if (e < 2 * p.half) {
            float c[N / 2], s[N / 2];
            load_n<false, N / 2>(cs, e / 2, c);
            load_n<false, N / 2>(sn, e / 2, s);
#pragma unroll
            for (int j = 0; j < N / 2; ++j) {
                const float a = x[2 * j], d = x[2 * j + 1];
                x[2 * j] = a * c[j] - d * s[j];
                x[2 * j + 1] = d * c[j] + a * s[j];
            }
        }
        store_n<BF16, N>(dst, to + e, x);
    } else if (i < p.pieces) {
        const int e = i * N;
        float x[N], z[N], c[N], s[N];
        load_n<BF16, N>(src, from + e, x);
        load_n<BF16, N>(src, from + p.half + e, z);
        load_n<false, N>(cs, e, c);
        load_n<false, N>(sn, e, s);
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const float a = x[j], d = z[j];
            x[j] = a * c[j] - d * s[j];
            z[j] = d * c[j] + a * s[j];
        }
        store_n<BF16, N>(dst, to + e, x);
        store_n<BF16, N>(dst, to + p.half + e, z);
    } else {
        const int e = 2 * p.half + (i - p.pieces) * N;
        float x[N];
        load_n<BF16, N>(src, from + e, x);
        store_n<BF16, N>(dst, to + e, x);
    }
}

template <bool BF16, bool PAIRS, int N>
static int launch_form(AppendParams &p, hipStream_t st)
{
    const int per = PAIRS ? (N < 2 ? 2 : N) : N;
    p.pieces = p.half / per;
    p.items_rot = PAIRS ? p.dim / per : p.pieces + (p.dim - 2 * p.half) / per;
    p.items_copy = p.dim / 8;
    p.items = (p.n_heads + p.kv_heads) * p.items_rot + p.kv_heads * p.items_copy;
    p.blocks = (p.items + 255) / 256;
    const int32_t tokens = p.seqs.cu[p.seqs.n], most = ((1 << 24) - 1) / p.blocks;        // a launch holds fewer than 2^32 threads
    for (p.token0 = 0; p.token0 < tokens; p.token0 += most) {
        const int32_t now = tokens - p.token0 < most ? tokens - p.token0 : most;
        hipLaunchKernelGGL((kv_append_kernel<BF16, PAIRS, N>), dim3((uint32_t)now * p.blocks), dim3(256), 0, st, p);
        const int rc = check_launch("kv_append_kernel");
        if (rc != GRIFFIN_OK)
            return rc;
    }
    return GRIFFIN_OK;
}

template <bool BF16>
static int launch_typed(AppendParams &p, int32_t style, hipStream_t st)
{
    // the widest piece whose loads of features, cos and sin are all aligned
    if (style == GRIFFIN_ROT_PAIRS)
        return p.half % 4 == 0 ? launch_form<BF16, true, 8>(p, st) : launch_form<BF16, true, 2>(p, st);
    if (p.half % 8 == 0)
        return launch_form<BF16, false, 8>(p, st);
    return p.half % 4 == 0 ? launch_form<BF16, false, 4>(p, st) : launch_form<BF16, false, 1>(p, st);
}

int launch_kv_append(const AppendJob &job, const SeqTable &seqs, hipStream_t st)
{
    const griffin_kv_cache &C = job.C;
    const griffin_kv_batch &B = job.B;
    AppendParams p = {};
    p.k = job.k; p.v = job.v; p.q = job.q; p.q_out = job.q_out; p.K = C.K; p.V = C.V;
    p.ldk = job.ldk; p.hsk = job.hsk; p.ldv = job.ldv; p.hsv = job.hsv;
    p.ldq = job.ldq; p.hsq = job.hsq; p.ldo = job.ldo; p.hso = job.hso;
    p.page_stride = C.page_stride; p.head_stride = C.head_stride; p.token_stride = C.token_stride;
    p.ld_pages = B.ld_pages; p.lens = B.lens; p.pages = B.pages;
    p.cos = job.cos; p.sin = job.sin; p.n_pos = job.n_pos;
    p.n_heads = job.n_heads; p.kv_heads = C.kv_heads; p.dim = C.dim; p.half = job.rot / 2;
    p.page_shift = __builtin_ctz(C.page_size);
    p.last_page = (int32_t)(C.n_pages - 1);
    p.max_len = B.max_len; p.n_prefix = B.n_prefix;
    p.seqs = seqs;
    p.each = seqs.cu[1];
    for (int s = 1; s < seqs.n; ++s)
        if (seqs.cu[s + 1] - seqs.cu[s] != p.each)
            p.each = 0;
    return C.dtype == GRIFFIN_BF16 ? launch_typed<true>(p, job.style, st) : launch_typed<false>(p, job.style, st);
}

}  // namespace griffin
