// A step's keys and values into a cache in 4 bits (griffin_kv_append_q4), and out of one (griffin_kv_read_q4).
//
// c = round((x - m) / s) with s = fp16((hi - lo) / 15), m = fp16(lo + 8 s) of a group's least and greatest value.  A thread takes eight features, a word of
// codes; a group's threads are neighbouring lanes, which exchange lo and hi.  Keys are rotated in 64 bits, where products of two fp32 are exact, and a code is taken
// from the quotient in 64 bits: a value next to the border of two codes falls to the side that the definition says, not to one that the order of fp32 operations
// chooses.  Few are that near: a quotient in fp32 decides the others.
#include "q4.h"

namespace griffin {

struct AppendQ4Params {
    const void *k, *v, *q;
    void *q_out;
    char *K, *V;
    int64_t ldk, hsk, ldv, hsv, ldq, hsq, ldo, hso, ld_pages;
    const int32_t *lens, *pages;
    const float *cos, *sin;
    int64_t n_pos;
    Q4Shape s;
    int32_t n_heads, dim, half, max_len, n_prefix;
    int32_t lanes_shift;                              // threads of a head, a power of two: those of one lie in one wavefront
    int32_t blocks;                                   // workgroups a token
    int32_t token0;                                   // this launch's first token
    int32_t each;                                     // new tokens of every sequence where they are equally many, else 0
    SeqTable seqs;
};

// the sequence of a token
__device__ __forceinline__ int q4_sequence(const SeqTable &seqs, int32_t each, int token)
{
    if (each > 0)
        return token / each;
    int b = 0, hi = seqs.n - 1;            // the last sequence that begins at or before the token
    while (b < hi) {
        const int mid = (b + hi + 1) / 2;
        if (seqs.cu[mid] <= token) b = mid;
        else hi = mid - 1;
    }
    return b;
}

template <bool BF16>
__device__ __forceinline__ void q4_load8(const void *p, int64_t i, float (&x)[8])
{
    if (BF16) {
        const uint4 w = *(const uint4 *)((const uint16_t *)p + i);
        x[0] = bf16_lo(w.x); x[1] = bf16_hi(w.x); x[2] = bf16_lo(w.y); x[3] = bf16_hi(w.y);
        x[4] = bf16_lo(w.z); x[5] = bf16_hi(w.z); x[6] = bf16_lo(w.w); x[7] = bf16_hi(w.w);
    } else {
        *(float4 *)x = *(const float4 *)((const float *)p + i);
        *(float4 *)(x + 4) = *(const float4 *)((const float *)p + i + 4);
    }
}

template <bool BF16>
__device__ __forceinline__ void q4_store8(void *p, int64_t i, const float (&x)[8])
{
    if (BF16)
        *(uint4 *)((uint16_t *)p + i) = make_uint4(f32x2_to_bf16x2(x[0], x[1]), f32x2_to_bf16x2(x[2], x[3]), f32x2_to_bf16x2(x[4], x[5]), f32x2_to_bf16x2(x[6], x[7]));
    else {
        *(float4 *)((float *)p + i) = *(const float4 *)x;
        *(float4 *)((float *)p + i + 4) = *(const float4 *)(x + 4);
    }
}

// a value of the lane l ^ 1, 2 or 4 of a row of eight
template <int STEP>
__device__ __forceinline__ double q4_other(double v)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const auto move = [](uint32_t w) {
        // row_half_mirror exchanges lanes l and 7 - l: the four of each half have the same value by then
        return (uint64_t)(uint32_t)__builtin_amdgcn_update_dpp(0, (int)w, STEP == 1 ? 0xB1 : STEP == 2 ? 0x4E : 0x141, 0xF, 0xF, true);
    };
    return __builtin_bit_cast(double, move((uint32_t)b) | move((uint32_t)(b >> 32)) << 32);
}

// To fp16 by way of fp32, two instructions.  The compiler makes one rounding of it by some forty, which gives another result where fp32 falls between two fp16.
__device__ __forceinline__ _Float16 q4_half(double v)
{
    float f = (float)v;
    asm("" : "+v"(f));
    return (_Float16)f;
}

// Quantises a thread's eight features (zeros and `in` false behind the head's last) and stores their codes and, one thread a group, the scale and middle.
template <bool WIDE>
__device__ __forceinline__ void q4_store_codes(const Q4Shape &s, char *head, uint32_t slot, int i, bool in, bool store, const double (&x)[8])
{
    double lo = 32768, hi = -32768;        // no value is outside
    bool odd = false;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        odd |= !(fabs(x[j]) <= 1.7976931348623157e308);
        const double c = fmin(fmax(x[j], -32768.0), 32768.0);
        lo = fmin(lo, c);
        hi = fmax(hi, c);
    }
    if (!in) {
        lo = 32768;
        hi = -32768;
        odd = false;
    }
    // a group that holds a value that is not finite is marked by a range no other has
    hi = odd ? 1e9 : hi;
    lo = fmin(lo, q4_other<1>(lo)); hi = fmax(hi, q4_other<1>(hi));
    lo = fmin(lo, q4_other<2>(lo)); hi = fmax(hi, q4_other<2>(hi));
    if (WIDE) {
        lo = fmin(lo, q4_other<4>(lo)); hi = fmax(hi, q4_other<4>(hi));
    }
    odd = hi > 1e8;
    const _Float16 scale = q4_half((hi - lo) / 15.0);
    const double step = (double)(float)scale;
    const _Float16 middle = q4_half(lo + 8.0 * step);
    const double mid = (double)(float)middle;
    const float inv = 1.0f / (float)step;
    const bool flat = odd || !(step > 0);
    uint32_t codes = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const double d = fmin(fmax(x[j], -32768.0), 32768.0) - mid;
        const float t = (float)d * inv;    // at most 9 or so, off by less than 2e-6
        float c = rintf(t);
        if (!flat && 0.5f - fabsf(t - c) < 8e-6f)
            c = (float)rint(d / step);
        c = flat ? 0.0f : fminf(fmaxf(c, -8.0f), 7.0f);
        codes |= (uint32_t)((int)c + 8) << 4 * j;
    }
    if (!store)
        return;
    if ((uint32_t)i * 4 < s.row_bytes)
        *(uint32_t *)(head + slot * s.row_bytes + i * 4) = in ? codes : 0;
    if (in && (i & (WIDE ? 7 : 3)) == 0) {
        const uint32_t pair = odd ? 0x7E00u : (uint32_t)__builtin_bit_cast(uint16_t, scale) | (uint32_t)__builtin_bit_cast(uint16_t, middle) << 16;
        *(uint32_t *)(head + s.pairs_at + (slot * s.groups + (i >> (WIDE ? 3 : 2))) * 4) = pair;
    }
}

// Heads of keys, of values, then of queries; a thread's item is eight features of one.  FAST: all of a thread's eight are rotated or none is, and cos and sin
// are loaded four at a time.
template <bool BF16, bool PAIRS, bool FAST, bool WIDE>
__global__ __launch_bounds__(256) void kv_append_q4_kernel(AppendQ4Params p)
{
    const int token = p.token0 + blockIdx.x / p.blocks;
    const int item = (blockIdx.x % p.blocks) * 256 + threadIdx.x, head = item >> p.lanes_shift, i = item & ((1 << p.lanes_shift) - 1);
    if (head >= 2 * p.s.kv_heads + p.n_heads)
        return;                            // whole heads leave
    const int b = q4_sequence(p.seqs, p.each, token);
    const int32_t held = p.lens[b] < 0 ? 0 : p.lens[b];
    const int64_t slot = (int64_t)held + token - p.seqs.cu[b];
    const int64_t pos = slot + p.n_prefix < p.n_pos ? slot + p.n_prefix : p.n_pos - 1;
    const bool room = slot < p.max_len;    // else no slot: only the query is of use
    const bool is_k = head < p.s.kv_heads, is_q = head >= 2 * p.s.kv_heads;
    const int h = is_k ? head : is_q ? head - 2 * p.s.kv_heads : head - p.s.kv_heads;
    const void *src = is_k ? p.k : is_q ? p.q : p.v;
    const int64_t from = is_k ? token * p.ldk + h * p.hsk : is_q ? token * p.ldq + h * p.hsq : token * p.ldv + h * p.hsv;
    const int f = i * 8;
    const bool in = f < p.dim;
    float x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (in)
        q4_load8<BF16>(src, from + f, x);
    double y[8];
#pragma unroll
    for (int j = 0; j < 8; ++j)
        y[j] = x[j];
    if ((is_k || is_q) && in && f < 2 * p.half) {
        // feature a of a pair becomes a cos - b sin, feature b becomes b cos + a sin: with the other one of a pair in z, x cos + z sin with sin's sign
        float z[8], c[8], s[8];
        const float *cs = p.cos + pos * p.half, *sn = p.sin + pos * p.half;
        if constexpr (PAIRS) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                z[j] = x[j ^ 1];
            if (FAST) {
                *(float4 *)c = *(const float4 *)(cs + f / 2);
                *(float4 *)s = *(const float4 *)(sn + f / 2);
            } else
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int e = f / 2 + j < p.half ? f / 2 + j : p.half - 1;
                    c[j] = cs[e];
                    s[j] = sn[e];
                }
#pragma unroll
            for (int j = 7; j >= 0; --j) {
                c[j] = f + j < 2 * p.half ? c[j / 2] : 1.0f;
                s[j] = f + j < 2 * p.half ? (j & 1 ? s[j / 2] : -s[j / 2]) : 0.0f;
            }
        } else if (FAST) {
            const bool first = f < p.half;
            const int e = first ? f : f - p.half;
            q4_load8<BF16>(src, from + (first ? f + p.half : e), z);
            q4_load8<false>(cs, e, c);
            q4_load8<false>(sn, e, s);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                s[j] = first ? -s[j] : s[j];
        } else
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const bool turned = f + j < 2 * p.half, first = f + j < p.half;
                const int e = turned ? (first ? f + j : f + j - p.half) : 0;
                z[j] = turned ? load_scalar<BF16>(src, from + (first ? f + j + p.half : e)) : 0.0f;
                c[j] = turned ? cs[e] : 1.0f;
                s[j] = turned ? (first ? -sn[e] : sn[e]) : 0.0f;
            }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const bool turned = FAST || f + j < 2 * p.half;          // 0 x Inf for those that stay as they are
            if (is_q)
                x[j] = turned ? x[j] * c[j] + z[j] * s[j] : x[j];
            else
                y[j] = turned ? (double)x[j] * (double)c[j] + (double)z[j] * (double)s[j] : y[j];
        }
    }
    if (is_q) {                            // q_out may be q: all of a head's threads have loaded by now, as they are of one wavefront
        if (in)
            q4_store8<BF16>(p.q_out, token * p.ldo + h * p.hso + f, x);
        return;
    }
    char *at = is_k ? p.K : p.V;
    if (room)
        at += (page_of(p.pages + (int64_t)b * p.ld_pages, (int32_t)(slot >> p.s.page_shift), p.s.last_page) * p.s.kv_heads + h) * p.s.head_bytes;
    q4_store_codes<WIDE>(p.s, at, (uint32_t)(slot & ((1 << p.s.page_shift) - 1)), i, in, room, y);
}

template <bool BF16, bool PAIRS, bool FAST>
static int launch_form(AppendQ4Params &p, bool wide, hipStream_t st)
{
    const int32_t tokens = p.seqs.cu[p.seqs.n], most = ((1 << 24) - 1) / p.blocks;        // a launch holds fewer than 2^32 threads
    for (p.token0 = 0; p.token0 < tokens; p.token0 += most) {
        const int32_t now = tokens - p.token0 < most ? tokens - p.token0 : most;
        if (wide)
            hipLaunchKernelGGL((kv_append_q4_kernel<BF16, PAIRS, FAST, true>), dim3((uint32_t)now * p.blocks), dim3(256), 0, st, p);
        else
            hipLaunchKernelGGL((kv_append_q4_kernel<BF16, PAIRS, FAST, false>), dim3((uint32_t)now * p.blocks), dim3(256), 0, st, p);
        const int rc = check_launch("kv_append_q4_kernel");
        if (rc != GRIFFIN_OK)
            return rc;
    }
    return GRIFFIN_OK;
}

template <bool BF16>
static int launch_typed(AppendQ4Params &p, int32_t style, bool wide, hipStream_t st)
{
    if (style == GRIFFIN_ROT_PAIRS)
        return p.half % 4 == 0 ? launch_form<BF16, true, true>(p, wide, st) : launch_form<BF16, true, false>(p, wide, st);
    return p.half % 8 == 0 ? launch_form<BF16, false, true>(p, wide, st) : launch_form<BF16, false, false>(p, wide, st);
}

static int32_t each_of(const SeqTable &seqs)
{
    for (int s = 1; s < seqs.n; ++s)
        if (seqs.cu[s + 1] - seqs.cu[s] != seqs.cu[1])
            return 0;
    return seqs.cu[1];
}

int launch_kv_append_q4(const AppendQ4Job &job, const SeqTable &seqs, hipStream_t st)
{
    const griffin_kv_cache_q4 &C = job.C;
    const griffin_kv_batch &B = job.B;
    AppendQ4Params p = {};
    p.k = job.k; p.v = job.v; p.q = job.q; p.q_out = job.q_out; p.K = (char *)C.K; p.V = (char *)C.V;
    p.ldk = job.ldk; p.hsk = job.hsk; p.ldv = job.ldv; p.hsv = job.hsv;
    p.ldq = job.ldq; p.hsq = job.hsq; p.ldo = job.ldo; p.hso = job.hso;
    p.ld_pages = B.ld_pages; p.lens = B.lens; p.pages = B.pages;
    p.cos = job.cos; p.sin = job.sin; p.n_pos = job.n_pos;
    p.s = q4_shape(C);
    p.n_heads = job.n_heads; p.dim = C.dim; p.half = job.rot / 2;
    p.max_len = B.max_len; p.n_prefix = B.n_prefix;
    const int32_t lanes = (int32_t)(C.group == 64 ? (p.s.row_bytes / 4 + 7) / 8 * 8 : p.s.row_bytes / 4);
    p.lanes_shift = lanes > 1 ? 32 - __builtin_clz(lanes - 1) : 0;
    p.blocks = (((2 * C.kv_heads + p.n_heads) << p.lanes_shift) + 255) / 256;
    p.seqs = seqs;
    p.each = each_of(seqs);
    return C.dtype == GRIFFIN_BF16 ? launch_typed<true>(p, job.style, C.group == 64, st) : launch_typed<false>(p, job.style, C.group == 64, st);
}

// ------------------------------------------------------------------ reading back
struct ReadQ4Params {
    const char *K, *V;
    void *k, *v;
    int64_t ldk, hsk, ldv, hsv, ld_pages;
    const int32_t *lens, *pages;
    Q4Shape s;
    int32_t items, pieces, blocks, max_len, token0, each;       // a token's and a head's pieces of eight features, workgroups a token
    SeqTable seqs;
};

template <bool BF16>
__global__ __launch_bounds__(256) void kv_read_q4_kernel(ReadQ4Params p)
{
    const int token = p.token0 + blockIdx.x / p.blocks;
    const int item = (blockIdx.x % p.blocks) * 256 + threadIdx.x;
    const int b = q4_sequence(p.seqs, p.each, token);
    const int32_t held = p.lens[b] < 0 ? 0 : p.lens[b];
    const int64_t slot = (int64_t)held + token - p.seqs.cu[b];
    if (slot >= p.max_len || item >= p.items)
        return;
    const int head = item / p.pieces, i = item % p.pieces;
    const bool is_k = p.k && head < p.s.kv_heads;
    const int h = p.k && !is_k ? head - p.s.kv_heads : head;
    const uint32_t row = (uint32_t)(slot & ((1 << p.s.page_shift) - 1));
    const char *at = (is_k ? p.K : p.V) +
                     (page_of(p.pages + (int64_t)b * p.ld_pages, (int32_t)(slot >> p.s.page_shift), p.s.last_page) * p.s.kv_heads + h) * p.s.head_bytes;
    const uint32_t w = *(const uint32_t *)(at + row * p.s.row_bytes + i * 4);
    const uint32_t pair = *(const uint32_t *)(at + p.s.pairs_at + (row * p.s.groups + (i * 8 >> p.s.group_shift)) * 4);
    float x[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const q4_pair v = q4_value_pair(w >> 4 * j, q4_scales(pair), q4_middles(pair));
        x[j] = (float)v[0];
        x[j + 4] = (float)v[1];
    }
    if (is_k)
        q4_store8<BF16>(p.k, token * p.ldk + h * p.hsk + i * 8, x);
    else
        q4_store8<BF16>(p.v, token * p.ldv + h * p.hsv + i * 8, x);
}

int launch_kv_read_q4(const ReadQ4Job &job, const SeqTable &seqs, hipStream_t st)
{
    const griffin_kv_cache_q4 &C = job.C;
    ReadQ4Params p = {};
    p.K = (const char *)C.K; p.V = (const char *)C.V; p.k = job.k; p.v = job.v;
    p.ldk = job.ldk; p.hsk = job.hsk; p.ldv = job.ldv; p.hsv = job.hsv;
    p.ld_pages = job.B.ld_pages; p.lens = job.B.lens; p.pages = job.B.pages; p.max_len = job.B.max_len;
    p.s = q4_shape(C);
    p.pieces = C.dim / 8;
    p.items = (job.k && job.v ? 2 : 1) * C.kv_heads * p.pieces;
    p.blocks = (p.items + 255) / 256;
    p.seqs = seqs;
    p.each = each_of(seqs);
    const int32_t tokens = seqs.cu[seqs.n], most = ((1 << 24) - 1) / p.blocks;
    for (p.token0 = 0; p.token0 < tokens; p.token0 += most) {
        const int32_t now = tokens - p.token0 < most ? tokens - p.token0 : most;
        if (C.dtype == GRIFFIN_BF16)
            hipLaunchKernelGGL((kv_read_q4_kernel<true>), dim3((uint32_t)now * p.blocks), dim3(256), 0, st, p);
        else
            hipLaunchKernelGGL((kv_read_q4_kernel<false>), dim3((uint32_t)now * p.blocks), dim3(256), 0, st, p);
        const int rc = check_launch("kv_read_q4_kernel");
        if (rc != GRIFFIN_OK)
            return rc;
    }
    return GRIFFIN_OK;
}

}  // namespace griffin
