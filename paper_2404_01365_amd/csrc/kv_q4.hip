// A step's keys and values into a cache in 4 bits (griffin_kv_append_q4), and out of one (griffin_kv_read_q4).
//
// c = round((x - m) / s) with s = fp16((hi - lo) / 15), m = fp16(lo + 8 s) of a group's least and greatest value.  A thread takes eight features, a word of
// codes; a group's threads are neighbouring lanes, which exchange lo and hi.  By its definition all of it is computed in 64 bits: a value next to the border of two codes falls to
// the side that the definition says, not to one that the order of fp32 operations chooses.  Few are that near, so everything is computed in fp32 with a bound on how far off it
// is, and in 64 bits only by wavefronts where a rounding lies within that bound.
//
// Bound by its instructions, some 250 a wavefront of eight features a lane: 4150 tokens of 32 heads of 128 on as many, halves of them rotated in pairs, 155 MB, 50 us (all
// of it in 64 bits: 54.7), 57 where 1.3 GB of states take turns; 16 tokens of 32 heads on 8 are a launch and a chain of loads, 5.0.  Reading back: 32768 tokens of 8 heads of 128, 172 MB, 37.6 us, 4.6 TB/s,
// again and again, part of it cached; where states take turns 54.4, 3.2 TB/s, two thirds of a copy's rate: a thread's 16 or 32 bytes wait for a length, a page and a code one after the other.
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

// a word, or a value, of the lane l ^ 1, 2 or 4 of a row of eight
template <int STEP>
__device__ __forceinline__ uint32_t q4_other(uint32_t w)
{
    // row_half_mirror exchanges lanes l and 7 - l: the four of each half have the same value by then
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)w, STEP == 1 ? 0xB1 : STEP == 2 ? 0x4E : 0x141, 0xF, 0xF, true);
}

template <int STEP>
__device__ __forceinline__ float q4_other(float v) { return __uint_as_float(q4_other<STEP>(__float_as_uint(v))); }

template <int STEP>
__device__ __forceinline__ double q4_other(double v)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    return __builtin_bit_cast(double, (uint64_t)q4_other<STEP>((uint32_t)b) | (uint64_t)q4_other<STEP>((uint32_t)(b >> 32)) << 32);
}

// the least, the greatest of a group's
__device__ __forceinline__ float q4_min(float a, float b) { return fminf(a, b); }
__device__ __forceinline__ double q4_min(double a, double b) { return fmin(a, b); }

template <bool WIDE, class T>
__device__ __forceinline__ T q4_group_min(T v)
{
    v = q4_min(v, q4_other<1>(v));
    v = q4_min(v, q4_other<2>(v));
    return WIDE ? q4_min(v, q4_other<4>(v)) : v;
}

template <bool WIDE, class T>
__device__ __forceinline__ T q4_group_max(T v) { return -q4_group_min<WIDE>(-v); }

// To fp16 by way of fp32, two instructions.  The compiler makes one rounding of it by some forty, which gives another result where fp32 falls between two fp16.
__device__ __forceinline__ _Float16 q4_half(double v)
{
    float f = (float)v;
    asm("" : "+v"(f));
    return (_Float16)f;
}

// What a thread has of its head's codes: a word, and its group's (scale, middle) word
struct Q4Out {
    uint32_t codes, pair;
};

__device__ __forceinline__ uint32_t q4_pair_word(_Float16 scale, _Float16 middle)
{
    return (uint32_t)__builtin_bit_cast(uint16_t, scale) | (uint32_t)__builtin_bit_cast(uint16_t, middle) << 16;
}

// The definition, in 64 bits; `in`: the features are the head's
template <bool WIDE>
__device__ __forceinline__ Q4Out q4_quantise_exactly(const double (&x)[8], bool in)
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
    lo = in ? lo : 32768.0;
    hi = in ? odd ? 1e9 : hi : -32768.0;   // a group that holds a value that is not finite is marked by a range no other has
    lo = q4_group_min<WIDE>(lo);
    hi = q4_group_max<WIDE>(hi);
    odd = hi > 1e8;
    const _Float16 scale = q4_half((hi - lo) / 15.0);
    const double step = (double)(float)scale;
    const _Float16 middle = q4_half(lo + 8.0 * step);
    const double mid = (double)(float)middle;
    const bool flat = odd || !(step > 0);
    uint32_t codes = 0;
#pragma unroll 1
    for (int j = 0; j < 8; ++j) {
        const double d = fmin(fmax(x[j], -32768.0), 32768.0) - mid;
        const double c = flat ? 0.0 : fmin(fmax(rint(d / step), -8.0), 7.0);
        codes |= (uint32_t)((int)c + 8) << 4 * j;
    }
    return {codes, odd ? 0x7E00u : q4_pair_word(scale, middle)};
}

// The same in fp32, from values that are up to `off` from the exact ones: false where a rounding to fp16, or a code, could be another, where values are cut to the
// format's range or are not finite.
template <bool WIDE>
__device__ __forceinline__ bool q4_quantise_fast(const float (&x)[8], float off, bool in, Q4Out &out)
{
    float lo = INFINITY, hi = -INFINITY;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        lo = fminf(lo, x[j]);
        hi = fmaxf(hi, x[j]);
    }
    lo = q4_group_min<WIDE>(in ? lo : INFINITY);
    hi = q4_group_max<WIDE>(in ? hi : -INFINITY);
    off = q4_group_max<WIDE>(off);
    // s: the difference and the product are off by 2^-24 of themselves, 1 / 15 as well.  m: what the sum has lost is known, and often nothing: values of few bits, as bf16 are, would
    // else be taken for ones next to a rounding's border whenever they lie on it.  t: the reciprocal is off by 2^-23 of itself, which counts for x and for the middle, at most as large
    // as the greatest value and four steps, and each product and sum by 2^-24 of itself.  A little more is allowed for each.
    const float size = fmaxf(fabsf(lo), fabsf(hi));
    const float s = (hi - lo) * (1.0f / 15.0f), se = off * 0.14f + 0x1p-22f * fabsf(s);
    const _Float16 scale = (_Float16)(s - se), above = (_Float16)(s + se);
    const float step = (float)scale, m = lo + 8.0f * step, part = m - lo;
    const float me = off + 1.01f * fabsf((lo - (m - part)) + (8.0f * step - part));
    const _Float16 middle = (_Float16)(m - me), beyond = (_Float16)(m + me);
    const float inv = __builtin_amdgcn_rcpf(step), shift = 8.0f - (float)middle * inv;
    const float near = 0.5f - (1.01f * off * inv + 0x1p-21f * size * inv + 4e-6f);
    const bool same = __builtin_bit_cast(uint16_t, middle) == __builtin_bit_cast(uint16_t, beyond);        // zeros of both signs are not
    bool sure = scale == above && same && size + off <= 32768.0f && step > 0;      // infinities: not sure
    // codes of even and of odd features in bytes, by a conversion that takes a number into a byte of a word
    uint32_t even = 0, odd = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float t = x[j] * inv + shift, c = rintf(t);
        sure &= fabsf(t - c) < near;                       // NaN: not sure
        uint32_t &word = j & 1 ? odd : even;
        word = __builtin_amdgcn_cvt_pk_u8_f32(fminf(c, 15.0f), j / 2, word);
    }
    const uint32_t codes = even | odd << 4;
    out = {codes, q4_pair_word(scale, middle)};
    return sure || !in;
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
    const bool is_k = head < p.s.kv_heads, is_q = head >= 2 * p.s.kv_heads;
    const int h = is_k ? head : is_q ? head - 2 * p.s.kv_heads : head - p.s.kv_heads;
    const void *src = is_k ? p.k : is_q ? p.q : p.v;
    const int64_t from = is_k ? token * p.ldk + h * p.hsk : is_q ? token * p.ldq + h * p.hsq : token * p.ldv + h * p.hsv;
    const int f = i * 8;
    const bool in = f < p.dim;
    float x[8], z[8], c[8], s[8];
    q4_load8<BF16>(src, from + (in ? f : 0), x);
    // places are looked up while that is on its way
    const int b = q4_sequence(p.seqs, p.each, token);
    const int32_t held = p.lens[b] < 0 ? 0 : p.lens[b];
    const int64_t slot = (int64_t)held + token - p.seqs.cu[b];
    const int64_t pos = slot + p.n_prefix < p.n_pos ? slot + p.n_prefix : p.n_pos - 1;
    const bool room = slot < p.max_len;    // else no slot: only the query is of use
    const int64_t page = room ? page_of(p.pages + (int64_t)b * p.ld_pages, (int32_t)(slot >> p.s.page_shift), p.s.last_page) : 0;
    // feature a of a pair becomes a cos - b sin, feature b becomes b cos + a sin: with the other one of a pair in z, x cos + z sin with sin's sign
    const bool rotated = (is_k || is_q) && in && f < 2 * p.half;
    const auto turned = [&](int j) { return FAST || f + j < 2 * p.half; };     // else the feature stays as it is: z sin could be 0 x Inf
    float y[8], off = 0;
    if (rotated) {
        const float *cs = p.cos + pos * p.half, *sn = p.sin + pos * p.half;
        if constexpr (PAIRS) {
            float c4[4], s4[4];
            if (FAST) {
                *(float4 *)c4 = *(const float4 *)(cs + f / 2);
                *(float4 *)s4 = *(const float4 *)(sn + f / 2);
            } else
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int e = f / 2 + j < p.half ? f / 2 + j : p.half - 1;
                    c4[j] = cs[e];
                    s4[j] = sn[e];
                }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                z[j] = x[j ^ 1];
                c[j] = c4[j / 2];
                s[j] = j & 1 ? s4[j / 2] : -s4[j / 2];
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
                const bool first = f + j < p.half;
                const int e = turned(j) ? (first ? f + j : f + j - p.half) : 0;
                z[j] = turned(j) ? load_scalar<BF16>(src, from + (first ? f + j + p.half : e)) : 0.0f;
                c[j] = cs[e];
                s[j] = first ? -sn[e] : sn[e];
            }
        // off by half a last place of the second product, and of the sum
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float second = z[j] * s[j];
            y[j] = turned(j) ? __builtin_fmaf(x[j], c[j], second) : x[j];
            off = fmaxf(off, turned(j) ? fabsf(second) + fabsf(y[j]) : 0.0f);
        }
        off *= 0x1.01p-24f;
    } else
#pragma unroll
        for (int j = 0; j < 8; ++j)
            y[j] = x[j];
    if (is_q) {                            // q_out may be q: all of a head's threads have loaded by now, as they are of one wavefront
        if (in)
            q4_store8<BF16>(p.q_out, token * p.ldo + h * p.hso + f, y);
        return;
    }
    Q4Out out;
    const bool sure = q4_quantise_fast<WIDE>(y, off, in, out);
    if (__any(!sure)) {                    // one wavefront in ten or so, of keys
        double exact[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            asm volatile("" : "+v"(x[j]), "+v"(z[j]), "+v"(c[j]), "+v"(s[j]));        // here, not ahead of the branch for everyone
            exact[j] = rotated && turned(j) ? (double)x[j] * (double)c[j] + (double)z[j] * (double)s[j] : (double)x[j];
        }
        out = q4_quantise_exactly<WIDE>(exact, in);
    }
    if (!room)
        return;
    char *at = (is_k ? p.K : p.V) + (page * p.s.kv_heads + h) * p.s.head_bytes;
    const uint32_t row = (uint32_t)(slot & ((1 << p.s.page_shift) - 1));
    if ((uint32_t)i * 4 < p.s.row_bytes)
        *(uint32_t *)(at + row * p.s.row_bytes + i * 4) = in ? out.codes : 0;
    if (in && (i & (WIDE ? 7 : 3)) == 0)
        *(uint32_t *)(at + p.s.pairs_at + (row * p.s.groups + (i >> (WIDE ? 3 : 2))) * 4) = out.pair;
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
