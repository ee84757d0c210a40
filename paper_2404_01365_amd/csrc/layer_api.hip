// C ABI of what surrounds the FF block: argument validation (before any HIP call), then the launchers.
#include <math.h>

#include "layer.h"

namespace griffin {

static bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }
static bool known_type(int32_t t) { return t == GRIFFIN_F32 || t == GRIFFIN_BF16; }
// a row stride for rows of `width` elements
static bool row_stride(int64_t ld, int64_t width) { return ld >= width && ld % 8 == 0; }

static int check_cache(const griffin_kv_cache *C)
{
    if (!C || !C->K || !C->V || !known_type(C->dtype) || C->kv_heads < 1 || C->dim < 1 || C->page_size < 1 || C->n_pages < 1)
        return GRIFFIN_EINVAL;
    if (C->dim % 8 != 0 || !aligned16(C->K) || !aligned16(C->V) || !row_stride(C->token_stride, C->dim) ||
        !row_stride(C->head_stride, C->dim) || C->page_stride < 0 || C->page_stride % 8 != 0 || C->n_pages > INT32_MAX)
        return GRIFFIN_ESHAPE;
    if (C->dim > 256 || C->token_stride > (1 << 26) || C->page_stride > (1ll << 33) || C->page_size < 16 || C->page_size > 65536 || (C->page_size & (C->page_size - 1)) || C->kv_heads > 1024)
        return GRIFFIN_EUNSUPPORTED;
    return GRIFFIN_OK;
}

// the host's table of n <= GRIFFIN_MAX_SEQS sequences; false: it does not begin at 0, or falls
static bool take_seqs(const int32_t *cu, int32_t n, SeqTable &seqs)
{
    seqs.n = n;
    for (int b = 0; b <= GRIFFIN_MAX_SEQS; ++b) {
        seqs.cu[b] = cu[b < n ? b : n];
        if (seqs.cu[b] < (b > 0 ? seqs.cu[b - 1] : 0))
            return false;
    }
    return seqs.cu[0] == 0;
}

// `sizes_only`: what a workspace query looks at
static int check_batch(int32_t page_size, const griffin_kv_batch *B, SeqTable &seqs, bool sizes_only)
{
    if (!B || !B->cu_seqlens || B->n_seqs < 1 || B->max_len < 1 || B->n_prefix < 0)
        return GRIFFIN_EINVAL;
    if (B->n_seqs > GRIFFIN_MAX_SEQS)
        return GRIFFIN_EUNSUPPORTED;
    if (!sizes_only && (!B->lens || !B->pages || (B->n_prefix > 0 && !B->prefix_pages)))
        return GRIFFIN_EINVAL;
    if ((int64_t)B->max_len + B->n_prefix > (1 << 30))
        return GRIFFIN_ESHAPE;
    if (!sizes_only && B->ld_pages < (B->max_len + page_size - 1) / page_size)
        return GRIFFIN_ESHAPE;
    if (!take_seqs(B->cu_seqlens, B->n_seqs, seqs))
        return GRIFFIN_ESHAPE;
    return seqs.cu[seqs.n] > (1 << 20) ? GRIFFIN_EUNSUPPORTED : GRIFFIN_OK;
}

static bool q4_sizes(int32_t kv_heads, int32_t dim, int32_t page_size, int32_t group)
{
    return kv_heads >= 1 && kv_heads <= 1024 && dim >= 8 && dim <= 256 && dim % 8 == 0 && page_size >= 16 && page_size <= 65536 &&
           !(page_size & (page_size - 1)) && (group == 32 || group == 64);
}

static int check_cache_q4(const griffin_kv_cache_q4 *C)
{
    if (!C || !C->K || !C->V || !known_type(C->dtype) || C->kv_heads < 1 || C->dim < 1 || C->page_size < 1 || C->group < 1 || C->n_pages < 1)
        return GRIFFIN_EINVAL;
    if (C->dim % 8 != 0 || !aligned16(C->K) || !aligned16(C->V) || C->n_pages > INT32_MAX)
        return GRIFFIN_ESHAPE;
    return q4_sizes(C->kv_heads, C->dim, C->page_size, C->group) ? GRIFFIN_OK : GRIFFIN_EUNSUPPORTED;
}

}  // namespace griffin

using namespace griffin;

extern "C" {

int griffin_norm_residual(const griffin_norm *N, int64_t rows, const void *h, int64_t ldh, int32_t h_dtype, const void *y, int64_t ldy,
                          const void *gate, int64_t ldg, void *h_out, int64_t ldo, void *x, int64_t ldx, void *stream)
{
    if (!N || rows < 0 || !known_type(N->dtype) || !known_type(h_dtype) || N->d < 1)
        return GRIFFIN_EINVAL;
    if (N->kind != GRIFFIN_NORM_RMS && N->kind != GRIFFIN_NORM_LAYER)
        return GRIFFIN_EINVAL;
    if (!(N->eps > 0) || !isfinite(N->eps) || !isfinite(N->w_offset) || !isfinite(N->h_scale) || !isfinite(N->y_scale))
        return GRIFFIN_EINVAL;
    if (rows == 0)
        return GRIFFIN_OK;
    if (!h || (!h_out && !x) || (x && !N->w_pre) || (N->b_pre && !N->w_pre) || (N->b_post && !N->w_post) || (!y && gate))
        return GRIFFIN_EINVAL;
    if (h_dtype == GRIFFIN_BF16 && N->dtype != GRIFFIN_BF16)
        return GRIFFIN_EUNSUPPORTED;
    if (N->d % 8 != 0 || rows > ((int64_t)1 << 30) || !row_stride(ldh, N->d) || (y && !row_stride(ldy, N->d)) ||
        (gate && ldg != 0 && !row_stride(ldg, N->d)) || (h_out && !row_stride(ldo, N->d)) || (x && !row_stride(ldx, N->d)))
        return GRIFFIN_ESHAPE;
    for (const void *p : {h, y, gate, (const void *)h_out, (const void *)x, N->w_pre, N->b_pre, N->w_post, N->b_post})
        if (!aligned16(p))
            return GRIFFIN_ESHAPE;
    if (x && x == h_out)
        return GRIFFIN_EINVAL;
    if ((h_out == h && ldo != ldh) || (x && x == y && ldx != ldy))
        return GRIFFIN_ESHAPE;
    if (N->d > 32768)
        return GRIFFIN_EUNSUPPORTED;
    const NormJob job = {*N, rows, ldh, ldy, ldg, ldo, ldx, h_dtype == GRIFFIN_BF16, h, y, gate, h_out, x};
    return launch_norm_residual(job, (hipStream_t)stream);
}

// k, v, q and the rotation of an append whose cache holds dim features
static int check_append(int32_t dim, const void *k, int64_t ldk, int64_t hsk, const void *v, int64_t ldv, int64_t hsv, const void *q, int64_t ldq, int64_t hsq,
                        const void *q_out, int64_t ldo, int64_t hso, int32_t n_heads, const float *cos, const float *sin, int64_t n_pos, int32_t rot, int32_t style)
{
    if (!k || !v || (q == nullptr) != (q_out == nullptr) || rot < 0 || (rot > 0 && (!cos || !sin || n_pos < 1)) || (q && n_heads < 1))
        return GRIFFIN_EINVAL;
    if (style != GRIFFIN_ROT_HALF && style != GRIFFIN_ROT_PAIRS)
        return GRIFFIN_EINVAL;
    if (rot > dim || rot % 2 != 0 || !row_stride(ldk, dim) || !row_stride(hsk, dim) || !row_stride(ldv, dim) ||
        !row_stride(hsv, dim) || !aligned16(k) || !aligned16(v) || !aligned16(q) || !aligned16(q_out) || !aligned16(cos) || !aligned16(sin))
        return GRIFFIN_ESHAPE;
    if (q && (!row_stride(ldq, dim) || !row_stride(hsq, dim) || !row_stride(ldo, dim) || !row_stride(hso, dim) ||
              (q == q_out && (ldq != ldo || hsq != hso))))
        return GRIFFIN_ESHAPE;
    return q && n_heads > 1024 ? GRIFFIN_EUNSUPPORTED : GRIFFIN_OK;
}

int griffin_kv_append(const griffin_kv_cache *C, const griffin_kv_batch *B, const void *k, int64_t ldk, int64_t hsk, const void *v,
                      int64_t ldv, int64_t hsv, const void *q, int64_t ldq, int64_t hsq, void *q_out, int64_t ldo, int64_t hso,
                      int32_t n_heads, const float *cos, const float *sin, int64_t n_pos, int32_t rot, int32_t style, void *stream)
{
    int rc = check_cache(C);
    if (rc != GRIFFIN_OK)
        return rc;
    SeqTable seqs;
    if ((rc = check_batch(C->page_size, B, seqs, false)) != GRIFFIN_OK)
        return rc;
    if (seqs.cu[seqs.n] == 0)
        return GRIFFIN_OK;
    if ((rc = check_append(C->dim, k, ldk, hsk, v, ldv, hsv, q, ldq, hsq, q_out, ldo, hso, n_heads, cos, sin, n_pos, rot, style)) != GRIFFIN_OK)
        return rc;
    const AppendJob job = {*C, *B, k, v, q, q_out, ldk, hsk, ldv, hsv, ldq, hsq, ldo, hso, q ? n_heads : 0, rot, style, cos, sin, n_pos};
    return launch_kv_append(job, seqs, (hipStream_t)stream);
}

static int check_heads(int32_t kv_heads, int32_t n_heads)
{
    if (n_heads < 1)
        return GRIFFIN_EINVAL;
    if (n_heads % kv_heads != 0)
        return GRIFFIN_ESHAPE;
    return n_heads > 1024 ? GRIFFIN_EUNSUPPORTED : GRIFFIN_OK;
}

size_t griffin_attention_workspace_bytes(const griffin_kv_cache *C, const griffin_kv_batch *B, int32_t n_heads)
{
    SeqTable seqs;
    if (check_cache(C) != GRIFFIN_OK || check_batch(C->page_size, B, seqs, true) != GRIFFIN_OK || check_heads(C->kv_heads, n_heads) != GRIFFIN_OK)
        return 0;
    return attend_floats(*C, *B, seqs, n_heads) * sizeof(float);
}

int griffin_attention(const griffin_kv_cache *C, const griffin_kv_batch *B, const void *q, int64_t ldq, int64_t hsq, void *out, int64_t ldo,
                      int64_t hso, int32_t n_heads, float scale, void *workspace, size_t workspace_bytes, void *stream)
{
    int rc = check_cache(C);
    if (rc != GRIFFIN_OK)
        return rc;
    SeqTable seqs;
    if ((rc = check_batch(C->page_size, B, seqs, false)) != GRIFFIN_OK || (rc = check_heads(C->kv_heads, n_heads)) != GRIFFIN_OK)
        return rc;
    if (seqs.cu[seqs.n] == 0)
        return GRIFFIN_OK;
    if (!q || !out || q == out || !(scale > 0) || !isfinite(scale))
        return GRIFFIN_EINVAL;
    if (!row_stride(ldq, C->dim) || !row_stride(hsq, C->dim) || !row_stride(ldo, C->dim) || !row_stride(hso, C->dim) || !aligned16(q) ||
        !aligned16(out))
        return GRIFFIN_ESHAPE;
    const size_t need = attend_floats(*C, *B, seqs, n_heads) * sizeof(float);
    if (need > 0 && (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < need))
        return GRIFFIN_EWORKSPACE;
    const AttendJob job = {*C, *B, q, out, ldq, hsq, ldo, hso, n_heads, scale, (float *)workspace};
    return launch_attend(job, seqs, (hipStream_t)stream);
}

size_t griffin_kv_q4_page_bytes(int32_t kv_heads, int32_t dim, int32_t page_size, int32_t group)
{
    if (!q4_sizes(kv_heads, dim, page_size, group))
        return 0;
    return (size_t)kv_heads * page_size * ((dim + 31) / 32 * 16 + (dim + group - 1) / group * 4);
}

int griffin_kv_append_q4(const griffin_kv_cache_q4 *C, const griffin_kv_batch *B, const void *k, int64_t ldk, int64_t hsk, const void *v,
                         int64_t ldv, int64_t hsv, const void *q, int64_t ldq, int64_t hsq, void *q_out, int64_t ldo, int64_t hso,
                         int32_t n_heads, const float *cos, const float *sin, int64_t n_pos, int32_t rot, int32_t style, void *stream)
{
    int rc = check_cache_q4(C);
    if (rc != GRIFFIN_OK)
        return rc;
    SeqTable seqs;
    if ((rc = check_batch(C->page_size, B, seqs, false)) != GRIFFIN_OK)
        return rc;
    if (seqs.cu[seqs.n] == 0)
        return GRIFFIN_OK;
    if ((rc = check_append(C->dim, k, ldk, hsk, v, ldv, hsv, q, ldq, hsq, q_out, ldo, hso, n_heads, cos, sin, n_pos, rot, style)) != GRIFFIN_OK)
        return rc;
    const AppendQ4Job job = {*C, *B, k, v, q, q_out, ldk, hsk, ldv, hsv, ldq, hsq, ldo, hso, q ? n_heads : 0, rot, style, cos, sin, n_pos};
    return launch_kv_append_q4(job, seqs, (hipStream_t)stream);
}

int griffin_kv_read_q4(const griffin_kv_cache_q4 *C, const griffin_kv_batch *B, void *k, int64_t ldk, int64_t hsk, void *v, int64_t ldv, int64_t hsv,
                       void *stream)
{
    int rc = check_cache_q4(C);
    if (rc != GRIFFIN_OK)
        return rc;
    SeqTable seqs;
    if ((rc = check_batch(C->page_size, B, seqs, false)) != GRIFFIN_OK)
        return rc;
    if (seqs.cu[seqs.n] == 0)
        return GRIFFIN_OK;
    if ((!k && !v) || k == v)
        return GRIFFIN_EINVAL;
    if ((k && (!row_stride(ldk, C->dim) || !row_stride(hsk, C->dim))) || (v && (!row_stride(ldv, C->dim) || !row_stride(hsv, C->dim))) || !aligned16(k) || !aligned16(v))
        return GRIFFIN_ESHAPE;
    const ReadQ4Job job = {*C, *B, k, v, ldk, hsk, ldv, hsv};
    return launch_kv_read_q4(job, seqs, (hipStream_t)stream);
}

size_t griffin_attention_q4_workspace_bytes(const griffin_kv_cache_q4 *C, const griffin_kv_batch *B, int32_t n_heads)
{
    SeqTable seqs;
    if (check_cache_q4(C) != GRIFFIN_OK || check_batch(C->page_size, B, seqs, true) != GRIFFIN_OK || check_heads(C->kv_heads, n_heads) != GRIFFIN_OK)
        return 0;
    return attend_q4_floats(*C, *B, seqs, n_heads) * sizeof(float);
}

int griffin_attention_q4(const griffin_kv_cache_q4 *C, const griffin_kv_batch *B, const void *q, int64_t ldq, int64_t hsq, void *out, int64_t ldo,
                         int64_t hso, int32_t n_heads, float scale, void *workspace, size_t workspace_bytes, void *stream)
{
    int rc = check_cache_q4(C);
    if (rc != GRIFFIN_OK)
        return rc;
    SeqTable seqs;
    if ((rc = check_batch(C->page_size, B, seqs, false)) != GRIFFIN_OK || (rc = check_heads(C->kv_heads, n_heads)) != GRIFFIN_OK)
        return rc;
    if (seqs.cu[seqs.n] == 0)
        return GRIFFIN_OK;
    if (!q || !out || q == out || !(scale > 0) || !isfinite(scale))
        return GRIFFIN_EINVAL;
    if (!row_stride(ldq, C->dim) || !row_stride(hsq, C->dim) || !row_stride(ldo, C->dim) || !row_stride(hso, C->dim) || !aligned16(q) ||
        !aligned16(out))
        return GRIFFIN_ESHAPE;
    const size_t need = attend_q4_floats(*C, *B, seqs, n_heads) * sizeof(float);
    if (need > 0 && (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < need))
        return GRIFFIN_EWORKSPACE;
    const AttendQ4Job job = {*C, *B, q, out, ldq, hsq, ldo, hso, n_heads, scale, (float *)workspace};
    return launch_attend_q4(job, seqs, (hipStream_t)stream);
}

size_t griffin_verify_workspace_bytes(int32_t n_seqs, int32_t vocab)
{
    return n_seqs < 1 || n_seqs > GRIFFIN_MAX_SEQS || vocab < 1 || vocab > (1 << 24) ? 0 : verify_bytes(n_seqs, vocab);
}

int griffin_verify_drafts(const float *p, int64_t ldp, const float *draft_p, int64_t ldq, const int32_t *drafted, const int32_t *cu_seqlens_host,
                          int32_t n_seqs, int32_t vocab, const float *accept_u, const float *draw_u, int32_t *tokens_out, int32_t *accepted,
                          const int32_t *lens, int32_t *lens_out, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!cu_seqlens_host || n_seqs < 1 || vocab < 1 || !draw_u || !accepted || (lens == nullptr) != (lens_out == nullptr))
        return GRIFFIN_EINVAL;
    if (n_seqs > GRIFFIN_MAX_SEQS || vocab > (1 << 24))
        return GRIFFIN_EUNSUPPORTED;
    SeqTable seqs;
    if (!take_seqs(cu_seqlens_host, n_seqs, seqs))
        return GRIFFIN_ESHAPE;
    const int32_t rows = seqs.cu[n_seqs];
    if (rows > 0 && (!p || !drafted || !accept_u || !tokens_out))
        return GRIFFIN_EINVAL;
    // a sequence's tokens are written while another's are read
    if ((uintptr_t)tokens_out < (uintptr_t)drafted + (uintptr_t)rows * 4 && (uintptr_t)drafted < (uintptr_t)tokens_out + (uintptr_t)rows * 4)
        return GRIFFIN_EINVAL;
    if (rows > 1 && (ldp < vocab || (draft_p && ldq < vocab)))
        return GRIFFIN_ESHAPE;
    for (const void *at : {(const void *)p, (const void *)draft_p, (const void *)drafted, (const void *)accept_u, (const void *)draw_u, (const void *)tokens_out,
                           (const void *)accepted, (const void *)lens, (const void *)lens_out})
        if ((uintptr_t)at & 3)
            return GRIFFIN_ESHAPE;
    const size_t need = verify_bytes(n_seqs, vocab);
    if (need > 0 && (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < need))
        return GRIFFIN_EWORKSPACE;
    const VerifyJob job = {p, draft_p, ldp, ldq, drafted, vocab, accept_u, draw_u, tokens_out, accepted, lens, lens_out, (double *)workspace};
    return launch_verify(job, seqs, (hipStream_t)stream);
}

}  // extern "C"
