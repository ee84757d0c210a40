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

// `sizes_only`: what a workspace query looks at
static int check_batch(const griffin_kv_cache &C, const griffin_kv_batch *B, SeqTable &seqs, bool sizes_only)
{
    if (!B || !B->cu_seqlens || B->n_seqs < 1 || B->max_len < 1 || B->n_prefix < 0)
        return GRIFFIN_EINVAL;
    if (B->n_seqs > GRIFFIN_MAX_SEQS)
        return GRIFFIN_EUNSUPPORTED;
    if (!sizes_only && (!B->lens || !B->pages || (B->n_prefix > 0 && !B->prefix_pages)))
        return GRIFFIN_EINVAL;
    if ((int64_t)B->max_len + B->n_prefix > (1 << 30))
        return GRIFFIN_ESHAPE;
    if (!sizes_only && B->ld_pages < (B->max_len + C.page_size - 1) / C.page_size)
        return GRIFFIN_ESHAPE;
    if (B->cu_seqlens[0] != 0)
        return GRIFFIN_ESHAPE;
    seqs.n = B->n_seqs;
    for (int b = 0; b <= GRIFFIN_MAX_SEQS; ++b) {
        seqs.cu[b] = B->cu_seqlens[b < B->n_seqs ? b : B->n_seqs];
        if (b > 0 && seqs.cu[b] < seqs.cu[b - 1])
            return GRIFFIN_ESHAPE;
    }
    return seqs.cu[seqs.n] > (1 << 20) ? GRIFFIN_EUNSUPPORTED : GRIFFIN_OK;
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

int griffin_kv_append(const griffin_kv_cache *C, const griffin_kv_batch *B, const void *k, int64_t ldk, int64_t hsk, const void *v,
                      int64_t ldv, int64_t hsv, const void *q, int64_t ldq, int64_t hsq, void *q_out, int64_t ldo, int64_t hso,
                      int32_t n_heads, const float *cos, const float *sin, int64_t n_pos, int32_t rot, int32_t style, void *stream)
{
    int rc = check_cache(C);
    if (rc != GRIFFIN_OK)
        return rc;
    SeqTable seqs;
    if ((rc = check_batch(*C, B, seqs, false)) != GRIFFIN_OK)
        return rc;
    if (seqs.cu[seqs.n] == 0)
        return GRIFFIN_OK;
    if (!k || !v || (q == nullptr) != (q_out == nullptr) || rot < 0 || (rot > 0 && (!cos || !sin || n_pos < 1)) || (q && n_heads < 1))
        return GRIFFIN_EINVAL;
    if (style != GRIFFIN_ROT_HALF && style != GRIFFIN_ROT_PAIRS)
        return GRIFFIN_EINVAL;
    if (rot > C->dim || rot % 2 != 0 || !row_stride(ldk, C->dim) || !row_stride(hsk, C->dim) || !row_stride(ldv, C->dim) ||
        !row_stride(hsv, C->dim) || !aligned16(k) || !aligned16(v) || !aligned16(q) || !aligned16(q_out) || !aligned16(cos) || !aligned16(sin))
        return GRIFFIN_ESHAPE;
    if (q && (!row_stride(ldq, C->dim) || !row_stride(hsq, C->dim) || !row_stride(ldo, C->dim) || !row_stride(hso, C->dim) ||
              (q == q_out && (ldq != ldo || hsq != hso))))
        return GRIFFIN_ESHAPE;
    if (q && n_heads > 1024)
        return GRIFFIN_EUNSUPPORTED;
    const AppendJob job = {*C, *B, k, v, q, q_out, ldk, hsk, ldv, hsv, ldq, hsq, ldo, hso, q ? n_heads : 0, rot, style, cos, sin, n_pos};
    return launch_kv_append(job, seqs, (hipStream_t)stream);
}

static int check_heads(const griffin_kv_cache &C, int32_t n_heads)
{
    if (n_heads < 1)
        return GRIFFIN_EINVAL;
    if (n_heads % C.kv_heads != 0)
        return GRIFFIN_ESHAPE;
    return n_heads > 1024 ? GRIFFIN_EUNSUPPORTED : GRIFFIN_OK;
}

size_t griffin_attention_workspace_bytes(const griffin_kv_cache *C, const griffin_kv_batch *B, int32_t n_heads)
{
    SeqTable seqs;
    if (check_cache(C) != GRIFFIN_OK || check_batch(*C, B, seqs, true) != GRIFFIN_OK || check_heads(*C, n_heads) != GRIFFIN_OK)
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
    if ((rc = check_batch(*C, B, seqs, false)) != GRIFFIN_OK || (rc = check_heads(*C, n_heads)) != GRIFFIN_OK)
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

}  // extern "C"
