// What the kernels around the FF block share: descriptors checked by layer_api.hip, launchers.
#pragma once

#include "common.h"

namespace griffin {

struct NormJob {
    griffin_norm N;
    int64_t rows, ldh, ldy, ldg, ldo, ldx;
    bool h_bf16;
    const void *h, *y, *gate;
    void *h_out, *x;
};
int launch_norm_residual(const NormJob &job, hipStream_t st);

struct AppendJob {
    griffin_kv_cache C;
    griffin_kv_batch B;
    const void *k, *v, *q;
    void *q_out;
    int64_t ldk, hsk, ldv, hsv, ldq, hsq, ldo, hso;
    int32_t n_heads, rot, style;
    const float *cos, *sin;
    int64_t n_pos;
};
int launch_kv_append(const AppendJob &job, const SeqTable &seqs, hipStream_t st);

struct AttendJob {
    griffin_kv_cache C;
    griffin_kv_batch B;
    const void *q;
    void *out;
    int64_t ldq, hsq, ldo, hso;
    int32_t n_heads;
    float scale;
    float *ws;
};
// floats of workspace
size_t attend_floats(const griffin_kv_cache &C, const griffin_kv_batch &B, const SeqTable &seqs, int32_t n_heads);
int launch_attend(const AttendJob &job, const SeqTable &seqs, hipStream_t st);

struct AppendQ4Job {
    griffin_kv_cache_q4 C;
    griffin_kv_batch B;
    const void *k, *v, *q;
    void *q_out;
    int64_t ldk, hsk, ldv, hsv, ldq, hsq, ldo, hso;
    int32_t n_heads, rot, style;
    const float *cos, *sin;
    int64_t n_pos;
};
int launch_kv_append_q4(const AppendQ4Job &job, const SeqTable &seqs, hipStream_t st);

struct ReadQ4Job {
    griffin_kv_cache_q4 C;
    griffin_kv_batch B;
    void *k, *v;
    int64_t ldk, hsk, ldv, hsv;
};
int launch_kv_read_q4(const ReadQ4Job &job, const SeqTable &seqs, hipStream_t st);

struct AttendQ4Job {
    griffin_kv_cache_q4 C;
    griffin_kv_batch B;
    const void *q;
    void *out;
    int64_t ldq, hsq, ldo, hso;
    int32_t n_heads;
    float scale;
    float *ws;
};
size_t attend_q4_floats(const griffin_kv_cache_q4 &C, const griffin_kv_batch &B, const SeqTable &seqs, int32_t n_heads);
int launch_attend_q4(const AttendQ4Job &job, const SeqTable &seqs, hipStream_t st);

struct VerifyJob {
    const float *p, *q;
    int64_t ldp, ldq;
    const int32_t *drafted;
    int32_t vocab;
    const float *accept_u, *draw_u;
    int32_t *tokens_out, *accepted;
    const int32_t *lens;
    int32_t *lens_out;
    double *ws;
};
size_t verify_bytes(int32_t n_seqs, int32_t vocab);
int launch_verify(const VerifyJob &job, const SeqTable &seqs, hipStream_t st);

// The page of a token, clamped into the pools; `at` is the same for the whole wavefront.
__device__ __forceinline__ int64_t page_of(const int32_t *pages, int32_t at, int32_t last_page)
{
    const int32_t p = pages[__builtin_amdgcn_readfirstlane(at)];
    return p < 0 ? 0 : (p > last_page ? last_page : p);
}

}  // namespace griffin
