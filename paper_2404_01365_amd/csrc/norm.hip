// Norms around a block (griffin_norm_residual): u = N(y) behind it, h' = h_scale h + y_scale gate u, x = N(h') before the next.
// Bound by bytes from some hundreds of rows on (h, y and a gate are read once, h' and x written once), by latency below.  A row is
// held in registers from its first load to its last store, so the second norm's statistics cost no second pass.
// Measured (a large copy reaches 4.9 TB/s; pass behind pass, part of the rows in the caches / caches cold): 1024 rows of 5120, fp32 stream, 63 MB, 13.1 us =
// 4.8 TB/s / 20.6 us = 3.1; 8191 rows of 4096 with a gate for each, layer norm, 335 MB, 61 us = 5.5 TB/s / 84 us = 4.0; one row of 4096 4.1 us, a launch's own.
#include "layer.h"

namespace griffin {

constexpr int64_t NORM_ROWS = 1 << 21;     // of one launch

struct NormParams {
    const void *h, *y, *gate, *w_pre, *b_pre, *w_post, *b_post;
    void *h_out, *x;
    int64_t rows, ldh, ldy, ldg, ldo, ldx;
    int32_t d;
    float eps, inv_d, w_offset, h_scale, y_scale;
};

// eight values of a row, in registers as fp32
template <bool BF16>
__device__ __forceinline__ void load8(const void *p, int64_t i, float (&v)[8])
{
    if (BF16) {
        const uint4 w = *(const uint4 *)((const uint16_t *)p + i);
        v[0] = bf16_lo(w.x); v[1] = bf16_hi(w.x); v[2] = bf16_lo(w.y); v[3] = bf16_hi(w.y);
        v[4] = bf16_lo(w.z); v[5] = bf16_hi(w.z); v[6] = bf16_lo(w.w); v[7] = bf16_hi(w.w);
    } else {
        const float4 a = *(const float4 *)((const float *)p + i), b = *(const float4 *)((const float *)p + i + 4);
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    }
}

template <bool BF16>
__device__ __forceinline__ void store8(void *p, int64_t i, const float (&v)[8])
{
    if (BF16)
        *(uint4 *)((uint16_t *)p + i) = make_uint4(f32x2_to_bf16x2(v[0], v[1]), f32x2_to_bf16x2(v[2], v[3]), f32x2_to_bf16x2(v[4], v[5]),
                                                   f32x2_to_bf16x2(v[6], v[7]));
    else {
        *(float4 *)((float *)p + i) = make_float4(v[0], v[1], v[2], v[3]);
        *(float4 *)((float *)p + i + 4) = make_float4(v[4], v[5], v[6], v[7]);
    }
}

// Sum over the row's wavefronts; every thread ends with it.  `patch` holds WAVES floats and is used by one sum only.
template <int WAVES>
__device__ __forceinline__ float row_sum(float v, float *patch)
{
    v = wave_sum(v);
    if (WAVES == 1)
        return v;
    if ((threadIdx.x & 63) == 0)
        patch[threadIdx.x >> 6] = v;
    __syncthreads();
    float s = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w)
        s += patch[w];
    return s;
}

// what N takes from the row: 1 / sqrt(mean square + eps), of deviations from `mean` for a layer norm (two passes over registers:
// the mean square less the squared mean would lose the digits of a row with a large mean)
template <bool LAYER, int WAVES, int CH>
__device__ __forceinline__ float row_stat(const float (&v)[CH][8], const bool (&in)[CH], float inv_d, float eps, float *patch, float &mean)
{
    mean = 0;
    if (LAYER) {
        float s = 0;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                s += in[c] ? v[c][j] : 0.0f;
        mean = row_sum<WAVES>(s, patch) * inv_d;
    }
    float s2 = 0;
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float t = in[c] ? v[c][j] - mean : 0.0f;
            s2 += t * t;
        }
    return rsqrtf(row_sum<WAVES>(s2, patch + 16) * inv_d + eps);
}

// One row per WAVES wavefronts, CH pieces of eight elements a lane.  Rows of up to 64 CH pieces take one wavefront each, four
// rows a workgroup, and no barrier.
template <bool BF16, bool HBF16, bool LAYER, int WAVES, int CH>
__global__ __launch_bounds__(WAVES == 1 ? 256 : WAVES * 64) void norm_residual_kernel(NormParams p)
{
    __shared__ float patch[4][16];
    const int t = WAVES == 1 ? (threadIdx.x & 63) : threadIdx.x;
    const int64_t row = WAVES == 1 ? (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6) : blockIdx.x;
    if (WAVES == 1 && row >= p.rows)
        return;
    const int pieces = p.d >> 3;
    bool in[CH];
    int at[CH];
    float h[CH][8];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int piece = t + c * WAVES * 64;
        in[c] = piece < pieces;
        at[c] = (in[c] ? piece : 0) * 8;          // lanes behind the row's end read its first piece and write nothing
        load8<HBF16>(p.h, row * p.ldh + at[c], h[c]);
    }
    float mean;
    if (p.y) {
        float u[CH][8];
#pragma unroll
        for (int c = 0; c < CH; ++c)
            load8<BF16>(p.y, row * p.ldy + at[c], u[c]);
        if (p.w_post) {
            const float r = row_stat<LAYER, WAVES, CH>(u, in, p.inv_d, p.eps, patch[0], mean);
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                float w[8], b[8] = {0, 0, 0, 0, 0, 0, 0, 0};
                load8<BF16>(p.w_post, at[c], w);
                if (p.b_post)
                    load8<BF16>(p.b_post, at[c], b);
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    u[c][j] = (u[c][j] - mean) * r * (w[j] + p.w_offset) + b[j];
            }
        }
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            float g[8] = {1, 1, 1, 1, 1, 1, 1, 1};
            if (p.gate)
                load8<BF16>(p.gate, row * p.ldg + at[c], g);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                h[c][j] = p.h_scale * h[c][j] + p.y_scale * (g[j] * u[c][j]);
        }
    }
    if (p.h_out)
#pragma unroll
        for (int c = 0; c < CH; ++c)
            if (in[c])
                store8<HBF16>(p.h_out, row * p.ldo + at[c], h[c]);
    if (!p.x)
        return;
    const float r = row_stat<LAYER, WAVES, CH>(h, in, p.inv_d, p.eps, patch[2], mean);
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        float w[8], b[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        load8<BF16>(p.w_pre, at[c], w);
        if (p.b_pre)
            load8<BF16>(p.b_pre, at[c], b);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            w[j] = (h[c][j] - mean) * r * (w[j] + p.w_offset) + b[j];
        if (in[c])
            store8<BF16>(p.x, row * p.ldx + at[c], w);
    }
}

template <bool BF16, bool HBF16, bool LAYER>
static int launch_typed(const NormParams &p, hipStream_t st)
{
    // Pieces of eight for each of 64 lanes: as many wavefronts as leave a lane one piece, up to the sixteen of a workgroup; a row of up to 512 needs no barrier.
    // (Fewer wavefronts of more pieces, caches cold, us: a row of 4096 6.2 by eight, 6.4 by four, 10.9 by one, 256 rows 6.7 / 7.1 / 11.2; a row of 8192 6.1 by
    // sixteen, 6.6 by eight, 7.9 by four; 256 rows of 2048 6.2 by four, 8.2 by one.  Thousands of rows take the same within 5 % either way, but for 4096 by one,
    // 42 against 37.)
    const int lanes = (p.d / 8 + 63) / 64;
#define NORM_GO(WAVES, CH)                                                                                                                  \
    hipLaunchKernelGGL((norm_residual_kernel<BF16, HBF16, LAYER, WAVES, CH>), dim3(WAVES == 1 ? (p.rows + 3) / 4 : p.rows),                  \
                       dim3(WAVES == 1 ? 256 : WAVES * 64), 0, st, p)
    if (lanes <= 1) NORM_GO(1, 1);
    else if (lanes <= 4) NORM_GO(4, 1);
    else if (lanes <= 8) NORM_GO(8, 1);
    else if (lanes <= 16) NORM_GO(16, 1);
    else if (lanes <= 32) NORM_GO(16, 2);
    else NORM_GO(16, 4);
#undef NORM_GO
    return check_launch("norm_residual_kernel");
}

int launch_norm_residual(const NormJob &job, hipStream_t st)
{
    const griffin_norm &N = job.N;
    const bool layer = N.kind == GRIFFIN_NORM_LAYER, bf16 = N.dtype == GRIFFIN_BF16;
    const int64_t es = bf16 ? 2 : 4, hs = job.h_bf16 ? 2 : 4;
    const auto at = [](const void *q, int64_t bytes) { return q ? (char *)q + bytes : nullptr; };
    for (int64_t r = 0; r < job.rows; r += NORM_ROWS) {        // a launch holds fewer than 2^32 threads
        const NormParams p = {at(job.h, r * job.ldh * hs), at(job.y, r * job.ldy * es), at(job.gate, r * job.ldg * es), N.w_pre, N.b_pre,
                              N.w_post, N.b_post, at(job.h_out, r * job.ldo * hs), at(job.x, r * job.ldx * es),
                              job.rows - r < NORM_ROWS ? job.rows - r : NORM_ROWS, job.ldh, job.ldy, job.ldg, job.ldo, job.ldx, N.d, N.eps,
                              1.0f / (float)N.d, N.w_offset, N.h_scale, N.y_scale};
        int rc;
        if (!bf16)
            rc = layer ? launch_typed<false, false, true>(p, st) : launch_typed<false, false, false>(p, st);
        else if (job.h_bf16)
            rc = layer ? launch_typed<true, true, true>(p, st) : launch_typed<true, true, false>(p, st);
        else
            rc = layer ? launch_typed<true, false, true>(p, st) : launch_typed<true, false, false>(p, st);
        if (rc != GRIFFIN_OK)
            return rc;
    }
    return GRIFFIN_OK;
}

}  // namespace griffin
