// The join of a row's chunks, which the attention's kernels leave as sums in fp32 (attend.hip, attend_q4.hip).
#pragma once

#include "attend.h"

namespace griffin {

// Where a row's chunks lie: `shared` slots one behind the other, and `own` ones stride_own apart
struct AttParts {
    int64_t first_shared, first_own;
    int32_t shared, own, stride_own;
};

// [row][chunk]: the prefix's, and the own ones that the row's token sees
__device__ __forceinline__ AttParts att_parts(const AttendParams &p, int32_t row, int32_t token, int32_t)
{
    const int b = att_sequence(token, p.each, p.seqs.cu, p.seqs.n);
    const int32_t held = p.lens[b] < 0 ? 0 : (p.lens[b] < p.max_len ? p.lens[b] : p.max_len);
    const int32_t seen = held + token - p.seqs.cu[b] + 1 < p.max_len ? held + token - p.seqs.cu[b] + 1 : p.max_len;
    return {(int64_t)row * (p.chunks_prefix + p.chunks_own), 0, p.chunks_prefix + (seen + p.chunk_own - 1) / p.chunk_own, 0, 0};
}

// Joins a row's chunks: with M = max m_c, o = sum o_c 2^(m_c - M) / sum l_c 2^(m_c - M).  A row per WPR wavefronts; a wavefront takes
// 64 / (DB / 4) chunks at a time, four features a lane.
template <class P, bool BF16, int DB, int WPR>
__global__ __launch_bounds__(256) void attend_join_kernel(P p)
{
    constexpr int LANES = DB / 4, PAR = 64 / LANES;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sub = lane / LANES, d = lane % LANES * 4;
    const int64_t row = (int64_t)blockIdx.x * (4 / WPR) + (WPR == 1 ? wave : 0);
    if (WPR == 1 && row >= (int64_t)p.tokens * p.n_heads)
        return;
    const int32_t token = __builtin_amdgcn_readfirstlane(p.by_heads((int32_t)row)), head = __builtin_amdgcn_readfirstlane((int32_t)row - token * p.n_heads);
    const AttParts parts = att_parts(p, (int32_t)row, token, head);
    const int chunks = parts.shared + parts.own;
    if (chunks == 0)
        return;
    // chunks c, c + WPR PAR, ... with a running maximum of their own, U on their way at a time
    constexpr int U = 8;
    float m = -INFINITY, l = 0;
    att_f32x4 o = {0, 0, 0, 0};
    const int d_in = d < p.dim ? d : 0;
    for (int c = (WPR == 1 ? 0 : wave * PAR) + sub; c < chunks; c += U * WPR * PAR) {
        float2 ml[U];
        att_f32x4 x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int at = c + u * WPR * PAR < chunks ? c + u * WPR * PAR : c;
            const int64_t slot = at < parts.shared ? parts.first_shared + at : parts.first_own + (int64_t)(at - parts.shared) * parts.stride_own;
            ml[u] = p.part_ml[slot];
            x[u] = *(const att_f32x4 *)(p.part + slot * p.dim + d_in);
        }
        float top = m;
#pragma unroll
        for (int u = 0; u < U; ++u)
            top = fmaxf(top, ml[u].x);
        const float base = top == -INFINITY ? 0.0f : top, f = __builtin_amdgcn_exp2f(m - base);
        m = top;
        l *= f;
        o *= f;
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (c + u * WPR * PAR < chunks) {
                const float g = __builtin_amdgcn_exp2f(ml[u].x - base);
                l += ml[u].y * g;
                o += x[u] * g;
            }
    }
#pragma unroll
    for (int off = LANES; off < 64; off <<= 1) {
        const float m2 = __shfl_xor(m, off), l2 = __shfl_xor(l, off), top = fmaxf(m, m2), base = top == -INFINITY ? 0.0f : top;
        const float f = __builtin_amdgcn_exp2f(m - base), f2 = __builtin_amdgcn_exp2f(m2 - base);
        m = top;
        l = l * f + l2 * f2;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            o[e] = o[e] * f + __shfl_xor(o[e], off) * f2;
    }
    if (WPR > 1) {
        __shared__ __align__(16) float lds[WPR][LANES * 4 + 4];
        if (sub == 0) {
            *(att_f32x4 *)&lds[wave][d] = o;
            if (d == 0) {
                lds[wave][LANES * 4] = m;
                lds[wave][LANES * 4 + 1] = l;
            }
        }
        __syncthreads();
        if (wave != 0)
            return;
        m = -INFINITY;
        l = 0;
        o = att_f32x4{0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < WPR; ++w)
            m = fmaxf(m, lds[w][LANES * 4]);
        const float base = m == -INFINITY ? 0.0f : m;
#pragma unroll
        for (int w = 0; w < WPR; ++w) {
            const float f = __builtin_amdgcn_exp2f(lds[w][LANES * 4] - base);
            l += lds[w][LANES * 4 + 1] * f;
            o += *(const att_f32x4 *)&lds[w][d] * f;
        }
    }
    if (sub != 0 || d >= p.dim)
        return;
    const float f = l == 0.0f ? 0.0f : 1.0f / l;
    const int64_t at = (int64_t)token * p.ldo + (int64_t)head * p.hso + d;
    if (BF16)
        *(uint2 *)((uint16_t *)p.out + at) = make_uint2(f32x2_to_bf16x2(o[0] * f, o[1] * f), f32x2_to_bf16x2(o[2] * f, o[3] * f));
    else
        *(att_f32x4 *)((float *)p.out + at) = o * f;
}

template <class P, bool BF16, int DB>
static int go_join(const P &p, int32_t most, hipStream_t st)
{
    const int64_t rows = (int64_t)p.tokens * p.n_heads;
    // A wavefront has 16 chunks of features on their way at a time (dim 128); of few rows with more, four share a row.  (One / four wavefronts a row, the whole call:
    // 256 rows of 60 chunks 34.4 / 31.4 us, 512 of 33 21.3 / 20.1, 32 of 32 10.3 / 9.9; 512 of 18 13.2 / 14.1, 1280 of 33 28.7 / 31.6.)
    if (rows <= 512 && most > 24)
        hipLaunchKernelGGL((attend_join_kernel<P, BF16, DB, 4>), dim3((uint32_t)rows), dim3(256), 0, st, p);
    else
        hipLaunchKernelGGL((attend_join_kernel<P, BF16, DB, 1>), dim3((uint32_t)((rows + 3) / 4)), dim3(256), 0, st, p);
    return check_launch("attend_join_kernel");
}

// most: chunks of a row; where the device cuts own parts, what they are on average, as no more is known here
template <class P>
static int launch_attend_join(const P &p, bool bf16, int32_t most, hipStream_t st)
{
    if (p.dim <= 64)
        return bf16 ? go_join<P, true, 64>(p, most, st) : go_join<P, false, 64>(p, most, st);
    if (p.dim <= 128)
        return bf16 ? go_join<P, true, 128>(p, most, st) : go_join<P, false, 128>(p, most, st);
    return bf16 ? go_join<P, true, 256>(p, most, st) : go_join<P, false, 256>(p, most, st);
}

}  // namespace griffin
