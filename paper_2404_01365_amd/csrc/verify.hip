// Verification of drafted tokens against the target's probabilities (griffin_verify_drafts).
//
// A sequence keeps its drafted tokens while u q(d) < p(d); where that ends a token is drawn from w = max(p - q, 0), or from p, by the inverse of the running
// sum: the first j with w_0 + .. + w_j > r W.  Sums are in 64 bits, so that their order does not decide which token that is.
//
// Only the row where the kept tokens end is read whole.  Its sum is taken in chunks by many workgroups, each of which finds that row for itself (a few numbers a
// drafted token); a second launch adds the chunks in order, finds the one that the sum falls into and goes through it again.
#include "layer.h"

namespace griffin {

constexpr int VERIFY_THREADS = 256;
constexpr int VERIFY_CHUNK = 4096;           // tokens of the vocabulary a workgroup adds up

struct VerifyParams {
    const float *p, *q;
    int64_t ldp, ldq;
    const int32_t *drafted;
    const float *accept_u, *draw_u;
    int32_t *tokens_out, *accepted, *lens_out;
    const int32_t *lens;
    double *sums;                            // [sequence][chunk] sums of w, then of p
    int32_t vocab, chunks;
    SeqTable seqs;
};

// Where a sequence's kept tokens end: its row, and what w is there
struct VerifyEnd {
    int32_t kept, row, without;              // without: the token that w leaves out (a draft without probabilities), or -1
    bool minus_q;
};

// by every wavefront for itself, 64 rows at a time
__device__ __forceinline__ VerifyEnd verify_end(const VerifyParams &p, int b)
{
    const int lane = threadIdx.x & 63;
    const int32_t first = p.seqs.cu[b], last = p.seqs.cu[b + 1] - 1;
    VerifyEnd e = {last - first, last, -1, false};
    for (int32_t at = first; at < last; at += 64) {
        const int32_t row = at + lane;
        bool kept = true;
        int32_t d = -1;
        if (row < last) {
            d = p.drafted[row];
            kept = d >= 0 && d < p.vocab;
            if (kept) {
                const float share = p.q ? p.q[row * p.ldq + d] : 1.0f;
                kept = p.accept_u[row] * share < p.p[row * p.ldp + d];
            }
        }
        const uint64_t stops = __ballot(!kept);
        if (stops) {
            const int l = __builtin_ctzll(stops);
            d = __builtin_amdgcn_readlane(d, l);
            e.row = at + l;
            e.kept = e.row - first;
            const bool is_draft = d >= 0 && d < p.vocab;
            e.minus_q = is_draft && p.q;
            e.without = is_draft && !p.q ? d : -1;
            break;
        }
    }
    return e;
}

// w of token j, and p
__device__ __forceinline__ float verify_weight(const VerifyParams &p, const VerifyEnd &e, int32_t j, float &whole)
{
    whole = p.p[e.row * p.ldp + j];
    if (e.minus_q)
        return fmaxf(whole - p.q[e.row * p.ldq + j], 0.0f);
    return j == e.without ? 0.0f : whole;
}

__device__ __forceinline__ double wave_sum64(double v)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1)
        v += __shfl_xor(v, off);
    return v;
}

__global__ __launch_bounds__(VERIFY_THREADS) void verify_sums_kernel(VerifyParams p)
{
    __shared__ double part[2][VERIFY_THREADS / 64];
    const int b = blockIdx.x / p.chunks, chunk = blockIdx.x - b * p.chunks;
    if (p.seqs.cu[b] == p.seqs.cu[b + 1])
        return;
    const VerifyEnd e = verify_end(p, b);
    double sum = 0, all = 0;
    const int32_t begin = chunk * VERIFY_CHUNK, end = begin + VERIFY_CHUNK < p.vocab ? begin + VERIFY_CHUNK : p.vocab;
    for (int32_t j = begin + threadIdx.x; j < end; j += VERIFY_THREADS) {
        float whole;
        sum += verify_weight(p, e, j, whole);
        all += whole;
    }
    sum = wave_sum64(sum);
    all = wave_sum64(all);
    if ((threadIdx.x & 63) == 0) {
        part[0][threadIdx.x >> 6] = sum;
        part[1][threadIdx.x >> 6] = all;
    }
    __syncthreads();
    if (threadIdx.x < 2) {
        double total = 0;
#pragma unroll
        for (int w = 0; w < VERIFY_THREADS / 64; ++w)
            total += part[threadIdx.x][w];
        p.sums[((int64_t)b * p.chunks + chunk) * 2 + threadIdx.x] = total;
    }
}

__global__ __launch_bounds__(VERIFY_THREADS) void verify_draw_kernel(VerifyParams p)
{
    const int b = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int32_t first = p.seqs.cu[b], rows = p.seqs.cu[b + 1] - first;
    if (rows == 0) {
        if (threadIdx.x == 0) {
            p.accepted[b] = 0;
            if (p.lens_out)
                p.lens_out[b] = p.lens[b];
        }
        return;
    }
    VerifyEnd e = verify_end(p, b);
    // the chunk that the goal falls into, by every thread alike
    const double *sums = p.sums + (int64_t)b * p.chunks * 2;
    double total = 0;
    for (int c = 0; c < p.chunks; ++c)
        total += sums[2 * c];
    int which = 0;
    if (!(total > 0)) {                      // nothing left over: the target's own probabilities
        which = 1;
        e.minus_q = false;
        e.without = -1;
        total = 0;
        for (int c = 0; c < p.chunks; ++c)
            total += sums[2 * c + 1];
    }
    const double goal = (double)p.draw_u[b] * total;
    double before = 0;
    int chunk = 0;
    for (; chunk < p.chunks; ++chunk) {
        if (before + sums[2 * chunk + which] > goal)
            break;
        before += sums[2 * chunk + which];
    }
    int32_t drawn = p.vocab - 1;
    if (chunk < p.chunks) {
        // 64 tokens a wavefront and 256 a workgroup at a time, sums carried on
        __shared__ double totals[VERIFY_THREADS / 64];
        __shared__ int32_t found;
        if (threadIdx.x == 0)
            found = INT32_MAX;
        const int32_t begin = chunk * VERIFY_CHUNK, end = begin + VERIFY_CHUNK < p.vocab ? begin + VERIFY_CHUNK : p.vocab;
        for (int32_t at = begin; at < end; at += VERIFY_THREADS) {
            const int32_t j = at + threadIdx.x;
            float whole;
            double run = j < end ? verify_weight(p, e, j, whole) : 0.0f;
#pragma unroll
            for (int off = 1; off < 64; off <<= 1) {
                const double other = __shfl_up(run, off);
                run += lane >= off ? other : 0.0;
            }
            __syncthreads();                 // everyone has read what the round before left
            if (lane == 63)
                totals[wave] = run;
            __syncthreads();
            double here = before;
            for (int w = 0; w < wave; ++w)
                here += totals[w];
            if (j < end && here + run > goal)
                atomicMin(&found, j);
            for (int w = 0; w < VERIFY_THREADS / 64; ++w)
                before += totals[w];
            __syncthreads();
            if (found != INT32_MAX)
                break;
        }
        // where the chunk's sum passes the goal and the running one, rounded otherwise, does not: its last token
        drawn = found != INT32_MAX ? found : end - 1;
    }
    for (int32_t i = threadIdx.x; i < rows; i += VERIFY_THREADS)
        p.tokens_out[first + i] = i < e.kept ? p.drafted[first + i] : i == e.kept ? drawn : -1;
    if (threadIdx.x == 0) {
        p.accepted[b] = e.kept;
        if (p.lens_out)
            p.lens_out[b] = p.lens[b] + e.kept + 1;
    }
}

static int32_t verify_chunks(int32_t vocab) { return (vocab + VERIFY_CHUNK - 1) / VERIFY_CHUNK; }

size_t verify_bytes(int32_t n_seqs, int32_t vocab) { return (size_t)n_seqs * verify_chunks(vocab) * 2 * sizeof(double); }

int launch_verify(const VerifyJob &job, const SeqTable &seqs, hipStream_t st)
{
    VerifyParams p = {};
    p.p = job.p; p.q = job.q; p.ldp = job.ldp; p.ldq = job.ldq; p.drafted = job.drafted;
    p.accept_u = job.accept_u; p.draw_u = job.draw_u; p.tokens_out = job.tokens_out; p.accepted = job.accepted;
    p.lens = job.lens; p.lens_out = job.lens_out; p.sums = job.ws;
    p.vocab = job.vocab;
    p.chunks = verify_chunks(job.vocab);
    p.seqs = seqs;
    hipLaunchKernelGGL(verify_sums_kernel, dim3((uint32_t)seqs.n * p.chunks), dim3(VERIFY_THREADS), 0, st, p);
    const int rc = check_launch("verify_sums_kernel");
    if (rc != GRIFFIN_OK)
        return rc;
    hipLaunchKernelGGL(verify_draw_kernel, dim3(seqs.n), dim3(VERIFY_THREADS), 0, st, p);
    return check_launch("verify_draw_kernel");
}

}  // namespace griffin
