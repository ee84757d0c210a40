// Verification of drafted tokens against the target's probabilities (griffin_verify_drafts).
//
// A sequence keeps its drafted tokens while u q(d) < p(d); where that ends a token is drawn from w = max(p - q, 0), or from p, by the inverse of the running
// sum: the first j with w_0 + .. + w_j > r W.  Sums are in 64 bits, so that their order does not decide which token that is.
//
// Only the row where the kept tokens end is read whole.  A wavefront adds up a piece of 1024 tokens of it, and finds that row for itself (a few numbers a drafted token); then
// a workgroup a sequence adds the pieces in order, finds the one that the sum falls into and goes through it again: in a launch of its own, or, of small vocabularies, in the same.
//
// Bound by latencies while there are few tokens (one sequence of 32000: 9.8 us, a launch, two steps of dependent loads to find the row, two of its pieces, one again), else by bytes: 64
// sequences of 128001, p and q, 66 MB, 11.4 + 5.3 us, and 13.1 + 5.0 where 1.3 GB of states take turns.
#include "layer.h"

namespace griffin {

constexpr int VERIFY_THREADS = 256;
constexpr int VERIFY_ALONE = 1024;           // ... of a workgroup that does all of a sequence
constexpr int VERIFY_ALONE_PIECES = 32;      // ... which has no more than so many pieces
constexpr int VERIFY_PIECE = 1024;           // tokens of the vocabulary a wavefront adds up

// Where a sequence's kept tokens end: its row, and what w is there
struct VerifyEnd {
    int32_t kept, row, without;              // without: the token that w leaves out (a draft without probabilities), or -1
    int32_t minus_q;
};

struct VerifyParams {
    const float *p, *q;
    int64_t ldp, ldq;
    const int32_t *drafted;
    const float *accept_u, *draw_u;
    int32_t *tokens_out, *accepted, *lens_out;
    const int32_t *lens;
    VerifyEnd *ends;                         // [sequence], left by the first launch
    double *sums;                            // [sequence][piece] sums of w
    int32_t vocab, pieces, blocks;           // workgroups a sequence
    bool wide;                               // rows in 16 bytes
    SeqTable seqs;
};

// by every wavefront for itself, 64 rows at a time
__device__ __forceinline__ VerifyEnd verify_end(const VerifyParams &p, int b)
{
    const int lane = threadIdx.x & 63;
    const int32_t first = p.seqs.cu[b], last = p.seqs.cu[b + 1] - 1;
    VerifyEnd e = {last - first, last, -1, 0};
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

// w of N consecutive tokens from j on, zero behind the vocabulary's end
template <int N>
__device__ __forceinline__ void verify_weights(const VerifyParams &p, const VerifyEnd &e, int32_t j, float (&w)[N])
{
    const float *at = p.p + e.row * p.ldp + j, *less = p.q + (e.minus_q ? e.row * p.ldq + j : 0);
    float q[N];
    if (N == 4 && p.wide && j + 4 <= p.vocab) {
        *(float4 *)w = *(const float4 *)at;
        if (e.minus_q)
            *(float4 *)q = *(const float4 *)less;
    } else
#pragma unroll
        for (int i = 0; i < N; ++i) {
            w[i] = j + i < p.vocab ? at[i] : 0.0f;
            if (e.minus_q)
                q[i] = j + i < p.vocab ? less[i] : 0.0f;
        }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (e.minus_q)
            w[i] = fmaxf(w[i] - q[i], 0.0f);
        w[i] = j + i == e.without ? 0.0f : w[i];
    }
}

// a piece's sum of w, by a wavefront; every lane ends with it
__device__ __forceinline__ double verify_piece(const VerifyParams &p, const VerifyEnd &e, int32_t piece)
{
    const int lane = threadIdx.x & 63;
    const int32_t begin = piece * VERIFY_PIECE;
    double sum = 0;
    const auto add = [&](auto &w) {
#pragma unroll
        for (auto &v : w)
#pragma unroll
            for (float x : v)
                sum += x;
    };
    if (p.wide) {
        float w[VERIFY_PIECE / 256][4];
#pragma unroll
        for (int i = 0; i < VERIFY_PIECE / 256; ++i)
            verify_weights(p, e, begin + (i * 64 + lane) * 4, w[i]);
        add(w);
    } else {
        float w[VERIFY_PIECE / 64][1];
#pragma unroll
        for (int i = 0; i < VERIFY_PIECE / 64; ++i)
            verify_weights(p, e, begin + i * 64 + lane, w[i]);
        add(w);
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1)
        sum += __shfl_xor(sum, off);
    return sum;
}

__global__ __launch_bounds__(VERIFY_THREADS) void verify_sums_kernel(VerifyParams p)
{
    const int b = blockIdx.x / p.blocks, lane = threadIdx.x & 63;
    const int32_t piece = (blockIdx.x - b * p.blocks) * (VERIFY_THREADS / 64) + (threadIdx.x >> 6);
    if (p.seqs.cu[b] == p.seqs.cu[b + 1] || piece >= p.pieces)
        return;
    const VerifyEnd e = verify_end(p, b);
    if (piece == 0 && lane == 0)
        p.ends[b] = e;
    const double sum = verify_piece(p, e, piece);
    if (lane == 0)
        p.sums[(int64_t)b * p.pieces + piece] = sum;
}

// The sum of what the threads before have, and of all; called by all threads of a workgroup
template <int THREADS>
__device__ __forceinline__ double verify_before(double v, double &all)
{
    __shared__ double totals[THREADS / 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    double run = v;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const double other = __shfl_up(run, off);
        run += lane >= off ? other : 0.0;
    }
    __syncthreads();                         // everyone has read what a call before left
    if (lane == 63)
        totals[wave] = run;
    __syncthreads();
    double before = 0;
    all = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
        before += w < wave ? totals[w] : 0.0;
        all += totals[w];
    }
    const double other = __shfl_up(run, 1);
    return before + (lane > 0 ? other : 0.0);
}

// the least of the threads' numbers
template <int THREADS>
__device__ __forceinline__ int32_t verify_least(int32_t v)
{
    __shared__ int32_t least[THREADS / 64];
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
        const int32_t other = __shfl_xor(v, off);
        v = other < v ? other : v;
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 0)
        least[threadIdx.x >> 6] = v;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w)
        v = least[w] < v ? least[w] : v;
    return v;
}

// The first token of a piece that has weight and whose running sum, with what comes before, passes the goal.  None does: VERIFY_LAST - j, more than any token, with j the piece's last token that
// has weight; INT32_MAX: none has.  (Weight is asked for, as the sum ahead of a thread's first token is added in another order than the one behind the thread before, and may pass the goal by a
// rounding where that did not.)  `before` is carried on.
constexpr int32_t VERIFY_LAST = INT32_MAX - 1;
template <int THREADS>
__device__ __forceinline__ int32_t verify_find(const VerifyParams &p, const VerifyEnd &e, int32_t begin, double goal, double &before)
{
    constexpr int N = VERIFY_PIECE / THREADS;
    const int32_t j = begin + threadIdx.x * N;
    float w[N];
    verify_weights(p, e, j, w);
    double all, mine = 0;
#pragma unroll
    for (int i = 0; i < N; ++i)
        mine += w[i];
    double run = verify_before<THREADS>(mine, all) + before;
    int32_t found = INT32_MAX;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        run += w[i];
        if (found >= p.vocab && w[i] > 0)
            found = run > goal ? j + i : VERIFY_LAST - (j + i);
    }
    before += all;
    return verify_least<THREADS>(found);
}

// Sequence b's outcome, from where its kept tokens end and the pieces' sums there; called by all threads of a workgroup
template <int THREADS>
__device__ __forceinline__ void verify_draw(const VerifyParams &p, int b, VerifyEnd e, const double *sums)
{
    const int32_t first = p.seqs.cu[b], rows = p.seqs.cu[b + 1] - first;
    const float u = p.draw_u[b];              // widened where it is used: a register less in between
    // a thread takes as many pieces as its share is, one behind the other
    const int32_t share = (p.pieces + THREADS - 1) / THREADS, from = threadIdx.x * share;
    const int32_t to = from + share < p.pieces ? from + share : p.pieces;
    double mine = 0, total;
    for (int32_t i = from; i < to; ++i)
        mine += sums[i];
    double before = verify_before<THREADS>(mine, total);
    int32_t drawn = INT32_MAX;
    if (total > 0) {
        const double goal = (double)u * total;
        int32_t piece = INT32_MAX;
        double run = before;
        for (int32_t i = from; i < to; ++i) {
            if (sums[i] > 0 && run + sums[i] > goal) {
                piece = i;
                break;
            }
            run += sums[i];
        }
        __shared__ double start;
        const int32_t least = verify_least<THREADS>(piece);
        if (piece == least && piece != INT32_MAX)        // one thread's
            start = run;
        __syncthreads();
        if (least != INT32_MAX) {
            before = start;
            drawn = verify_find<THREADS>(p, e, least * VERIFY_PIECE, goal, before);
            // where the piece's sum passes the goal and the running one, rounded otherwise, does not: its last token with weight
            drawn = drawn < p.vocab ? drawn : VERIFY_LAST - drawn;
        }
    } else {
        // nothing left over: the target's own probabilities, by this workgroup alone
        e.minus_q = 0;
        e.without = -1;
        before = 0;
        for (int32_t at = 0; at < p.vocab; at += VERIFY_PIECE)
            verify_find<THREADS>(p, e, at, INFINITY, before);
        const double goal = (double)u * before;
        before = 0;
        for (int32_t at = 0; at < p.vocab && drawn >= p.vocab; at += VERIFY_PIECE)
            drawn = verify_find<THREADS>(p, e, at, goal, before);
    }
    drawn = drawn < p.vocab ? drawn : p.vocab - 1;
    for (int32_t i = threadIdx.x; i < rows; i += THREADS)
        p.tokens_out[first + i] = i < e.kept ? p.drafted[first + i] : i == e.kept ? drawn : -1;
    if (threadIdx.x == 0) {
        p.accepted[b] = e.kept;
        if (p.lens_out)
            p.lens_out[b] = p.lens[b] + e.kept + 1;
    }
}

// true, and done: a sequence without rows
__device__ __forceinline__ bool verify_nothing(const VerifyParams &p, int b)
{
    if (p.seqs.cu[b] != p.seqs.cu[b + 1])
        return false;
    if (threadIdx.x == 0) {
        p.accepted[b] = 0;
        if (p.lens_out)
            p.lens_out[b] = p.lens[b];
    }
    return true;
}

__global__ __launch_bounds__(VERIFY_THREADS) void verify_draw_kernel(VerifyParams p)
{
    const int b = blockIdx.x;
    if (!verify_nothing(p, b))
        verify_draw<VERIFY_THREADS>(p, b, p.ends[b], p.sums + (int64_t)b * p.pieces);
}

// All of a sequence whose vocabulary is no more than VERIFY_ALONE_PIECES pieces: sixteen wavefronts take them in turn
__global__ __launch_bounds__(VERIFY_ALONE) void verify_alone_kernel(VerifyParams p)
{
    __shared__ double sums[VERIFY_ALONE_PIECES];
    const int b = blockIdx.x;
    if (verify_nothing(p, b))
        return;
    const VerifyEnd e = verify_end(p, b);
    for (int32_t piece = threadIdx.x >> 6; piece < p.pieces; piece += VERIFY_ALONE / 64) {
        const double sum = verify_piece(p, e, piece);
        if ((threadIdx.x & 63) == 0)
            sums[piece] = sum;
    }
    __syncthreads();
    verify_draw<VERIFY_ALONE>(p, b, e, sums);
}

static int32_t verify_pieces(int32_t vocab) { return (vocab + VERIFY_PIECE - 1) / VERIFY_PIECE; }

// Vocabularies of up to 32768 tokens go in one launch, a workgroup a sequence.  (One launch / two, us a call: one sequence of 4000 9.0 / 11.9, of 32000 10.4 / 13.2, of 65536 12.6 / 11.8, 16 of 50257
// 12.5 / 11.5, 64 of 32000 12.1 / 12.0, of 65536 16.6 / 12.8, 256 of 32000 14.7 / 15.7.)
static bool verify_alone(int32_t vocab) { return verify_pieces(vocab) <= VERIFY_ALONE_PIECES; }

size_t verify_bytes(int32_t n_seqs, int32_t vocab)
{
    static_assert(sizeof(VerifyEnd) == 2 * sizeof(double), "the sums behind the ends are aligned");
    if (verify_alone(vocab))
        return 0;
    return (size_t)n_seqs * (verify_pieces(vocab) * sizeof(double) + sizeof(VerifyEnd));
}

int launch_verify(const VerifyJob &job, const SeqTable &seqs, hipStream_t st)
{
    VerifyParams p = {};
    p.p = job.p; p.q = job.q; p.ldp = job.ldp; p.ldq = job.ldq; p.drafted = job.drafted;
    p.accept_u = job.accept_u; p.draw_u = job.draw_u; p.tokens_out = job.tokens_out; p.accepted = job.accepted;
    p.lens = job.lens; p.lens_out = job.lens_out;
    const bool alone = verify_alone(job.vocab);
    if (!alone) {
        p.ends = (VerifyEnd *)job.ws;
        p.sums = job.ws + 2 * seqs.n;
    }
    p.vocab = job.vocab;
    p.pieces = verify_pieces(job.vocab);
    p.blocks = (p.pieces + VERIFY_THREADS / 64 - 1) / (VERIFY_THREADS / 64);
    const auto wide = [](const float *at, int64_t ld) { return !at || (((uintptr_t)at & 15) == 0 && ld % 4 == 0); };
    p.wide = wide(job.p, job.ldp) && wide(job.q, job.ldq);
    p.seqs = seqs;
    if (alone) {
        hipLaunchKernelGGL(verify_alone_kernel, dim3(seqs.n), dim3(VERIFY_ALONE), 0, st, p);
        return check_launch("verify_alone_kernel");
    }
    hipLaunchKernelGGL(verify_sums_kernel, dim3((uint32_t)seqs.n * p.blocks), dim3(VERIFY_THREADS), 0, st, p);
    const int rc = check_launch("verify_sums_kernel");
    if (rc != GRIFFIN_OK)
        return rc;
    hipLaunchKernelGGL(verify_draw_kernel, dim3(seqs.n), dim3(VERIFY_THREADS), 0, st, p);
    return check_launch("verify_draw_kernel");
}

}  // namespace griffin
