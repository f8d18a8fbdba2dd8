// Verification of drafted tokens: accept while the given random number times the draft's probability stays below the target's, then draw
// one token from what is left of the target.
//
// A product of two fp32 numbers is exact in fp64, so the acceptance is decided without rounding.  What is left, max(p - q, 0), and its sums are
// held in fp64: a sum of 10^5 terms moves the borders between tokens by about 1e-16 of the total.
#include "internal.h"

namespace det {

constexpr int kVerifyThreads = 1024, kVerifyWaves = kVerifyThreads / kWave, kVerifyDrafts = 64;

__device__ __forceinline__ double wave_sum_f64(double v)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v = v + __shfl_xor(v, off, kWave);
    return v;
}

// What is left of token j: p_j - q_j (q null: p_j) where that is positive, else 0 (NaN too).
__device__ __forceinline__ double left_over(const float* p, const float* q, int j)
{
    const double d = q ? (double)p[j] - (double)q[j] : (double)p[j];
    return d > 0.0 ? d : 0.0;
}

// One workgroup a sequence.  Each wave sums a contiguous sixteenth of the row; the sixteenth that holds the target is then read again, a contiguous
// run a thread.
__global__ __launch_bounds__(kVerifyThreads) void verify_kernel(const float* __restrict__ p, const float* __restrict__ q,
                                                                const int32_t* __restrict__ drafts, const int32_t* __restrict__ n_drafts,
                                                                const float* __restrict__ u, int32_t* __restrict__ accepted,
                                                                int32_t* __restrict__ tokens, int N, int V)
{
    __shared__ double sums[kVerifyWaves];
    __shared__ double before[kVerifyWaves];
    __shared__ int found[kVerifyWaves];
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int n = min(max(n_drafts ? n_drafts[b] : N, 0), N);

    // every wave decides the acceptance for itself: lane i has draft i
    bool ok = false;
    int32_t draft = -1;
    if (lane < n) {
        draft = drafts[(size_t)b * N + lane];
        if ((unsigned)draft < (unsigned)V) {
            const double px = p[((size_t)b * (N + 1) + lane) * V + draft];
            const double qx = q ? q[((size_t)b * N + lane) * V + draft] : 1.0;
            ok = (double)u[(size_t)b * (N + 1) + lane] * qx < px;
        }
    }
    const int take = __builtin_ctzll(~__ballot(ok) | (1ull << n));
    const float* pr = p + ((size_t)b * (N + 1) + take) * V;
    const float* qr = q && take < n ? q + ((size_t)b * N + take) * V : nullptr;
    // without the draft's probabilities the drafted token was certain: it takes no part in the second draw
    const int barred = !q && take < n ? __builtin_amdgcn_readlane(draft, take) : -1;

    const int part = (V + kVerifyWaves - 1) / kVerifyWaves;
    double total = 0.0;
    bool plain = false;  // nothing is left of p - q: the token comes from p itself
    for (int pass = 0; pass < 2; ++pass) {
        double s = 0.0;
        const int end = min((wave + 1) * part, V);
        for (int j = wave * part + lane; j < end; j += kWave) s = s + (j == barred && !plain ? 0.0 : left_over(pr, plain ? nullptr : qr, j));
        s = wave_sum_f64(s);
        __syncthreads();
        if (lane == 0) sums[wave] = s;
        __syncthreads();
        total = 0.0;
        for (int w = 0; w < kVerifyWaves; ++w) total = total + sums[w];
        if (total > 0.0 || plain) break;
        plain = true;
    }
    const double target = (double)u[(size_t)b * (N + 1) + N] * total;
    // the part of the row that holds the target: the first whose end lies beyond it, else the last that is not empty
    int at = 0;
    double start = 0.0, sum = 0.0;
    for (int w = 0; w < kVerifyWaves; ++w) {
        if (sums[w] > 0.0) {
            at = w;
            start = sum;
        }
        sum = sum + sums[w];
        if (sum > target) break;
    }
    // again, a run of it for each thread
    const int first = at * part, last = min(first + part, V), run = (part + kVerifyThreads - 1) / kVerifyThreads;
    const int from = min(first + tid * run, last), to = min(from + run, last);
    auto value = [&](int j) { return j == barred && !plain ? 0.0 : left_over(pr, plain ? nullptr : qr, j); };
    double mine = 0.0;
    for (int j = from; j < to; ++j) mine = mine + value(j);
    double up = mine;  // sums of the lanes up to this one
#pragma unroll
    for (int off = 1; off < kWave; off <<= 1) {
        const double other = __shfl_up(up, off, kWave);
        if (lane >= off) up = up + other;
    }
    if (lane == kWave - 1) before[wave] = up;
    __syncthreads();
    double base = start;
    for (int w = 0; w < wave; ++w) base = base + before[w];
    base = base + (up - mine);
    int token = -1;  // the first token of this run whose end lies beyond the target, else (negative, less 2) its last that is not empty
    double c = base;
    for (int j = from; j < to; ++j) {
        const double x = value(j);
        c = c + x;
        if (x > 0.0) {
            token = c > target ? j : -2 - j;
            if (token >= 0) break;
        }
    }
    // the lowest token that was found in any run, else the highest that is not empty
    int best = token >= 0 ? token : 0x7FFFFFFF, rest = token < -1 ? -2 - token : -1;
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
        best = min(best, __shfl_xor(best, off, kWave));
        rest = max(rest, __shfl_xor(rest, off, kWave));
    }
    if (lane == 0) found[wave] = best < 0x7FFFFFFF ? best : -2 - rest;
    __syncthreads();
    if (tid == 0) {
        best = 0x7FFFFFFF;
        rest = 0;
        for (int w = 0; w < kVerifyWaves; ++w) {
            const int f = found[w];
            if (f >= 0) best = min(best, f);
            else rest = max(rest, -2 - f);
        }
        accepted[b] = take;
        tokens[(size_t)b * (N + 1) + take] = best < 0x7FFFFFFF ? best : rest;
    }
    if (tid <= N && tid != take) tokens[(size_t)b * (N + 1) + tid] = tid < take ? draft : -1;
}

}  // namespace det

using namespace det;

extern "C" int det_verify_drafts(const float* p, const float* q, const int32_t* drafts, const int32_t* n_drafts, const float* u,
                                 int32_t* accepted, int32_t* tokens, int B, int N, int V, void* stream)
{
    if (!p || !drafts || !u || !accepted || !tokens || B < 1 || N < 1 || V < 1) return DET_EINVAL;
    if (N >= kVerifyDrafts || V > (1 << 30)) return DET_ESHAPE;
    if (!aligned16(p) || (q && !aligned16(q))) return DET_EALIGN;
    hipLaunchKernelGGL(verify_kernel, dim3(B), dim3(kVerifyThreads), 0, static_cast<hipStream_t>(stream), p, q, drafts, n_drafts, u, accepted,
                       tokens, N, V);
    return check_launch();
}
