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

// What the token is drawn from: p_j - q_j (q null: p_j) where that is positive, else 0 (NaN too); nothing of token `barred`.
struct left_over {
    const float* p;
    const float* q;
    int barred;
    __device__ __forceinline__ double of(float pj, float qj, int j) const
    {
        const double d = (double)pj - (double)qj;
        return d > 0.0 && j != barred ? d : 0.0;
    }
    __device__ __forceinline__ double operator()(int j) const { return of(p[j], q ? q[j] : 0.0f, j); }
};

// Sum over the tokens from..to-1 (VEC: rows lie on 16 bytes, `from` is a multiple of four), the same in every lane.  A lane asks for sixteen values
// of either row before it uses the first.
template <bool VEC>
__device__ __forceinline__ double wave_sum(const left_over& left, int from, int to)
{
    constexpr int W = VEC ? 4 : 1, AHEAD = VEC ? 4 : 16;
    const int lane = threadIdx.x & 63;
    double s = 0.0;
    int j = from;
    for (; j + 64 * W * AHEAD <= to; j += 64 * W * AHEAD) {
        float p[AHEAD * W], q[AHEAD * W];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int at = j + 64 * W * k + W * lane;
            if constexpr (VEC) {
                const float4 x = *reinterpret_cast<const float4*>(left.p + at);
                const float4 y = left.q ? *reinterpret_cast<const float4*>(left.q + at) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                p[4 * k] = x.x, p[4 * k + 1] = x.y, p[4 * k + 2] = x.z, p[4 * k + 3] = x.w;
                q[4 * k] = y.x, q[4 * k + 1] = y.y, q[4 * k + 2] = y.z, q[4 * k + 3] = y.w;
            } else {
                p[k] = left.p[at];
                q[k] = left.q ? left.q[at] : 0.0f;
            }
        }
#pragma unroll
        for (int k = 0; k < AHEAD * W; ++k) s = s + left.of(p[k], q[k], j + 64 * W * (k / W) + W * lane + k % W);
    }
    for (j += lane; j < to; j += 64) s = s + left(j);
    return wave_sum_f64(s);
}

// One workgroup a sequence.  Each wave sums a contiguous sixteenth of the row; the sixteenth that holds the target is cut into sixteenths again until
// one wave can hold what is left.  Bound by how fast one compute unit reads two rows: where there are few sequences most of the chip idles, which a
// second launch over parts of rows would cost more than it gives below some hundred thousand tokens.
template <bool VEC>
__global__ __launch_bounds__(kVerifyThreads) void verify_kernel(const float* __restrict__ p, const float* __restrict__ q,
                                                                const int32_t* __restrict__ drafts, const int32_t* __restrict__ n_drafts,
                                                                const float* __restrict__ u, int32_t* __restrict__ accepted,
                                                                int32_t* __restrict__ tokens, int N, int V)
{
    __shared__ double sums[2][kVerifyWaves];
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
    // without the draft's probabilities the drafted token was certain: it takes no part in the second draw
    left_over left{p + ((size_t)b * (N + 1) + take) * V, q && take < n ? q + ((size_t)b * N + take) * V : nullptr,
                   !q && take < n ? __builtin_amdgcn_readlane(draft, take) : -1};

    // from..to-1 holds the target; before: the sum of what lies in front of it
    int from = 0, to = V;
    double before = 0.0, target = 0.0;
    bool plain = false, first = true;
    for (int level = 0;; ++level) {
        if (!first && to - from <= 512) break;
        const int part = ((to - from + kVerifyWaves - 1) / kVerifyWaves + 3) & ~3;
        const int begin = min(from + wave * part, to);
        const double s = wave_sum<VEC>(left, begin, min(begin + part, to));
        double* mine = sums[level & 1];  // the other half is still read by waves that are behind
        if (lane == 0) mine[wave] = s;
        __syncthreads();
        if (first) {
            double total = 0.0;
            for (int w = 0; w < kVerifyWaves; ++w) total = total + mine[w];
            if (!(total > 0.0) && !plain) {  // nothing is left of p - q: the token comes from p itself
                plain = true;
                left.q = nullptr;
                left.barred = -1;
                continue;
            }
            target = (double)u[(size_t)b * (N + 1) + N] * total;
            first = false;
        }
        // the first part whose end lies beyond the target, else the last that is not empty
        int at = 0;
        double start = before, sum = before;
        for (int w = 0; w < kVerifyWaves; ++w) {
            if (mine[w] > 0.0) {
                at = w;
                start = sum;
            }
            sum = sum + mine[w];
            if (sum > target) break;
        }
        before = start;
        from = min(from + at * part, to);
        to = min(from + part, to);
    }
    if (wave != 0) return;

    // a run of up to eight tokens a lane
    const int run = (to - from + 63) / 64, mine = min(from + lane * run, to), end = min(mine + run, to);
    double x[8], own = 0.0;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        x[k] = mine + k < end ? left(mine + k) : 0.0;
        own = own + x[k];
    }
    double c = own;  // sums of the lanes up to this one
#pragma unroll
    for (int off = 1; off < kWave; off <<= 1) {
        const double other = __shfl_up(c, off, kWave);
        if (lane >= off) c = other + c;
    }
    c = before + (c - own);
    int best = 0x7FFFFFFF, rest = -1;  // the lowest token whose end lies beyond the target; the highest that is not empty
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        c = c + x[k];
        if (x[k] > 0.0) {
            rest = mine + k;
            if (c > target) best = min(best, mine + k);
        }
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
        best = min(best, __shfl_xor(best, off, kWave));
        rest = max(rest, __shfl_xor(rest, off, kWave));
    }
    const int token = best < 0x7FFFFFFF ? best : max(rest, 0);
    if (lane == 0) accepted[b] = take;
    if (lane <= N) tokens[(size_t)b * (N + 1) + lane] = lane < take ? draft : (lane == take ? token : -1);
}

}  // namespace det

using namespace det;

extern "C" int det_verify_drafts(const float* p, const float* q, const int32_t* drafts, const int32_t* n_drafts, const float* u,
                                 int32_t* accepted, int32_t* tokens, int B, int N, int V, void* stream)
{
    if (!p || !drafts || !u || !accepted || !tokens || B < 1 || N < 1 || V < 1) return DET_EINVAL;
    if (N >= kVerifyDrafts || V > (1 << 30)) return DET_ESHAPE;
    if (!aligned16(p) || (q && !aligned16(q))) return DET_EALIGN;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (V % 4 == 0) hipLaunchKernelGGL(verify_kernel<true>, dim3(B), dim3(kVerifyThreads), 0, s, p, q, drafts, n_drafts, u, accepted, tokens, N, V);
    else hipLaunchKernelGGL(verify_kernel<false>, dim3(B), dim3(kVerifyThreads), 0, s, p, q, drafts, n_drafts, u, accepted, tokens, N, V);
    return check_launch();
}
