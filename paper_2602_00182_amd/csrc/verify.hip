// Verification of drafted tokens: accept while the given random number times the draft's probability stays below the target's, then draw
// one token from what is left of the target.
//
// A product of two fp32 numbers is exact in fp64, so the acceptance is decided without rounding.  What is left, max(p - q, 0), and its sums are
// held in fp64: a sum of 10^5 terms moves the borders between tokens by about 1e-16 of the total.
//
// Two launches: parts of 2048 tokens are summed by a workgroup each, then one workgroup a sequence finds the part that holds the target and reads it
// again.  One workgroup for a whole row (one launch) is bound by what one compute unit can ask for: 64 sequences of 128000 tokens took 36 us, as many as this way take 19 (the sums 14, the pick 6, which is
// four trips to memory one after the other).
#include "internal.h"

namespace det {

constexpr int kVerifyDrafts = 64, kPartTokens = 2048, kRunTokens = kPartTokens / kBlock;

struct verify_args {
    const float* p;           // [B, N+1, V]
    const float* q;           // [B, N, V] or null
    const int32_t* drafts;    // [B, N]
    const int32_t* n_drafts;  // [B] or null
    const float* u;           // [B, N+1]
    int32_t* accepted;
    int32_t* tokens;
    double2* parts;           // [B, n_parts]: the sums of max(p - q, 0) and of max(p, 0)
    int N, V, n_parts;
};

// What a sequence's last token is drawn from: p_j - q_j (q null: p_j) where that is positive, else 0 (NaN too); nothing of token `barred`, which
// is one only where q is null: without the draft's probabilities a rejected draft was certain.
struct left_over {
    const float* p;
    const float* q;
    int barred;
    __device__ __forceinline__ double of(float pj, float qj, int j) const { return j == barred ? 0.0 : __builtin_fmax((double)pj - (double)qj, 0.0); }
};

// The number of accepted drafts (lane i of a wave decides draft i) and this lane's draft.
__device__ __forceinline__ int accept_drafts(const verify_args& a, int b, int32_t& draft, left_over& left)
{
    const int lane = threadIdx.x & 63, n = min(max(a.n_drafts ? a.n_drafts[b] : a.N, 0), a.N);
    bool ok = false;
    draft = -1;
    if (lane < n) {
        draft = a.drafts[(size_t)b * a.N + lane];
        if ((unsigned)draft < (unsigned)a.V) {
            const double px = a.p[((size_t)b * (a.N + 1) + lane) * a.V + draft];
            const double qx = a.q ? a.q[((size_t)b * a.N + lane) * a.V + draft] : 1.0;
            ok = (double)a.u[(size_t)b * (a.N + 1) + lane] * qx < px;
        }
    }
    const int take = __builtin_ctzll(~__ballot(ok) | (1ull << n));
    left.p = a.p + ((size_t)b * (a.N + 1) + take) * a.V;
    left.q = a.q && take < n ? a.q + ((size_t)b * a.N + take) * a.V : nullptr;
    left.barred = !a.q && take < n ? __builtin_amdgcn_readlane(draft, take) : -1;
    return take;
}

// Eight neighbouring tokens of a row from j on, zeros past V.  VEC: rows lie on 16 bytes.
template <bool VEC>
__device__ __forceinline__ void load_run(const float* row, int j, int V, float (&x)[kRunTokens])
{
    if (VEC && j + kRunTokens <= V) {
        const float4 a = *reinterpret_cast<const float4*>(row + j), b = *reinterpret_cast<const float4*>(row + j + 4);
        x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
    } else {
#pragma unroll
        for (int k = 0; k < kRunTokens; ++k) x[k] = j + k < V ? row[j + k] : 0.0f;
    }
}
template <bool VEC>
__device__ __forceinline__ void load_left(const left_over& left, int j, int V, float (&p)[kRunTokens], float (&q)[kRunTokens])
{
    load_run<VEC>(left.p, j, V, p);
#pragma unroll
    for (int k = 0; k < kRunTokens; ++k) q[k] = 0.0f;
    if (left.q) load_run<VEC>(left.q, j, V, q);
}

__device__ __forceinline__ double wave_sum_f64(double v)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v = v + __shfl_xor(v, off, kWave);
    return v;
}

// Grid (parts, B).
template <bool VEC>
__global__ __launch_bounds__(kBlock) void verify_parts_kernel(verify_args a)
{
    __shared__ double2 sums[kBlock / kWave];
    const int b = blockIdx.y, j = blockIdx.x * kPartTokens + kRunTokens * (int)threadIdx.x;
    int32_t draft;
    left_over left;
    accept_drafts(a, b, draft, left);
    float p[kRunTokens], q[kRunTokens];
    load_left<VEC>(left, j, a.V, p, q);
    double s = 0.0, plain = 0.0;
#pragma unroll
    for (int k = 0; k < kRunTokens; ++k) {
        s = s + left.of(p[k], q[k], j + k);
        plain = plain + __builtin_fmax((double)p[k], 0.0);
    }
    s = wave_sum_f64(s);
    plain = wave_sum_f64(plain);
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = make_double2(s, plain);
    __syncthreads();
    if (threadIdx.x == 0)
        a.parts[(size_t)b * a.n_parts + blockIdx.x] = make_double2((sums[0].x + sums[1].x) + (sums[2].x + sums[3].x), (sums[0].y + sums[1].y) + (sums[2].y + sums[3].y));
}

// The thread of the workgroup whose run holds the target: the first that is not empty with before + (sums of the runs up to its own) > target, else the last whose run
// is not empty, else thread 0.  start: the sum in front of the run of the calling thread.
__device__ __forceinline__ int find_run(double mine, double before, double target, double& start, double (&wave_sums)[kBlock / kWave],
                                        int (&firsts)[kBlock / kWave], int (&lasts)[kBlock / kWave])
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    double up = mine;  // sums of the lanes up to this one
#pragma unroll
    for (int off = 1; off < kWave; off <<= 1) {
        const double other = __shfl_up(up, off, kWave);
        if (lane >= off) up = other + up;
    }
    __syncthreads();  // earlier readers are done
    if (lane == kWave - 1) wave_sums[wave] = up;
    __syncthreads();
    double front = before;
    for (int w = 0; w < wave; ++w) front = front + wave_sums[w];
    start = front + (up - mine);
    // (an empty run is never taken: sums that take another way through the scan may differ in their last bit)
    const unsigned long long past = __ballot(front + up > target && mine > 0.0), full = __ballot(mine > 0.0);
    if (lane == 0) {
        firsts[wave] = past ? 64 * wave + __builtin_ctzll(past) : -1;
        lasts[wave] = full ? 64 * wave + 63 - __builtin_clzll(full) : -1;
    }
    __syncthreads();
    int at = 0;
    for (int w = 0; w < kBlock / kWave; ++w) at = lasts[w] >= 0 ? lasts[w] : at;
    for (int w = kBlock / kWave - 1; w >= 0; --w) at = firsts[w] >= 0 ? firsts[w] : at;
    return at;
}

// Grid (B).
template <bool VEC>
__global__ __launch_bounds__(kBlock) void verify_pick_kernel(verify_args a)
{
    __shared__ double wave_sums[kBlock / kWave], found_start;
    __shared__ int firsts[kBlock / kWave], lasts[kBlock / kWave], found_part;
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
    int32_t draft;
    left_over left;
    const int take = accept_drafts(a, b, draft, left);

    // a run of parts for each thread
    const double2* parts = a.parts + (size_t)b * a.n_parts;
    const int per = (a.n_parts + kBlock - 1) / kBlock, from = min(tid * per, a.n_parts), to = min(from + per, a.n_parts);
    double s = 0.0, plain = 0.0;
    for (int i = from; i < to; ++i) {
        s = s + parts[i].x;
        plain = plain + parts[i].y;
    }
    auto total_of = [&](double x) {
        x = wave_sum_f64(x);
        __syncthreads();
        if (lane == 0) wave_sums[tid >> 6] = x;
        __syncthreads();
        return (wave_sums[0] + wave_sums[1]) + (wave_sums[2] + wave_sums[3]);
    };
    double total = total_of(s);
    const bool from_p = !(total > 0.0);  // nothing is left of p - q: the token comes from p itself
    if (from_p) {
        total = total_of(plain);
        s = plain;
        left.q = nullptr;
        left.barred = -1;
    }
    const double target = (double)a.u[(size_t)b * (a.N + 1) + a.N] * total;
    double start;
    if (tid == find_run(s, 0.0, target, start, wave_sums, firsts, lasts)) {
        int part = from < a.n_parts ? from : 0;  // the first whose end lies beyond the target, else the last that is not empty
        double c = start, front = start;
        for (int i = from; i < to; ++i) {
            const double x = from_p ? parts[i].y : parts[i].x;
            if (!(x > 0.0)) continue;
            part = i;
            front = c;
            c = c + x;
            if (c > target) break;
        }
        found_part = part;
        found_start = front;
    }
    __syncthreads();

    // eight tokens of it for each thread
    const int j = found_part * kPartTokens + kRunTokens * tid;
    float p[kRunTokens], q[kRunTokens];
    load_left<VEC>(left, j, a.V, p, q);
    double x[kRunTokens], mine = 0.0;
#pragma unroll
    for (int k = 0; k < kRunTokens; ++k) {
        x[k] = left.of(p[k], q[k], j + k);
        mine = mine + x[k];
    }
    if (tid == find_run(mine, found_start, target, start, wave_sums, firsts, lasts)) {
        int token = -1;
        double c = start;
        bool past = false;
#pragma unroll
        for (int k = 0; k < kRunTokens; ++k) {
            c = c + x[k];
            if (x[k] > 0.0 && !past) {
                token = j + k;
                past = c > target;
            }
        }
        a.tokens[(size_t)b * (a.N + 1) + take] = max(token, 0);
        a.accepted[b] = take;
    }
    if (tid <= a.N && tid != take) a.tokens[(size_t)b * (a.N + 1) + tid] = tid < take ? draft : -1;
}

}  // namespace det

using namespace det;

extern "C" size_t det_verify_drafts_workspace_bytes(int B, int V)
{
    if (B < 1 || V < 1 || V > (1 << 30)) return 0;
    return (size_t)B * ((V + kPartTokens - 1) / kPartTokens) * sizeof(double2);
}

extern "C" int det_verify_drafts(const float* p, const float* q, const int32_t* drafts, const int32_t* n_drafts, const float* u,
                                 int32_t* accepted, int32_t* tokens, void* ws, size_t ws_bytes, int B, int N, int V, void* stream)
{
    if (!p || !drafts || !u || !accepted || !tokens || !ws || B < 1 || N < 1 || V < 1) return DET_EINVAL;
    if (N >= kVerifyDrafts || V > (1 << 30) || B > 65535) return DET_ESHAPE;
    if (!aligned16(p) || (q && !aligned16(q)) || !aligned16(ws)) return DET_EALIGN;
    if (ws_bytes < det_verify_drafts_workspace_bytes(B, V)) return DET_EWORKSPACE;
    const verify_args a{p, q, drafts, n_drafts, u, accepted, tokens, static_cast<double2*>(ws), N, V, (V + kPartTokens - 1) / kPartTokens};
    hipStream_t s = static_cast<hipStream_t>(stream);
    const dim3 grid(a.n_parts, B);
    if (V % 4 == 0) {
        hipLaunchKernelGGL(verify_parts_kernel<true>, grid, dim3(kBlock), 0, s, a);
        hipLaunchKernelGGL(verify_pick_kernel<true>, dim3(B), dim3(kBlock), 0, s, a);
    } else {
        hipLaunchKernelGGL(verify_parts_kernel<false>, grid, dim3(kBlock), 0, s, a);
        hipLaunchKernelGGL(verify_pick_kernel<false>, dim3(B), dim3(kBlock), 0, s, a);
    }
    return check_launch();
}
