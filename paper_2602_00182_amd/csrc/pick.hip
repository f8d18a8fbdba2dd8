// The pages that a sequence of the 8-bit cache gives up: of those that may go, the ones that got the least weight.
//
// One workgroup a slot.  The weights become integers that order like them; the last one to go is found digit by digit (eight bits at a time, the counts
// of a digit's values in LDS), and of equal weights the first pages go.
//
// Bound by its chain of steps, not by bytes (4 a page): one slot of 63 pages 4.5 us, where a launch that moves a few words takes 1.4, 64 slots of up to 512
// pages 7.2, four passes with three barriers each.  The weights are read again in every pass, from cache: held in registers 6.5 us for the latter and 5.0 for the
// former, and no more than a fixed number of pages.
#include "kv8.h"

namespace det {

struct pick_args {
    const float* weights;   // [n_slots, max_pages]
    const int32_t* table;
    const int32_t* lengths; // [n_slots]
    const int32_t* keep;
    uint8_t* dropped;       // [n_slots, max_pages]
    int n_pages, max_pages, first, recent;
};

// An integer that orders like the weight; a NaN is the smallest, -0 is 0.
__device__ __forceinline__ uint32_t weight_key(float w)
{
    if (w != w) return 0u;
    const uint32_t u = __float_as_uint(w + 0.0f);
    return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

__global__ __launch_bounds__(kBlock) void pick_pages_kernel(pick_args a)
{
    __shared__ __attribute__((aligned(16))) int counts[256];
    __shared__ int totals[2][4];
    const int slot = blockIdx.x, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const float* weights = a.weights + (size_t)slot * a.max_pages;
    const int32_t* table = a.table + (size_t)slot * a.max_pages;
    uint8_t* dropped = a.dropped + (size_t)slot * a.max_pages;
    const long long len = a.lengths[slot];
    const int pages = len <= 0 ? 0 : (int)min((long long)a.max_pages, (len + kPage - 1) / kPage);
    const int begin = min(a.first, pages), end = max(begin, pages - min(a.recent, pages));
    auto there = [&](int i) { return (unsigned)table[i] < (unsigned)a.n_pages; };

    // the pages there are, and those of them that may go
    int present = 0, may = 0;
    for (int i = tid; i < pages; i += kBlock) {
        const bool is = there(i);
        present += is;
        may += is && i >= begin && i < end;
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
        present += __shfl_xor(present, off, kWave);
        may += __shfl_xor(may, off, kWave);
    }
    if (lane == 0) totals[0][wave] = present, totals[1][wave] = may;
    __syncthreads();
    present = totals[0][0] + totals[0][1] + totals[0][2] + totals[0][3];
    may = totals[1][0] + totals[1][1] + totals[1][2] + totals[1][3];
    const long long want = (long long)present - max(a.keep[slot], 0);
    int drop = want <= 0 ? 0 : (int)min(want, (long long)may);
    if (drop == 0) {
        for (int i = tid; i < a.max_pages; i += kBlock) dropped[i] = 0;
        return;
    }
    // the drop-th smallest key: its digits from the highest; `drop` becomes how many go among those equal to it
    uint32_t key = 0u;
    for (int shift = 24; shift >= 0; shift -= 8) {
        __syncthreads();
        counts[tid] = 0;
        __syncthreads();
        for (int i = begin + tid; i < end; i += kBlock) {
            if (!there(i)) continue;
            const uint32_t k = weight_key(weights[i]);
            if (shift == 24 || (k >> (shift + 8)) == (key >> (shift + 8))) atomicAdd(&counts[(k >> shift) & 255u], 1);
        }
        __syncthreads();
        // every wave looks for the value for itself: four values a lane
        const int4 c = *reinterpret_cast<const int4*>(&counts[4 * lane]);
        const int mine = c.x + c.y + c.z + c.w;
        int sum = mine;
#pragma unroll
        for (int off = 1; off < kWave; off <<= 1) {
            const int x = __shfl_up(sum, off, kWave);
            sum += lane >= off ? x : 0;
        }
        const int at = __builtin_ctzll(__ballot(sum >= drop));
        int before = __builtin_amdgcn_readlane(sum - mine, at);
        const int v[4] = {__builtin_amdgcn_readlane(c.x, at), __builtin_amdgcn_readlane(c.y, at), __builtin_amdgcn_readlane(c.z, at), 0};
        int value = 4 * at;
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            const bool on = value == 4 * at + k && before + v[k] < drop;
            before += on ? v[k] : 0;
            value += on;
        }
        key |= (uint32_t)value << shift;
        drop -= before;
    }
    // in order: below the key all go, of those equal to it the first `drop`
    int equal = 0;  // so far
    for (int i0 = 0; i0 < a.max_pages; i0 += kBlock) {
        const int i = i0 + tid;
        bool less = false, same = false;
        if (i >= begin && i < end && there(i)) {
            const uint32_t k = weight_key(weights[i]);
            less = k < key;
            same = k == key;
        }
        const unsigned long long all = __ballot(same);
        __syncthreads();
        if (lane == 0) totals[0][wave] = __popcll(all);
        __syncthreads();
        int rank = equal + __popcll(all & ((1ull << lane) - 1ull));
        for (int w = 0; w < 4; ++w) {
            rank += w < wave ? totals[0][w] : 0;
            equal += totals[0][w];
        }
        if (i < a.max_pages) dropped[i] = less || (same && rank < drop);
    }
}

}  // namespace det

using namespace det;

extern "C" int det_kv8_pick_pages(const float* weights, const int32_t* page_table, int n_pages, int n_slots, int max_pages, const int32_t* lengths,
                                  const int32_t* keep, int first, int recent, uint8_t* dropped, void* stream)
{
    if (!weights || !page_table || !lengths || !keep || !dropped || n_pages < 1 || n_slots < 1 || max_pages < 1 || first < 0 || recent < 0)
        return DET_EINVAL;
    if (max_pages > DET_KV8_MAX_PAGES) return DET_ESHAPE;
    const pick_args a{weights, page_table, lengths, keep, dropped, n_pages, max_pages, first, recent};
    hipLaunchKernelGGL(pick_pages_kernel, dim3((unsigned)n_slots), dim3(kBlock), 0, static_cast<hipStream_t>(stream), a);
    return check_launch();
}
