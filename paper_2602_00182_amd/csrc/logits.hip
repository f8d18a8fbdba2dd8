// Rules on logits between the output head and the choice of a token: penalties for tokens that a sequence has had, biases, masks; and the bookkeeping
// behind them, a step's token into the history and the grammar's next state.
//
// A workgroup takes a stretch of 4096 of one row's tokens.  It counts the history's tokens that lie in the stretch in LDS (integers: their order is free)
// while the logits are on their way, so a history of any length costs no table in memory and nothing is kept from step to step; every stretch of a row
// reads the whole history, which comes from L2.  Bound by memory: 64 rows of 128000 fp32 logits without rules 11.8 us (65 MB: 5.5 TB/s), with histories of
// 100 to 4000 tokens 15.6, with biases and masks too 16.5 (the median of a profiled run, whose inputs change, 17.0).  Smaller stretches read the history more often (2048 tokens 17.8), larger ones leave too few
// waves a compute unit (8192 tokens 19 to 28), and ids asked for one after the other, not eight a lane, took 25.
//
// A vector of logits that the mask takes whole is not read.  In place, nothing that no rule reaches is read or written.
#include "internal.h"

namespace det {

struct logits_args {
    const char* logits;
    char* out;
    int64_t ld_in, ld_out;  // elements
    det_logits_rules r;
    int V;
};

constexpr int kStretchTokens = 4096, kStretchThreads = 512;  // of large calls; small ones take a vector a lane of 256, to fill more of the chip
constexpr long long kSmallWgs = 1024;  // workgroups of small stretches up to which a call is small
constexpr int kIds = 8;                // history tokens a lane asks for at once
constexpr uint32_t kSeen = 0x80000000u;  // in a count: had, but not among the generated tokens

// 16 bytes of a row; rows of an odd width lie on any element.
template <class T>
struct vec16 {
    static constexpr int N = 16 / sizeof(T);
    T x[N];
};
template <class T>
__device__ __forceinline__ vec16<T> load_vec(const T* from)
{
    vec16<T> v;
    __builtin_memcpy(&v, from, 16);
    return v;
}
__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(uint16_t x) { return bf16_to_f32(x); }
__device__ __forceinline__ void from_f32(float x, float& to) { to = x; }
__device__ __forceinline__ void from_f32(float x, uint16_t& to) { to = f32_to_bf16_rne(x); }

// One stretch of TH * NV vectors.  Grid (stretches, rows).
template <class T, int TH, int NV, bool IN_PLACE>
__global__ __launch_bounds__(TH) void logits_process_kernel(logits_args a)
{
    constexpr int N = vec16<T>::N, kStretch = TH * NV * N;
    constexpr uint32_t kAll = (1u << N) - 1u;  // the mask's bits of a vector
    __shared__ __attribute__((aligned(16))) uint32_t counts[kStretch];
    __shared__ __attribute__((aligned(16))) uint32_t biased[kStretch];  // a token's last entry in the row's biases, from 1 on
    const int tid = threadIdx.x, b = blockIdx.y, begin = blockIdx.x * kStretch;
    const T* in = reinterpret_cast<const T*>(a.logits) + (size_t)b * a.ld_in;
    T* out = reinterpret_cast<T*>(a.out) + (size_t)b * a.ld_out;
    const det_logits_rules& r = a.r;

    const uint32_t* mask = nullptr;
    if (r.masks) {
        const int m = r.mask_rows ? r.mask_rows[b] : b;
        if ((unsigned)m < (unsigned)r.n_masks) mask = r.masks + (size_t)m * r.mask_words;
    }
    uint32_t allowed[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int j = begin + (k * TH + tid) * N;
        allowed[k] = (mask && j < a.V ? mask[j >> 5] >> (j & 31) : ~0u) & kAll;
    }
    vec16<T> v[NV];
    auto ask = [&](int k) {
        const int j = begin + (k * TH + tid) * N;
        if (j + N <= a.V) {
            v[k] = load_vec(in + j);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) v[k].x[i] = j + i < a.V ? in[j + i] : T(0);
        }
    };
    if constexpr (!IN_PLACE) {  // a vector that the mask takes whole is not read: a strict grammar's rows are little but written
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (allowed[k] != 0u) ask(k);
    }
    float repetition = 1.0f, frequency = 0.0f, presence = 0.0f;
    int len = 0, from = 0;
    const int32_t* ids = r.history;
    if (r.penalties) {
        repetition = r.penalties[3 * b], frequency = r.penalties[3 * b + 1], presence = r.penalties[3 * b + 2];
        const int row = r.history_rows ? r.history_rows[b] : b;
        if ((unsigned)row < (unsigned)r.n_history) {
            len = min(r.history_lens[b], r.ld_history);
            ids = r.history + (size_t)row * r.ld_history;
        }
        if (r.generated_from) from = r.generated_from[b];
    }
    // a run of the history, many ids a lane at once: one after the other they were most of a workgroup's time
    int32_t id[kIds];
    auto ask_ids = [&](int i0) {
#pragma unroll
        for (int k = 0; k < kIds; ++k) {
            const int i = i0 + k * TH + tid;
            id[k] = i < len ? ids[i] : -1;
        }
    };
    ask_ids(0);
    int bias_from = 0, bias_to = 0;
    if (r.bias_begin) {
        bias_from = min(max(r.bias_begin[b], 0), r.n_biases);
        bias_to = min(r.bias_begin[b + 1], r.n_biases);
    }
    if (len > 0)
        for (int i = tid * 4; i < kStretch; i += TH * 4) *reinterpret_cast<uint4*>(&counts[i]) = make_uint4(0u, 0u, 0u, 0u);
    if (bias_to > bias_from)
        for (int i = tid * 4; i < kStretch; i += TH * 4) *reinterpret_cast<uint4*>(&biased[i]) = make_uint4(0u, 0u, 0u, 0u);
    __syncthreads();
    for (int i0 = 0; i0 < len; i0 += kIds * TH) {
        if (i0 > 0) ask_ids(i0);
#pragma unroll
        for (int k = 0; k < kIds; ++k) {
            const unsigned at = (unsigned)id[k] - (unsigned)begin;
            if (id[k] >= 0 && at < (unsigned)kStretch) {
                if (i0 + k * TH + tid >= from) atomicAdd(&counts[at], 1u);
                else atomicOr(&counts[at], kSeen);
            }
        }
    }
    for (int i = bias_from + tid; i < bias_to; i += TH) {
        const unsigned at = (unsigned)r.bias_tokens[i] - (unsigned)begin;
        if (at < (unsigned)kStretch) atomicMax(&biased[at], (uint32_t)(i - bias_from) + 1u);
    }
    __syncthreads();
    uint32_t c[NV][N], e[NV][N];
    bool store[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int at = (k * TH + tid) * N;
        bool touched = false;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            c[k][i] = len > 0 ? counts[at + i] : 0u, e[k][i] = bias_to > bias_from ? biased[at + i] : 0u;
            touched |= (c[k][i] | e[k][i]) != 0u && ((allowed[k] >> i) & 1u) != 0u;
        }
        store[k] = begin + at < a.V && (!IN_PLACE || touched || allowed[k] != kAll);
        if (IN_PLACE && store[k] && allowed[k] != 0u) ask(k);  // in place nothing else moves
    }
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        if (!store[k]) continue;
        const int j = begin + (k * TH + tid) * N;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if ((c[k][i] | e[k][i]) != 0u) {
                float z = to_f32(v[k].x[i]);
                if (c[k][i] != 0u) {
                    const uint32_t made = c[k][i] & ~kSeen;
                    z = z > 0.0f ? z / repetition : z * repetition;
                    if (made != 0u) z = z - frequency * (float)made - presence;
                }
                if (e[k][i] != 0u) z = z + r.bias_values[bias_from + e[k][i] - 1u];
                from_f32(z, v[k].x[i]);
            }
            if (((allowed[k] >> i) & 1u) == 0u) from_f32(-__builtin_inff(), v[k].x[i]);
        }
        if (j + N <= a.V) {
            __builtin_memcpy(out + j, &v[k], 16);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (j + i < a.V) out[j + i] = v[k].x[i];
        }
    }
}

struct advance_args {
    const int32_t* tokens;
    int32_t* history;
    const int32_t* lens_in;
    int32_t* lens_out;
    const int32_t* transitions;  // [n_states, n_classes] or null
    const int32_t* token_class;  // [V] or null
    const int32_t* states_in;
    int32_t* states_out;
    int ld_history, n_states, n_classes, V, B;
};

__global__ __launch_bounds__(kBlock) void logits_advance_kernel(advance_args a)
{
    const int b = blockIdx.x * kBlock + threadIdx.x;
    if (b >= a.B) return;
    const int token = a.tokens[b];
    if (a.history) {
        int len = max(a.lens_in[b], 0);
        if (len < a.ld_history) a.history[(size_t)b * a.ld_history + len++] = token;
        a.lens_out[b] = len;
    }
    if (a.transitions) {
        const int state = a.states_in[b];
        int next = -1;
        if ((unsigned)state < (unsigned)a.n_states && (unsigned)token < (unsigned)a.V) {
            const int of = a.token_class ? a.token_class[token] : token;
            if ((unsigned)of < (unsigned)a.n_classes) next = a.transitions[(size_t)state * a.n_classes + of];
        }
        a.states_out[b] = (unsigned)next < (unsigned)a.n_states ? next : -1;
    }
}

template <class T, bool IN_PLACE>
static void launch_process(const logits_args& a, int B, hipStream_t s)
{
    const long long vectors = ((long long)a.V + vec16<T>::N - 1) / vec16<T>::N;
    auto grid = [&](int each) { return dim3((unsigned)((vectors + each - 1) / each), (unsigned)B); };
    constexpr int kEach = kStretchTokens / vec16<T>::N;
    if (vectors * B >= kBlock * kSmallWgs)
        hipLaunchKernelGGL((logits_process_kernel<T, kStretchThreads, kEach / kStretchThreads, IN_PLACE>), grid(kEach), dim3(kStretchThreads), 0, s, a);
    else
        hipLaunchKernelGGL((logits_process_kernel<T, kBlock, 1, IN_PLACE>), grid(kBlock), dim3(kBlock), 0, s, a);
}

}  // namespace det

using namespace det;

extern "C" int det_logits_process(const void* logits, int64_t ld_logits, void* out, int64_t ld_out, int dtype, int B, int V,
                                  const det_logits_rules* rules, void* stream)
{
    if (!logits || !out || !rules || B < 1 || V < 1 || ld_logits < V || ld_out < V || (dtype != DET_F32 && dtype != DET_BF16)) return DET_EINVAL;
    const det_logits_rules& r = *rules;
    if (r.penalties && (!r.history || !r.history_lens || r.ld_history < 1 || r.n_history < 1 || (!r.history_rows && r.n_history < B))) return DET_EINVAL;
    if (r.bias_begin && (r.n_biases < 0 || (r.n_biases > 0 && (!r.bias_tokens || !r.bias_values)))) return DET_EINVAL;
    if (r.masks && (r.n_masks < 1 || r.mask_words < 1)) return DET_EINVAL;
    if (B > 65535 || V > (1 << 30) || (r.penalties && r.ld_history > (1 << 30)) || (r.bias_begin && r.n_biases > (1 << 30)) || (r.masks && (long long)r.mask_words * 32 < V)) return DET_ESHAPE;
    const int size = dtype == DET_F32 ? 4 : 2;
    if (!aligned16(logits) || !aligned16(out)) return DET_EALIGN;
    // the same rows in place, or rows apart
    if (logits == out ? ld_logits != ld_out
                      : static_cast<const char*>(logits) < static_cast<char*>(out) + ((B - 1) * ld_out + V) * size &&
                            static_cast<char*>(out) < static_cast<const char*>(logits) + ((B - 1) * ld_logits + V) * size)
        return DET_EINVAL;
    const logits_args a{static_cast<const char*>(logits), static_cast<char*>(out), ld_logits, ld_out, r, V};
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (dtype == DET_F32) logits == out ? launch_process<float, true>(a, B, st) : launch_process<float, false>(a, B, st);
    else logits == out ? launch_process<uint16_t, true>(a, B, st) : launch_process<uint16_t, false>(a, B, st);
    return check_launch();
}

extern "C" int det_logits_advance(const int32_t* tokens, int32_t* history, int ld_history, const int32_t* lens_in, int32_t* lens_out,
                                  const int32_t* transitions, int n_states, int n_classes, const int32_t* token_class, int V,
                                  const int32_t* states_in, int32_t* states_out, int B, void* stream)
{
    if (!tokens || B < 1 || (!history && !transitions)) return DET_EINVAL;
    if (history && (!lens_in || !lens_out || ld_history < 1)) return DET_EINVAL;
    if (transitions && (!states_in || !states_out || n_states < 1 || n_classes < 1 || V < 1 || (!token_class && V > n_classes))) return DET_EINVAL;
    const advance_args a{tokens, history, lens_in, lens_out, transitions, token_class, states_in, states_out, ld_history, n_states, n_classes, V, B};
    hipLaunchKernelGGL(logits_advance_kernel, dim3((unsigned)((B + kBlock - 1) / kBlock)), dim3(kBlock), 0, static_cast<hipStream_t>(stream), a);
    return check_launch();
}
