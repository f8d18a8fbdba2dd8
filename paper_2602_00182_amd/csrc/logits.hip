// Rules on logits between the output head and the choice of a token: penalties for tokens that a sequence has had, biases, masks; and the bookkeeping
// behind them, a step's token into the history and the grammar's next state.
//
// A workgroup takes a stretch of one row's tokens.  It counts the history's tokens that lie in the stretch in LDS (integers: their order is free) while the
// logits are on their way, so a history of any length costs no table in memory and nothing is kept from step to step.  Bound by memory: each logit
// is read and written once.
#include "internal.h"

namespace det {

struct logits_args {
    const char* logits;
    char* out;
    int64_t ld_in, ld_out;  // elements
    det_logits_rules r;
    int V;
};

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

// One stretch of kBlock * NV vectors.  Grid (stretches, rows).
template <class T, int NV>
__global__ __launch_bounds__(kBlock) void logits_process_kernel(logits_args a)
{
    constexpr int N = vec16<T>::N, kStretch = kBlock * NV * N;
    __shared__ __attribute__((aligned(16))) uint32_t counts[kStretch];
    __shared__ __attribute__((aligned(16))) uint32_t biased[kStretch];  // a token's last entry in the row's biases, from 1 on
    const int tid = threadIdx.x, b = blockIdx.y, begin = blockIdx.x * kStretch;
    const T* in = reinterpret_cast<const T*>(a.logits) + (size_t)b * a.ld_in;
    T* out = reinterpret_cast<T*>(a.out) + (size_t)b * a.ld_out;
    const det_logits_rules& r = a.r;

    vec16<T> v[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int j = begin + (k * kBlock + tid) * N;
        if (j + N <= a.V) {
            v[k] = load_vec(in + j);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) v[k].x[i] = j + i < a.V ? in[j + i] : T(0);
        }
    }
    const uint32_t* mask = nullptr;
    if (r.masks) {
        const int m = r.mask_rows ? r.mask_rows[b] : b;
        if ((unsigned)m < (unsigned)r.n_masks) mask = r.masks + (size_t)m * r.mask_words;
    }
    float repetition = 1.0f, frequency = 0.0f, presence = 0.0f;
    if (r.penalties) {
        repetition = r.penalties[3 * b], frequency = r.penalties[3 * b + 1], presence = r.penalties[3 * b + 2];
        for (int i = tid * 4; i < kStretch; i += kBlock * 4) *reinterpret_cast<uint4*>(&counts[i]) = make_uint4(0u, 0u, 0u, 0u);
    }
    int bias_from = 0, bias_to = 0;
    if (r.bias_begin) {
        bias_from = min(max(r.bias_begin[b], 0), r.n_biases);
        bias_to = min(r.bias_begin[b + 1], r.n_biases);
        for (int i = tid * 4; i < kStretch; i += kBlock * 4) *reinterpret_cast<uint4*>(&biased[i]) = make_uint4(0u, 0u, 0u, 0u);
    }
    __syncthreads();
    if (r.penalties) {
        const int row = r.history_rows ? r.history_rows[b] : b;
        const int len = (unsigned)row < (unsigned)r.n_history ? min(r.history_lens[b], r.ld_history) : 0;
        const int from = r.generated_from ? r.generated_from[b] : 0;
        const int32_t* ids = r.history + (size_t)row * r.ld_history;
        for (int i = tid; i < len; i += kBlock) {
            const unsigned at = (unsigned)ids[i] - (unsigned)begin;
            if (at < (unsigned)kStretch) {
                if (i >= from) atomicAdd(&counts[at], 1u);
                else atomicOr(&counts[at], kSeen);
            }
        }
    }
    for (int i = bias_from + tid; i < bias_to; i += kBlock) {
        const unsigned at = (unsigned)r.bias_tokens[i] - (unsigned)begin;
        if (at < (unsigned)kStretch) atomicMax(&biased[at], (uint32_t)(i - bias_from) + 1u);
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int at = (k * kBlock + tid) * N, j = begin + at;
        if (j >= a.V) continue;
        uint32_t allowed = ~0u;
        if (mask) allowed = mask[j >> 5] >> (j & 31);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint32_t c = r.penalties ? counts[at + i] : 0u, e = bias_to > bias_from ? biased[at + i] : 0u;
            if ((c | e) != 0u) {
                float z = to_f32(v[k].x[i]);
                if (c != 0u) {
                    const uint32_t made = c & ~kSeen;
                    z = z > 0.0f ? z / repetition : z * repetition;
                    if (made != 0u) z = z - frequency * (float)made - presence;
                }
                if (e != 0u) z = z + r.bias_values[bias_from + e - 1u];
                from_f32(z, v[k].x[i]);
            }
            if (((allowed >> i) & 1u) == 0u) from_f32(-__builtin_inff(), v[k].x[i]);
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

template <class T>
static void launch_process(const logits_args& a, int B, hipStream_t s)
{
    const long long vectors = ((long long)a.V + vec16<T>::N - 1) / vec16<T>::N;
    auto grid = [&](int nv) { return dim3((unsigned)((vectors + (long long)kBlock * nv - 1) / ((long long)kBlock * nv)), (unsigned)B); };
    if (vectors * B >= 4ll * kBlock * 512) hipLaunchKernelGGL((logits_process_kernel<T, 4>), grid(4), dim3(kBlock), 0, s, a);
    else hipLaunchKernelGGL((logits_process_kernel<T, 1>), grid(1), dim3(kBlock), 0, s, a);
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
    if (B > 65535 || V > (1 << 30) || (r.masks && (long long)r.mask_words * 32 < V)) return DET_ESHAPE;
    const int size = dtype == DET_F32 ? 4 : 2;
    if (!aligned16(logits) || !aligned16(out)) return DET_EALIGN;
    // the same rows in place, or rows apart
    if (logits == out ? ld_logits != ld_out
                      : static_cast<const char*>(logits) < static_cast<char*>(out) + ((B - 1) * ld_out + V) * size &&
                            static_cast<char*>(out) < static_cast<const char*>(logits) + ((B - 1) * ld_logits + V) * size)
        return DET_EINVAL;
    const logits_args a{static_cast<const char*>(logits), static_cast<char*>(out), ld_logits, ld_out, r, V};
    if (dtype == DET_F32) launch_process<float>(a, B, static_cast<hipStream_t>(stream));
    else launch_process<uint16_t>(a, B, static_cast<hipStream_t>(stream));
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
