// What the kernels of attention over the 8-bit paged cache share: the numbers (attn_kv8.hip says which and why), a tile's query, the weights' digits.
#pragma once

#include "kv8.h"

namespace det {

typedef __attribute__((__vector_size__(4 * sizeof(int)))) int v4i;

constexpr int kChunk = 256;               // tokens of a chunk
constexpr int kChunkPages = kChunk / kPage;
constexpr int kPairs = 16;                // (row, head) pairs of a tile

struct kv8_attn_args {
    const uint16_t* q;  // [R, Hq, 128]
    kv8_cache c;
    const int32_t* seqlens;
    const int32_t* slots;
    uint16_t* out;  // [R, Hq, 128]
    float* part_o;  // [R, Hq, chunks, 128]: a chunk's weighted sums, in units of its 2^(E-22)
    float4* part;   // [R, Hq, chunks]: its m, l, 2^(E-22)
    int R, Hq, G, rows_per_tile, len_offset, chunks, chunk_step, inverse_G;
    float scale_log2;  // scale * log2(e)
};

// ---------------------------------------------------------------- numbers

// 2^(a - b) for integers a <= b held as floats (or infinite): 0 from a difference of 127 on.
__device__ __forceinline__ float pow2_step(float a, float b)
{
    const float d = fmaxf(a - b, -127.0f);
    return __uint_as_float((uint32_t)((int)d + 127) << 23);
}

// Exponent E with x < 2^E, for x >= 0; from 2^-100 down it stays there.
__device__ __forceinline__ int exponent_above(float x)
{
    const int e = (int)((__float_as_uint(x) >> 23) & 0xFF) - 126;
    return e < -100 ? -100 : e;
}
__device__ __forceinline__ float pow2i(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// Bytes 0, 1 and 2 of four words, each gathered into one word.
__device__ __forceinline__ void gather_bytes(const uint32_t (&y)[4], uint32_t& b0, uint32_t& b1, uint32_t& b2)
{
    const uint32_t lo = __builtin_amdgcn_perm(y[1], y[0], 0x05010400u), hi = __builtin_amdgcn_perm(y[3], y[2], 0x05010400u);
    b0 = __builtin_amdgcn_perm(hi, lo, 0x05040100u);
    b1 = __builtin_amdgcn_perm(hi, lo, 0x07060302u);
    const uint32_t l2 = __builtin_amdgcn_perm(y[1], y[0], 0x0C0C0602u), h2 = __builtin_amdgcn_perm(y[3], y[2], 0x0C0C0602u);
    b2 = __builtin_amdgcn_perm(h2, l2, 0x05040100u);
}

// The larger of two, the largest of three, in one instruction: fmaxf would first have every operand quieted, which nothing here needs.
__device__ __forceinline__ float max2(float a, float b)
{
    float d;
    asm("v_max_f32 %0, %1, %2" : "=v"(d) : "v"(a), "v"(b));
    return d;
}
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float d;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(d) : "v"(a), "v"(b), "v"(c));
    return d;
}

// Maximum and sum over the sixteen lanes of a row of lanes (rotations: every lane has the result; a sum adds the same pairs in each).
template <int N>
__device__ __forceinline__ float row_ror(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x120 + N, 0xF, 0xF, true));
}
__device__ __forceinline__ float row_max(float v)
{
    v = max2(v, row_ror<8>(v));
    v = max2(v, row_ror<4>(v));
    v = max2(v, row_ror<2>(v));
    return max2(v, row_ror<1>(v));
}
__device__ __forceinline__ float row_sum(float v)
{
    v = v + row_ror<8>(v);
    v = v + row_ror<4>(v);
    v = v + row_ror<2>(v);
    return v + row_ror<1>(v);
}

// The running softmax of a row: weights relative to 2^m, their sum l.  fold_step joins a chunk's (mc, lc), whose sums are in units of `unit`, and
// gives the factors of the sums so far (a) and of the chunk's (b): powers of two, so where a rounding falls does not hang on when they are applied.
__device__ __forceinline__ void fold_step(float& m, float& l, float mc, float lc, float unit, float& a, float& b)
{
    const float to = fmaxf(m, mc);
    a = pow2_step(m, to);
    b = pow2_step(mc, to);
    l = __builtin_fmaf(lc, b, l * a);
    b = b * unit;
    m = to;
}
__device__ __forceinline__ float fold_value(float o, float oc, float a, float b) { return __builtin_fmaf(oc, b, o * a); }
__device__ __forceinline__ float digits_value(int d0, int d1, int d2) { return __builtin_fmaf((float)d0, 65536.0f, (float)(d1 * 256 + d2)); }
// What a row's sums are multiplied with.  A row that no token reaches has l = 0 and gives zeros.
__device__ __forceinline__ float row_factor(float l) { return l == 0.0f ? 0.0f : 1.0f / l; }
__device__ __forceinline__ uint16_t to_bf16(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }

// ---------------------------------------------------------------- a tile's query

// Sixteen consecutive columns of a query as digits: the bytes of one operand of the matrix instruction.
struct q_digits {
    v4i d[3];  // the highest digit first
};

// w: eight words of two bf16 each; up = 2^(22 - E).
__device__ __forceinline__ q_digits cut_half(const uint32_t* w, float up)
{
    q_digits o;
#pragma unroll
    for (int k = 0; k < 4; ++k) {  // four columns
        uint32_t y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t pair = w[2 * k + (i >> 1)];
            const float x = (i & 1) ? bf16hi_to_f32(pair) : bf16lo_to_f32(pair);
            // adding 1.5 * 2^23 leaves the nearest integer n in the low bits; + 0x8080 makes bytes 0 and 1 the digits plus 128
            y[i] = __float_as_uint(__builtin_fmaf(x, up, 12582912.0f)) - 0x4B400000u + 0x8080u;
        }
        uint32_t b0, b1, b2;
        gather_bytes(y, b0, b1, b2);
        o.d[0][k] = (int)b2;
        o.d[1][k] = (int)(b1 ^ 0x80808080u);
        o.d[2][k] = (int)(b0 ^ 0x80808080u);
    }
    return o;
}

// The query of this lane's operand row: q its 128 values (or null), of which the lane takes columns 64 h + 16 (lane / 16) + 0..15.
__device__ __forceinline__ void ask_query(const uint16_t* q, uint32_t (&w)[16])
{
    const int group = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int k = 0; k < 16; ++k) w[k] = 0u;
    if (!q) return;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint4 x = *reinterpret_cast<const uint4*>(q + 64 * (k >> 1) + 16 * group + 8 * (k & 1));
        w[4 * k] = x.x, w[4 * k + 1] = x.y, w[4 * k + 2] = x.z, w[4 * k + 3] = x.w;
    }
}
// factor: what an integer score stands for, in units of log2 (NaN for a query that is not finite).
__device__ __forceinline__ void cut_query(const uint32_t (&w)[16], float scale_log2, q_digits (&digits)[2], float& factor)
{
    uint32_t big = 0u;  // magnitudes of bf16 order like the integers of their bits; NaN and infinities are the largest
#pragma unroll
    for (int k = 0; k < 16; ++k) big = max(big, max(w[k] & 0x7FFF0000u, (w[k] << 16) & 0x7FFF0000u));
    big = max(big, (uint32_t)__shfl_xor((int)big, 16, kWave));
    big = max(big, (uint32_t)__shfl_xor((int)big, 32, kWave));
    const int e = exponent_above(__uint_as_float(big));
    const float up = pow2i(22 - e);
    // never 0: a masked score, -inf, stays what it is
    factor = big < 0x7F800000u ? fmaxf(scale_log2 * pow2i(e - 22), 0x1p-126f) : __builtin_nanf("");
    digits[0] = cut_half(w, up);
    digits[1] = cut_half(w + 8, up);
}

// Sixteen bytes of a record: one address for the wave, one offset a lane.
__device__ __forceinline__ v4i load16(const uint8_t* rec, uint32_t offset, int constant)
{
    return *reinterpret_cast<const v4i*>(rec + (size_t)offset + constant);
}

__device__ __forceinline__ void wave_lds_order()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
}

// Length of a row of the call: 0 where its slot is none.
__device__ __forceinline__ int row_length(const kv8_attn_args& a, int row, int& slot)
{
    slot = a.slots ? a.slots[row] : row;
    const long long n = (long long)a.seqlens[row] + a.len_offset, most = (long long)a.c.max_pages * kPage;
    return (unsigned)slot < (unsigned)a.c.n_slots ? (int)(n < 0 ? 0 : (n > most ? most : n)) : 0;
}

// What a score's token contributes with: d^K, poisoned where the token's V row is not finite (the rows that see the token become NaN, the others
// do not), and d^V, 0 there.  scales: the page's K scales, its V scales behind them.
__device__ __forceinline__ void clean_scales(float (&dk)[4], float (&dv)[4])
{
    bool bad = false;
#pragma unroll
    for (int t = 0; t < 4; ++t) bad |= !(fabsf(dv[t]) < __builtin_inff());
    if (__ballot(bad) == 0) return;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        dk[t] = dk[t] + 0.0f * dv[t];
        dv[t] = fabsf(dv[t]) < __builtin_inff() ? dv[t] : 0.0f;
    }
}
__device__ __forceinline__ void ask_scales(const uint8_t* scales, int col, float (&dk)[4], float (&dv)[4])
{
    const uint32_t at = 16 * col;
    const float4 ks = *reinterpret_cast<const float4*>(scales + (size_t)at);
    const float4 vs = *reinterpret_cast<const float4*>(scales + (size_t)at + (kRecordVs - kRecordKs));
    dk[0] = ks.x, dk[1] = ks.y, dk[2] = ks.z, dk[3] = ks.w;
    dv[0] = vs.x, dv[1] = vs.y, dv[2] = vs.z, dv[3] = vs.w;
}
__device__ __forceinline__ void clean_scales(const uint8_t* scales, int col, float (&dk)[4], float (&dv)[4])
{
    ask_scales(scales, col, dk, dv);
    clean_scales(dk, dv);
}
__device__ __forceinline__ void token_scales(const uint8_t* rec, int col, float (&dk)[4], float (&dv)[4])
{
    clean_scales(rec + kRecordKs, col, dk, dv);
}
// Row and head within the KV head of pair p of a tile (p < 16, exact).
__device__ __forceinline__ int pair_row(const kv8_attn_args& a, int p) { return (p * a.inverse_G) >> 16; }

// The row's factor for scores whose largest is x.  Where none is above -inf they are masked or NaN, and a query's NaN would make NaN of the masked ones:
// 1 leaves both what they are.
__device__ __forceinline__ float seen_factor(float x, float factor) { return x == -__builtin_inff() ? 1.0f : factor; }

// From 2^24 on a score's product with the factor is rounded by a unit and more, and an fma that keeps it exact would leave the largest score anywhere
// within 2^7 units of m at 2^31: its weight 0 or infinite.  There the product is rounded first, so that the largest is m itself.  (An infinite m stays one:
// the row becomes NaN.)
constexpr float kFarScore = 0x1p24f;
__device__ __forceinline__ void far_scores(float (&s)[4], float f, float m)
{
#pragma unroll
    for (int t = 0; t < 4; ++t) s[t] = fabsf(m) >= kFarScore ? s[t] * f - m : s[t];
}

// A score from its digit sums; times the row's factor it is in units of log2.
__device__ __forceinline__ float score_of(int d0, int d1, int d2, float dk)
{
    return digits_value(d0, d1, d2) * dk;
}

// ---------------------------------------------------------------- the weights' digits

// One digit of four neighbouring tokens' weights to a word: the weights as integers of 22 bits.
template <int NP>
__device__ __forceinline__ void cut_weights(const float (&w)[4][NP], int r, float up, uint32_t (&b)[3])
{
    uint32_t y[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) y[t] = __float_as_uint(__builtin_fmaf(w[t][r], up, 8421504.0f));  // 2^23 + 0x8080
    gather_bytes(y, b[2], b[1], b[0]);
    b[1] ^= 0x80808080u;
    b[2] ^= 0x80808080u;
}

// The digits of a chunk's weights into a wave's LDS, as the second product takes them: of each digit sixteen rows (pairs) of 256 bytes (tokens), the
// sixteen-byte pieces of a row swizzled by the pair.  here: the lane, hidden from the compiler, so that it keeps no addresses over a loop.
constexpr int kChunkDigits = 3 * kPairs * kChunk;
__device__ __forceinline__ void store_digits(const float (&w)[kChunkPages][4][4], const float (&up)[4], uint8_t* digits, int here)
{
    const int g4 = here >> 4, c = here & 15;
    wave_lds_order();
#pragma unroll
    for (int p = 0; p < kChunkPages; ++p) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            uint32_t b[3];
            cut_weights(w[p], r, up[r], b);
            // piece (4 p + c / 4) ^ (4 g4 + r) of row 4 g4 + r
            uint8_t* at = digits + kChunk * (4 * g4 + r) + 64 * (p ^ g4) + 16 * ((c >> 2) ^ r) + 4 * (c & 3);
#pragma unroll
            for (int g = 0; g < 3; ++g) *reinterpret_cast<uint32_t*>(at + g * kPairs * kChunk) = b[g];
        }
        __builtin_amdgcn_sched_barrier(0);
    }
    wave_lds_order();
}
// This lane's operand of digit g, tokens of page p.
__device__ __forceinline__ v4i load_digits(const uint8_t* digits, int g, int p, int here)
{
    return *reinterpret_cast<const v4i*>(digits + g * kPairs * kChunk + ((272 * (here & 15)) ^ (16 * (here >> 4) + 64 * p)));
}

// ---------------------------------------------------------------- a chunk by one wave

// Scores to weights e d^V, in place, and what the fold needs of the chunk.  scales(p, dk, dv): those of this lane's tokens of page p.  PAGES: of each
// page the sum of its e too.
template <bool PAGES = false, class Scales>
__device__ __forceinline__ void softmax_weights(float (&s)[kChunkPages][4][4], const float (&factors)[4], Scales scales, float (&mc)[4],
                                                float (&lc)[4], float (&up)[4], float (&unit)[4],
                                                float (*pages)[4] = nullptr)
{
    float safe[4], sum[kChunkPages][4], top[4], f[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        float x = -__builtin_inff();
#pragma unroll
        for (int p = 0; p < kChunkPages; ++p)
#pragma unroll
            for (int t = 0; t < 4; t += 2) x = max3(x, s[p][t][r], s[p][t + 1][r]);
        x = row_max(x);
        f[r] = seen_factor(x, factors[r]);
        mc[r] = __builtin_ceilf(x * f[r]);
        safe[r] = mc[r] == -__builtin_inff() ? 0.0f : mc[r];
        top[r] = 0.0f;
    }
    if (__builtin_expect(__ballot(max3(max2(fabsf(safe[0]), fabsf(safe[1])), fabsf(safe[2]), fabsf(safe[3])) >= kFarScore) != 0, 0)) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
#pragma unroll
            for (int p = 0; p < kChunkPages; ++p) {
                float x[4] = {s[p][0][r], s[p][1][r], s[p][2][r], s[p][3][r]};
                far_scores(x, f[r], safe[r]);
#pragma unroll
                for (int t = 0; t < 4; ++t) s[p][t][r] = x[t];
            }
            if (fabsf(safe[r]) >= kFarScore) f[r] = 1.0f, safe[r] = 0.0f;
        }
    }
#pragma unroll
    for (int p = 0; p < kChunkPages; ++p) {
        float dk[4], dv[4];
        scales(p, dk, dv);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            float e[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                e[t] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[p][t][r], f[r], -safe[r]));
                s[p][t][r] = e[t] * dv[t];
            }
            top[r] = max3(max3(top[r], s[p][0][r], s[p][1][r]), s[p][2][r], s[p][3][r]);
            sum[p][r] = (e[0] + e[1]) + (e[2] + e[3]);
        }
        __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        if constexpr (PAGES) {
#pragma unroll
            for (int p = 0; p < kChunkPages; ++p) pages[p][r] = row_sum(sum[p][r]);
        }
        lc[r] = row_sum((sum[0][r] + sum[1][r]) + (sum[2][r] + sum[3][r]));
        const int e = exponent_above(row_max(top[r]));
        up[r] = pow2i(22 - e);
        unit[r] = pow2i(e - 22);
    }
}

template <int N>
__device__ __forceinline__ void wait_loads_barrier()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

}  // namespace det
