// Attention over the 8-bit paged cache, on the int8 matrix instruction.
//
// Both products are sums of integers, so their order is free and their result exact:
//   scores   q of a (row, head) as a fixed-point number of 23 bits relative to its largest element, in three signed digits of base 256; digit
//            sums are below 2^21 and exact in fp32.
//   values   the weights w_j = e_j d^V_j of a chunk of 256 tokens as fixed-point numbers of 22 bits relative to the chunk's largest, three
//            digits; a chunk's digit sums are below 2^22.  What a weight loses is at most 2^-22 of the chunk's largest, so a result is off by at
//            most 2^-22 of the largest weight times its column's codes.  That is small beside the row, whose other columns hold that weight times codes up
//            to 127, but not always beside a column in which the heaviest token's code is 0: relative to such a column the error is 3e-7 where all
//            weights are of a size, 3e-4 where that token outweighs the others by 2^10, 2e-2 by 2^16 (a host model; bf16 rounds by 4e-3 at most).  The query
//            likewise: an element of less than 2^-14 of the largest keeps fewer than its eight bits.  A fourth digit would need 16 KB of LDS more
//            a workgroup of the walk, which then has a compute unit for itself.
// Softmax: a chunk's reference m_c is an integer (the ceiling of its largest score in units of log2), so the factors by which chunks are
// brought together are powers of two.  Chunks are folded in ascending order.
//
// Three forms, the same bytes: a row (or a tile of rows that name slots) a chunk at a time by four waves with the chunks' sums in memory and a second launch;
// calls of DET_KV8_WALK_TILES tiles and more, where the tiles alone fill most of the chip, walk their chunks in one launch.  Chunk by chunk against the
// walk, rows of one slot, 32/8 heads: 256 rows before 8000 tokens (512 tiles) 215 and 223 us, 512 (1024) 380 and 226, 1000 rows of a prompt (2000) 137
// and 35; slots of 100 rows at 100 to 2000 tokens (800) 69 and 97, of 64 rows at 100 to 1500 (1024) 73 and 47; 16/4 heads, 1000 rows (1000) 56 and 34.
// The line knows tiles, not slots: calls of few rows a slot, whose tiles go alone, lose by the walk (slots of 200 to 2000 tokens, 32/8 heads: 128 of 9 rows
// 225 and 170, 256 of 5 rows 291 and 227, but 300 of 3 rows 287 and 369, 600 of 2 rows 364 and 407, 500 of one row 323 and 632, with slots NULL 259; 16/4
// heads: 128 of 9 rows 129 and 167, 256 of 5 rows 170 and 224, 300 of 3 rows 186 and 298).
#include <type_traits>

#include "geometry.h"
#include "kv8.h"
#include "stream.h"

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

// ---------------------------------------------------------------- a chunk by four waves

// One chunk for a tile of up to sixteen (row, head) pairs that read one KV head.  Rows of a tile may name different slots: those that name the
// same one go through it together, one slot after the other.  Grid (KV heads x chunk_step, tiles): neighbouring workgroups read
// one page's records, which lie side by side (16 rows of up to 32768 tokens 200 -> 190 us against tiles in front of chunks).  A workgroup takes every
// chunk_step-th chunk: a table much wider than its sequences are long costs no workgroups that find nothing.
//
// For the scores a wave takes one of the four pages; the digits of the weights meet in LDS, and for the weighted sums it takes 32 of the 128 columns of
// all four, so that no sums have to be joined and few are held.  All of a wave's loads (8 KB of K, 8 KB of V) are asked for before the first
// is used; the workgroups of a compute unit hide one another's way to memory.
//
// PACK: up to four pairs (one row of up to four heads a KV head).  Their digits fill the sixteen rows of one operand, row 4 pair + digit, so a
// product is one instruction instead of three and a lane has all digits of one pair: a quarter of the scores' arithmetic.
template <bool PACK>
__global__ __launch_bounds__(256, PACK ? 3 : 2) void kv8_attn_chunk_kernel(kv8_attn_args a)
{
    constexpr int NP = PACK ? 1 : 4;                 // pairs of a lane
    constexpr int PAIRS = PACK ? 4 : kPairs, DIGITS = PACK ? 1 : 3;
    __shared__ __attribute__((aligned(1024))) uint8_t digits[DIGITS * kPairs * kChunk];
    __shared__ float top[2][4][PAIRS];               // largest score, largest weight of each wave
    __shared__ float lsum[4][PAIRS][16];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, group = lane >> 4, col = lane & 15;
    const int kvh = blockIdx.x % a.c.Hkv, first_chunk = blockIdx.x / a.c.Hkv, row0 = blockIdx.y * a.rows_per_tile;
    // pair number `col` of the tile
    const bool live = col < a.rows_per_tile * a.G && row0 + pair_row(a, col) < a.R;
    int slot = -1, len = 0;
    if (live) len = row_length(a, row0 + pair_row(a, col), slot);
    // chunk 0 also answers for rows that see nothing
    if (first_chunk == 0) {
        for (int p = wave; p < a.rows_per_tile * a.G; p += 4) {
            const int r = pair_row(a, p);
            if (row0 + r < a.R && __builtin_amdgcn_readlane(len, p) == 0)
                reinterpret_cast<uint32_t*>(a.out + ((size_t)(row0 + r) * a.Hq + kvh * a.G + p - r * a.G) * kHeadDim)[lane] = 0u;
        }
    }
    if (__ballot(len > first_chunk * kChunk) == 0) return;

    const int qp = PACK ? col >> 2 : col, qrow = pair_row(a, qp);  // the pair of this lane's operand row
    uint32_t words[16];
    ask_query(qp < a.rows_per_tile * a.G && row0 + qrow < a.R ? a.q + ((size_t)(row0 + qrow) * a.Hq + kvh * a.G + qp - qrow * a.G) * kHeadDim : nullptr, words);
    q_digits qd[2];
    float factors[NP];
    auto cut = [&] {
        float factor;
        cut_query(words, a.scale_log2, qd, factor);
#pragma unroll
        for (int r = 0; r < NP; ++r) factors[r] = __shfl(factor, PACK ? 4 * group : 4 * group + r, kWave);
        if constexpr (PACK) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int dg = col & 3;
                    qd[h].d[0][i] = dg == 0 ? qd[h].d[0][i] : dg == 1 ? qd[h].d[1][i] : dg == 2 ? qd[h].d[2][i] : 0;
                }
        }
    };
    if constexpr (!PACK) cut();
    const v4i zero = {0, 0, 0, 0};
    const uint32_t key_at = 512 * col + 16 * group, value_at = kRecordV + 2048 * group + 16 * col + 512 * wave;
    bool first = true;
    for (int chunk = first_chunk;; chunk += a.chunk_step) {
        unsigned todo = (unsigned)(__ballot(len > chunk * kChunk) & 0xFFFFull);
        if (todo == 0) return;
        while (todo != 0) {
            const int now = __builtin_amdgcn_readlane(slot, __builtin_ctz(todo));
            const int mine = slot == now ? len : 0;
            const unsigned members = (unsigned)(__ballot(mine > chunk * kChunk) & 0xFFFFull);
            todo = PACK ? 0u : todo & ~members;  // PACK: one row, one slot
            int longest = mine;
#pragma unroll
            for (int off = 1; off < 16; off <<= 1) longest = max(longest, __shfl_xor(longest, off, kWave));
            longest = __builtin_amdgcn_readfirstlane(longest);
            int lens[NP];
#pragma unroll
            for (int r = 0; r < NP; ++r) lens[r] = __shfl(mine, PACK ? group : 4 * group + r, kWave);
            // the chunk's pages; where one is missing, any record (its tokens weigh nothing)
            const uint8_t *rec[kChunkPages], *keys = nullptr;
#pragma unroll
            for (int p = 0; p < kChunkPages; ++p) {
                const int page = chunk * kChunkPages + p;
                const uint8_t* at = page * kPage < longest ? kv8_record_uniform(a.c, now, page, kvh) : nullptr;
                keys = p == wave ? at : keys;
                rec[p] = at ? at : a.c.pool;
            }
            if (!first) __syncthreads();  // the last slot's digits have been read

            v4i kc[4][2], vc[kChunkPages][2];
            float dk[4], dv[4] = {};
            if (keys) {
                ask_scales(keys + kRecordKs, col, dk, dv);
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int h = 0; h < 2; ++h) kc[t][h] = load16(keys, key_at, t * kHeadDim + 64 * h);
            }
#pragma unroll
            for (int p = 0; p < kChunkPages; ++p)
#pragma unroll
                for (int n = 0; n < 2; ++n) vc[p][n] = load16(rec[p], value_at, 256 * n);
            __builtin_amdgcn_sched_barrier(0);
            if (PACK && first) cut();  // while they are on their way
            first = false;
            float s[4][NP];
            if (keys) {
                clean_scales(dk, dv);
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    v4i d[DIGITS];
#pragma unroll
                    for (int g = 0; g < DIGITS; ++g) d[g] = __builtin_amdgcn_mfma_i32_16x16x64_i8(qd[0].d[g], kc[t][0], zero, 0, 0, 0);
#pragma unroll
                    for (int g = 0; g < DIGITS; ++g) d[g] = __builtin_amdgcn_mfma_i32_16x16x64_i8(qd[1].d[g], kc[t][1], d[g], 0, 0, 0);
                    const int token = (chunk * kChunkPages + wave) * kPage + 4 * col + t;
#pragma unroll
                    for (int r = 0; r < NP; ++r) {
                        float x;
                        if constexpr (PACK) x = score_of(d[0][0], d[0][1], d[0][2], dk[t]);
                        else x = score_of(d[0][r], d[1][r], d[2][r], dk[t]);
                        s[t][r] = token < lens[r] ? x : -__builtin_inff();
                    }
                    if constexpr (!PACK) __builtin_amdgcn_sched_barrier(0);
                }
            } else {
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int r = 0; r < NP; ++r) s[t][r] = -__builtin_inff();
            }
            // the chunk's largest score, then its largest weight, over the waves
            float mc[NP], unit[NP], up[NP], f[NP];
#pragma unroll
            for (int r = 0; r < NP; ++r) {
                const float x = row_max(max2(max3(s[0][r], s[1][r], s[2][r]), s[3][r]));
                f[r] = seen_factor(x, factors[r]);
                if (col == 0) top[0][wave][PACK ? group : 4 * group + r] = x * f[r];
            }
            __syncthreads();
            float safe[NP], most = 0.0f;
#pragma unroll
            for (int r = 0; r < NP; ++r) {
                const int p = PACK ? group : 4 * group + r;
                mc[r] = __builtin_ceilf(fmaxf(fmaxf(top[0][0][p], top[0][1][p]), fmaxf(top[0][2][p], top[0][3][p])));
                safe[r] = mc[r] == -__builtin_inff() ? 0.0f : mc[r];
                most = max2(most, fabsf(safe[r]));
            }
            if (__builtin_expect(__ballot(most >= kFarScore) != 0, 0)) {
#pragma unroll
                for (int r = 0; r < NP; ++r) {
                    float x[4] = {s[0][r], s[1][r], s[2][r], s[3][r]};
                    far_scores(x, f[r], safe[r]);
#pragma unroll
                    for (int t = 0; t < 4; ++t) s[t][r] = x[t];
                    if (fabsf(safe[r]) >= kFarScore) f[r] = 1.0f, safe[r] = 0.0f;
                }
            }
#pragma unroll
            for (int r = 0; r < NP; ++r) {
                const int p = PACK ? group : 4 * group + r;
                float e[4];
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    e[t] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][r], f[r], -safe[r]));
                    s[t][r] = e[t] * dv[t];
                }
                lsum[wave][p][col] = (e[0] + e[1]) + (e[2] + e[3]);
                const float w = row_max(max3(max3(0.0f, s[0][r], s[1][r]), s[2][r], s[3][r]));
                if (col == 0) top[1][wave][p] = w;
            }
            __syncthreads();
#pragma unroll
            for (int r = 0; r < NP; ++r) {
                const int p = PACK ? group : 4 * group + r;
                const int e = exponent_above(fmaxf(fmaxf(top[1][0][p], top[1][1][p]), fmaxf(top[1][2][p], top[1][3][p])));
                up[r] = pow2i(22 - e);
                unit[r] = pow2i(e - 22);
                uint32_t b[3];
                cut_weights(s, r, up[r], b);
                // operand rows: PACK 4 pair + digit; else one operand a digit, row = pair.  Pieces swizzled by the row (see store_digits).
                if constexpr (PACK) {
#pragma unroll
                    for (int g = 0; g < 4; ++g)
                        *reinterpret_cast<uint32_t*>(digits + kChunk * (4 * group + g) + 64 * (wave ^ group) + 16 * ((col >> 2) ^ g) + 4 * (col & 3)) = g < 3 ? b[g] : 0u;
                } else {
#pragma unroll
                    for (int g = 0; g < 3; ++g)
                        *reinterpret_cast<uint32_t*>(digits + kChunk * (g * kPairs + 4 * group + r) + 64 * (wave ^ group) + 16 * ((col >> 2) ^ r) + 4 * (col & 3)) = b[g];
                }
            }
            __syncthreads();
            v4i acc[DIGITS][2];
#pragma unroll
            for (int p = 0; p < kChunkPages; ++p)
#pragma unroll
                for (int g = 0; g < DIGITS; ++g) {
                    const v4i w = load_digits(digits, g, p, lane);
#pragma unroll
                    for (int n = 0; n < 2; ++n) acc[g][n] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w, vc[p][n], p == 0 ? zero : acc[g][n], 0, 0, 0);
                }

            // of each pair two columns a lane
#pragma unroll
            for (int r = 0; r < NP; ++r) {
                const int p = PACK ? group : 4 * group + r;
                const float lc = row_sum((lsum[0][p][col] + lsum[1][p][col]) + (lsum[2][p][col] + lsum[3][p][col]));
                const int pair_len = __shfl(len, p, kWave);
                if (!((members >> p) & 1u)) continue;
                const int row = pair_row(a, p);
                const size_t head = (size_t)(row0 + row) * a.Hq + kvh * a.G + p - row * a.G;
                float o[2];
#pragma unroll
                for (int n = 0; n < 2; ++n) o[n] = PACK ? digits_value(acc[0][n][0], acc[0][n][1], acc[0][n][2]) : digits_value(acc[0][n][r], acc[PACK ? 0 : 1][n][r], acc[PACK ? 0 : 2][n][r]);
                if (pair_len <= kChunk) {  // the row's only chunk
                    float fm = -__builtin_inff(), l = 0.0f, fa, fb;
                    fold_step(fm, l, mc[r], lc, unit[r], fa, fb);
                    const float by = row_factor(l);
#pragma unroll
                    for (int n = 0; n < 2; ++n) __builtin_nontemporal_store(to_bf16(fold_value(0.0f, o[n], fa, fb) * by), &a.out[head * kHeadDim + 32 * wave + 16 * n + col]);
                } else {
                    const size_t at = head * a.chunks + chunk;
                    if (wave == 0 && col == 0) a.part[at] = make_float4(mc[r], lc, unit[r], 0.0f);
#pragma unroll
                    for (int n = 0; n < 2; ++n) __builtin_nontemporal_store(o[n], &a.part_o[at * kHeadDim + 32 * wave + 16 * n + col]);
                }
            }
        }
    }
}

// The chunks of one (row, head) of more than one chunk, folded in ascending order.  Grid (R * Hq), one column a thread.  Blocks of sixteen chunks are
// asked for at once, the next one before the one at hand is folded.
constexpr int kFoldBlock = 16;
__global__ __launch_bounds__(128) void kv8_attn_combine_kernel(kv8_attn_args a)
{
    const size_t at = blockIdx.x;
    int slot;
    const int len = row_length(a, (int)(at / a.Hq), slot);
    if (len <= kChunk) return;
    const int chunks = (len + kChunk - 1) / kChunk;
    const float4* ps = a.part + at * a.chunks;
    const float* po = a.part_o + at * a.chunks * kHeadDim + threadIdx.x;
    float x[2][kFoldBlock];
    auto ask = [&](float (&to)[kFoldBlock], int c0) {
#pragma unroll
        for (int k = 0; k < kFoldBlock; ++k) to[k] = po[(size_t)min(c0 + k, chunks - 1) * kHeadDim];
    };
    ask(x[0], 0);
    float m = -__builtin_inff(), l = 0.0f, o = 0.0f;
    auto fold = [&](const float (&from)[kFoldBlock], int c0) {
        float4 st[kFoldBlock];
#pragma unroll
        for (int k = 0; k < kFoldBlock; ++k) st[k] = ps[min(c0 + k, chunks - 1)];
#pragma unroll
        for (int k = 0; k < kFoldBlock; ++k) {  // past the last chunk: one without tokens, which changes nothing
            const bool there = c0 + k < chunks;
            float fa, fb;
            fold_step(m, l, there ? st[k].x : -__builtin_inff(), there ? st[k].y : 0.0f, st[k].z, fa, fb);
            o = fold_value(o, there ? from[k] : 0.0f, fa, fb);
        }
    };
    for (int c0 = 0; c0 < chunks; c0 += 2 * kFoldBlock) {
        if (c0 + kFoldBlock < chunks) ask(x[1], c0 + kFoldBlock);
        fold(x[0], c0);
        if (c0 + kFoldBlock >= chunks) break;
        if (c0 + 2 * kFoldBlock < chunks) ask(x[0], c0 + 2 * kFoldBlock);
        fold(x[1], c0 + kFoldBlock);
    }
    __builtin_nontemporal_store(to_bf16(o * row_factor(l)), &a.out[at * kHeadDim + threadIdx.x]);
}

// Scores to weights e d^V, in place, and what the fold needs of the chunk.  scales(p, dk, dv): those of this lane's tokens of page p.
template <class Scales>
__device__ __forceinline__ void softmax_weights(float (&s)[kChunkPages][4][4], const float (&factors)[4], Scales scales, float (&mc)[4],
                                                float (&lc)[4], float (&up)[4], float (&unit)[4])
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
        lc[r] = row_sum((sum[0][r] + sum[1][r]) + (sum[2][r] + sum[3][r]));
        const int e = exponent_above(row_max(top[r]));
        up[r] = pow2i(22 - e);
        unit[r] = pow2i(e - 22);
    }
}

__device__ __forceinline__ void store_rows(const kv8_attn_args& a, int row0, int kvh, unsigned members, const float (&l)[4], const float (&o)[8][4])
{
    const int lane = threadIdx.x & 63, group = lane >> 4, col = lane & 15;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int p = 4 * group + r;
        if (!((members >> p) & 1u)) continue;
        const int row = pair_row(a, p);
        uint16_t* out = a.out + ((size_t)(row0 + row) * a.Hq + kvh * a.G + p - row * a.G) * kHeadDim;
        const float by = row_factor(l[r]);
#pragma unroll
        for (int n = 0; n < 8; ++n) __builtin_nontemporal_store(to_bf16(o[n][r] * by), &out[16 * n + col]);
    }
}

// One wave walks its tile for itself, its pages straight from memory, one slot after the other: for tiles whose neighbours' rows name other slots.
// digits_of: the workgroup's digits.
__device__ __forceinline__ void walk_alone(const kv8_attn_args& a, int kvh, int tile, uint8_t* digits_of)
{
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, group = lane >> 4, col = lane & 15;
    uint8_t* digits = digits_of + wave * kChunkDigits;
    const int row0 = tile * a.rows_per_tile;
    const bool live = col < a.rows_per_tile * a.G && row0 + pair_row(a, col) < a.R;
    int slot = -1, len = 0;
    if (live) len = row_length(a, row0 + pair_row(a, col), slot);
    const int my_pair_row = pair_row(a, col);
    uint32_t words[16];
    ask_query(live ? a.q + ((size_t)(row0 + my_pair_row) * a.Hq + kvh * a.G + col - my_pair_row * a.G) * kHeadDim : nullptr, words);
    q_digits qd[2];
    float factor, factors[4];
    cut_query(words, a.scale_log2, qd, factor);
#pragma unroll
    for (int r = 0; r < 4; ++r) factors[r] = __shfl(factor, 4 * group + r, kWave);
    const v4i zero = {0, 0, 0, 0};
    const uint32_t key_at = 512 * col + 16 * group, value_at = kRecordV + 2048 * group + 16 * col;

    unsigned todo = (unsigned)(__ballot(live) & 0xFFFFull);
    while (todo != 0) {
        const int now = __builtin_amdgcn_readlane(slot, __builtin_ctz(todo));
        const unsigned members = (unsigned)(__ballot(live && slot == now) & 0xFFFFull);
        todo &= ~members;
        int longest = (members >> col) & 1u ? len : 0;
        float m[4], l[4], o[8][4];
        int lens[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            lens[r] = __shfl(longest, 4 * group + r, kWave);
            m[r] = -__builtin_inff();
            l[r] = 0.0f;
#pragma unroll
            for (int n = 0; n < 8; ++n) o[n][r] = 0.0f;
        }
#pragma unroll
        for (int off = 1; off < 16; off <<= 1) longest = max(longest, __shfl_xor(longest, off, kWave));
        longest = __builtin_amdgcn_readfirstlane(longest);
        for (int chunk = 0; chunk * kChunk < longest; ++chunk) {
            const int pages = min(kChunkPages, (longest - chunk * kChunk + kPage - 1) / kPage);
            const uint8_t* rec[kChunkPages];
            unsigned gone = 0;
#pragma unroll
            for (int p = 0; p < kChunkPages; ++p) {
                const uint8_t* at = p < pages ? kv8_record_uniform(a.c, now, chunk * kChunkPages + p, kvh) : nullptr;
                gone |= at ? 0u : 1u << p;
                rec[p] = at ? at : a.c.pool;
            }
            float s[kChunkPages][4][4];
#pragma unroll
            for (int p = 0; p < kChunkPages; ++p) {
                float dk[4], dv[4];
                token_scales(rec[p], col, dk, dv);
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    const v4i k0 = load16(rec[p], key_at, t * kHeadDim), k1 = load16(rec[p], key_at, t * kHeadDim + 64);
                    v4i d[3];
#pragma unroll
                    for (int g = 0; g < 3; ++g) d[g] = __builtin_amdgcn_mfma_i32_16x16x64_i8(qd[0].d[g], k0, zero, 0, 0, 0);
#pragma unroll
                    for (int g = 0; g < 3; ++g) d[g] = __builtin_amdgcn_mfma_i32_16x16x64_i8(qd[1].d[g], k1, d[g], 0, 0, 0);
                    const int token = (gone >> p) & 1u ? 0x7FFFFFFF : chunk * kChunk + p * kPage + 4 * col + t;
#pragma unroll
                    for (int r = 0; r < 4; ++r) s[p][t][r] = token < lens[r] ? score_of(d[0][r], d[1][r], d[2][r], dk[t]) : -__builtin_inff();
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            float mc[4], lc[4], up[4], unit[4];
            softmax_weights(s, factors, [&](int p, float (&dk)[4], float (&dv)[4]) { token_scales(rec[p], col, dk, dv); }, mc, lc, up, unit);
            int here = lane;
            asm volatile("" : "+v"(here));
            float fa[4], fb[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) fold_step(m[r], l[r], mc[r], lc[r], unit[r], fa[r], fb[r]);
            store_digits(s, up, digits, here);
#pragma unroll
            for (int n = 0; n < 8; ++n) {
                v4i acc[3];
#pragma unroll
                for (int p = 0; p < kChunkPages; ++p) {
                    const v4i v = load16(rec[p], value_at, 256 * n);
#pragma unroll
                    for (int g = 0; g < 3; ++g) acc[g] = __builtin_amdgcn_mfma_i32_16x16x64_i8(load_digits(digits, g, p, here), v, p == 0 ? zero : acc[g], 0, 0, 0);
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) o[n][r] = fold_value(o[n][r], digits_value(acc[0][r], acc[1][r], acc[2][r]), fa[r], fb[r]);
                if (n % 2) __builtin_amdgcn_sched_barrier(0);
            }
        }
        store_rows(a, row0, kvh, members, l, o);
    }
}

// ---------------------------------------------------------------- many rows: the chunks of a tile, one after the other

// A workgroup takes four neighbouring tiles of sixteen (row, head) pairs of one KV head, a tile a wave, through all chunks of the slot they name, the
// running softmax in registers: nothing is stored between.  A chunk comes in eight steps of 8 KB through a ring of three LDS slots, two in flight, one
// barrier a step: the K codes of its four pages, then four times 32 columns of all its V codes, so that a step's digit sums are finished when it
// ends and few are held.  The scales come beside the K codes.  Tiles whose rows name several slots go through them one after the other.
//
// K rows lie in LDS as the products take them: row 16 t + c holds token 4 c + t (so that a lane's scores are of four neighbouring tokens, and four
// digits make a word), its sixteen-byte pieces swizzled by c / 2: a read of sixteen bytes a lane is served in quarters of lanes 0-3, 12-15 and, of the
// next sixteen, 4-11, and those then lie in different banks.  The digits' rows of 256 tokens are swizzled by the pair.
constexpr int kRing = 3, kRingAhead = kRing - 1, kStepBytes = kRecordV;  // slots, steps in flight, bytes of a slot
constexpr int kSteps = 2 * kChunkPages;                             // of a chunk: its pages' K codes, then quarters of its V codes
constexpr int kWalkSlots = 4;                                       // slots that a workgroup's rows may name to be walked together

// DMA instructions of a wave that may stay in flight when step j's data is needed: those of the steps behind it (3 for K codes, 2 for V codes).
constexpr int walk_wait(int j)
{
    int n = 0;
    for (int k = 1; k < kRingAhead; ++k) n += (j + k) % kSteps < kChunkPages ? 3 : 2;
    return n;
}
template <int N>
__device__ __forceinline__ void wait_loads_barrier()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

__global__ __launch_bounds__(256, 2) void kv8_attn_walk_kernel(kv8_attn_args a)
{
    __shared__ __attribute__((aligned(1024))) uint8_t ring[kRing * kStepBytes];
    __shared__ __attribute__((aligned(1024))) uint8_t scales[2 * kChunkPages * 512 + 512];  // two chunks' (K, V of each page); what no one reads
    __shared__ __attribute__((aligned(1024))) uint8_t digits_of[4 * kChunkDigits];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, group = lane >> 4, col = lane & 15;
    uint8_t* digits = digits_of + wave * kChunkDigits;
    const int kvh = blockIdx.x % a.c.Hkv, tile0 = 4 * ((gridDim.x - 1 - blockIdx.x) / a.c.Hkv);  // the last rows, which have most to read, begin
    // lane: pair `col` of tile `group`; every wave knows all four tiles
    const int in_tile = pair_row(a, col), lane_row = (tile0 + group) * a.rows_per_tile + in_tile;
    const bool live = col < a.rows_per_tile * a.G && lane_row < a.R;
    int slot = -1, len = 0;
    if (live) len = row_length(a, lane_row, slot);

    int kinds = 0;
    for (unsigned long long left = __ballot(live); left != 0 && kinds <= kWalkSlots; ++kinds) {
        const int now = __builtin_amdgcn_readlane(slot, __builtin_ctzll(left));
        left &= ~__ballot(live && slot == now);
    }
    if (kinds > kWalkSlots) {
        walk_alone(a, kvh, tile0 + wave, digits_of);
        return;
    }

    const int my_row0 = (tile0 + wave) * a.rows_per_tile;
    uint32_t words[16];
    ask_query(col < a.rows_per_tile * a.G && my_row0 + in_tile < a.R
                  ? a.q + ((size_t)(my_row0 + in_tile) * a.Hq + kvh * a.G + col - in_tile * a.G) * kHeadDim : nullptr,
              words);
    q_digits qd[2];
    float factor, factors[4];
    cut_query(words, a.scale_log2, qd, factor);
#pragma unroll
    for (int r = 0; r < 4; ++r) factors[r] = __shfl(factor, 4 * group + r, kWave);
    const v4i zero = {0, 0, 0, 0};

    // what this wave brings of a step: two blocks of 1 KB, of V codes those of one page; and with K codes one of the page's rows of scales
    const uint32_t ring_at = (uint32_t)(uintptr_t)(lds_char_t*)ring, scales_at = (uint32_t)(uintptr_t)(lds_char_t*)scales;
    uint32_t key_from[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
        const int c = 8 * b + (lane >> 3);  // LDS row 16 wave + c: token 4 c + wave
        key_from[b] = 512 * c + 128 * wave + 16 * ((lane & 7) ^ (c >> 1));
    }
    const uint32_t value_from = kRecordV + 2048 * (lane >> 5) + 16 * (lane & 31);  // of sixteen tokens 32 columns, of the next sixteen too
    const uint32_t scale_from = kRecordKs + 256 * (wave & 1) + 4 * lane;
    // where it reads: a K row's piece, a V operand, a pair's digits
    const uint32_t key_at = 128 * col + 16 * (group ^ (col >> 1)), value_at = 512 * group + 16 * col;

    unsigned long long todo = __ballot(live);
    while (todo != 0) {
        const int now = __builtin_amdgcn_readlane(slot, __builtin_ctzll(todo));
        const unsigned long long all = __ballot(live && slot == now);
        todo &= ~all;
        // of the workgroup, and of this wave's tile
        int longest = (all >> lane) & 1ull ? len : 0;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) longest = max(longest, __shfl_xor(longest, off, kWave));
        longest = __builtin_amdgcn_readfirstlane(longest);
        const unsigned members = (unsigned)(all >> (16 * wave)) & 0xFFFFu;
        const int pair_len = __shfl(len, 16 * wave + col, kWave);
        int mine = (members >> col) & 1u ? pair_len : 0, least = (members >> col) & 1u ? pair_len : 0x7FFFFFFF;
        int lens[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) lens[r] = __shfl(mine, 4 * group + r, kWave);
#pragma unroll
        for (int off = 1; off < 16; off <<= 1) {
            mine = max(mine, __shfl_xor(mine, off, kWave));
            least = min(least, __shfl_xor(least, off, kWave));
        }
        const int my_longest = __builtin_amdgcn_readfirstlane(mine), my_shortest = __builtin_amdgcn_readfirstlane(least);

        float m[4], l[4], o[8][4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            m[r] = -__builtin_inff();
            l[r] = 0.0f;
#pragma unroll
            for (int n = 0; n < 8; ++n) o[n][r] = 0.0f;
        }
        // records of a chunk; where a page is missing, any (its tokens are masked)
        auto look_up = [&](int chunk, const uint8_t* (&rec)[kChunkPages + 1]) {
            unsigned gone = 0;
            rec[kChunkPages] = a.c.pool;
#pragma unroll
            for (int p = 0; p < kChunkPages; ++p) {
                const int page = chunk * kChunkPages + p;
                const uint8_t* at = page * kPage < longest ? kv8_record_uniform(a.c, now, page, kvh) : nullptr;
                gone |= at ? 0u : 1u << p;
                rec[p] = at ? at : a.c.pool;
                rec[kChunkPages] = p == wave ? rec[p] : rec[kChunkPages];  // the page whose V codes this wave brings
            }
            return gone;
        };
        // step j of a chunk with the records rec, into ring slot `to`
        auto bring = [&](int j, const uint8_t* const (&rec)[kChunkPages + 1], int chunk, int to) {
            const uint8_t* from = rec[j < kChunkPages ? j : kChunkPages];
            const uint32_t at = ring_at + to * kStepBytes + 2048 * wave;
            if (j < kChunkPages) {
                dma_block(from, key_from[0], at);
                dma_block(from, key_from[1], at + 1024);
                dma_words(from, scale_from, wave < 2 ? scales_at + ((chunk & 1) * kChunkPages + j) * 512 + 256 * wave
                                                     : scales_at + 2 * kChunkPages * 512 + 256 * (wave - 2));
            } else {
                dma_block(from + 512 * (j - kChunkPages), value_from, at);
                dma_block(from + 512 * (j - kChunkPages) + 4096, value_from, at + 1024);
            }
        };
        const uint8_t *rec[kChunkPages + 1], *next[kChunkPages + 1];
        unsigned gone = look_up(0, rec);
        int place = 0;  // ring slot of the step at hand
#pragma unroll
        for (int j = 0; j < kRingAhead; ++j) bring(j, rec, 0, j);
        for (int chunk = 0; chunk * kChunk < longest; ++chunk) {
            const unsigned next_gone = look_up(chunk + 1, next);
            int here = lane;  // unknown to the compiler: what follows from it is not kept in registers over the loop
            asm volatile("" : "+v"(here));
            const bool busy = chunk * kChunk < my_longest;
            const int pages = min(kChunkPages, (my_longest - chunk * kChunk + kPage - 1) / kPage);  // of this wave's rows
            auto arrive = [&](auto step) {
                constexpr int j = decltype(step)::value;
                wait_loads_barrier<walk_wait(j)>();
                const int to = place == 0 ? kRing - 1 : place - 1;
                if (j + kRingAhead < kSteps) bring((j + kRingAhead) % kSteps, rec, chunk, to);
                else bring((j + kRingAhead) % kSteps, next, chunk + 1, to);
                const uint8_t* codes = ring + place * kStepBytes;
                place = place + 1 == kRing ? 0 : place + 1;
                return codes;
            };
            const uint8_t* chunk_scales = scales + (chunk & 1) * kChunkPages * 512;
            float s[kChunkPages][4][4];  // page, token 4 col + t, pair
            auto keys = [&](auto step) {
                constexpr int p = decltype(step)::value;
                const uint8_t* codes = arrive(step);
                if (!busy || p >= pages) {
#pragma unroll
                    for (int t = 0; t < 4; ++t)
#pragma unroll
                        for (int r = 0; r < 4; ++r) s[p][t][r] = 0.0f;
                    return;
                }
                float dk[4], dv[4];
                clean_scales(chunk_scales + 512 * p, col, dk, dv);
                v4i d[4][3];
#pragma unroll
                for (int two = 0; two < 4; two += 2) {
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int t = two; t < two + 2; ++t) {
                            const v4i k = *reinterpret_cast<const v4i*>(codes + (h ? key_at ^ 64u : key_at) + 2048 * t);
#pragma unroll
                            for (int g = 0; g < 3; ++g) d[t][g] = __builtin_amdgcn_mfma_i32_16x16x64_i8(qd[h].d[g], k, h ? d[t][g] : zero, 0, 0, 0);
                        }
                    __builtin_amdgcn_sched_barrier(0);
                }
#pragma unroll
                for (int t = 0; t < 4; ++t) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) s[p][t][r] = score_of(d[t][0][r], d[t][1][r], d[t][2][r], dk[t]);
                    __builtin_amdgcn_sched_barrier(0);
                }
            };
            keys(std::integral_constant<int, 0>{});
            keys(std::integral_constant<int, 1>{});
            keys(std::integral_constant<int, 2>{});
            keys(std::integral_constant<int, 3>{});
            float fa[4], fb[4];
            if (busy) {
                float mc[4], up[4], unit[4], lc[4];
                if ((chunk + 1) * kChunk > my_shortest || gone != 0) {
#pragma unroll
                    for (int p = 0; p < kChunkPages; ++p)
#pragma unroll
                        for (int t = 0; t < 4; ++t) {
                            const int token = (gone >> p) & 1u ? 0x7FFFFFFF : chunk * kChunk + p * kPage + 4 * (here & 15) + t;
#pragma unroll
                            for (int r = 0; r < 4; ++r) s[p][t][r] = token < lens[r] ? s[p][t][r] : -__builtin_inff();
                        }
                }
                softmax_weights(s, factors, [&](int p, float (&dk)[4], float (&dv)[4]) { clean_scales(chunk_scales + 512 * p, col, dk, dv); }, mc, lc, up, unit);
#pragma unroll
                for (int r = 0; r < 4; ++r) fold_step(m[r], l[r], mc[r], lc[r], unit[r], fa[r], fb[r]);
                store_digits(s, up, digits, here);
            }
            auto values = [&](auto step) {
                constexpr int j = decltype(step)::value - kChunkPages;
                const uint8_t* codes = arrive(step);
                if (!busy) return;
                v4i acc[3][2];
#pragma unroll
                for (int p = 0; p < kChunkPages; ++p) {
                    if (p < pages) {
                        v4i w[3];
#pragma unroll
                        for (int g = 0; g < 3; ++g) w[g] = load_digits(digits, g, p, here);
#pragma unroll
                        for (int n = 0; n < 2; ++n) {
                            const v4i v = *reinterpret_cast<const v4i*>(codes + value_at + 2048 * p + 256 * n);
#pragma unroll
                            for (int g = 0; g < 3; ++g) acc[g][n] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[g], v, p == 0 ? zero : acc[g][n], 0, 0, 0);
                        }
                    }
                }
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        o[2 * j + n][r] = fold_value(o[2 * j + n][r], digits_value(acc[0][n][r], acc[1][n][r], acc[2][n][r]), fa[r], fb[r]);
            };
            values(std::integral_constant<int, 4>{});
            values(std::integral_constant<int, 5>{});
            values(std::integral_constant<int, 6>{});
            values(std::integral_constant<int, 7>{});
            gone = next_gone;
#pragma unroll
            for (int p = 0; p <= kChunkPages; ++p) rec[p] = next[p];
        }
        // the steps asked for past the last chunk have to land before the ring begins anew
        wait_loads_barrier<0>();
        store_rows(a, my_row0, kvh, members, l, o);
    }
}

// Whether a call walks its chunks (nothing in the workspace).
static bool walks(bool named, long long tiles, int Hkv) { return named && tiles * Hkv >= DET_KV8_WALK_TILES; }

size_t attn_decode_kv8_workspace(int R, int Hq, int Hkv, int max_pages, bool named)
{
    const size_t chunks = ((size_t)max_pages + kChunkPages - 1) / kChunkPages;
    // of more rows than these, only calls that walk
    const int most = named ? (DET_KV8_WALK_TILES - 1) / Hkv * (kPairs / (Hq / Hkv)) : R;
    const size_t bytes = (size_t)(R < most ? R : most) * Hq * chunks * (kHeadDim + 4) * sizeof(float);
    return bytes < 16 ? 16 : bytes;
}

int attn_decode_kv8_impl(const void* q, const kv8_cache& cache, const int32_t* seqlens, const int32_t* slots, int len_offset, void* out,
                         void* ws, size_t ws_bytes, int R, int Hq, int D, float scale, hipStream_t s)
{
    if (!q || !seqlens || !out || !ws || R < 1 || Hq < 1 || !(scale > 0.0f) || !(scale < __builtin_inff()))
        return DET_EINVAL;
    const int rc = kv8_check(cache.pool, cache.table, cache.n_pages, cache.n_slots, cache.max_pages, cache.Hkv, D);
    if (rc != DET_OK) return rc;
    if (Hq % cache.Hkv != 0 || Hq / cache.Hkv > kPairs || cache.Hkv > 65535) return DET_ESHAPE;
    if (!slots && cache.n_slots < R) return DET_ESHAPE;
    if (!aligned16(q) || !aligned16(out) || !aligned16(ws)) return DET_EALIGN;
    const int tile_rows = slots ? kPairs / (Hq / cache.Hkv) : 1;
    const long long tiles = ((long long)R + tile_rows - 1) / tile_rows;
    const bool walk = walks(slots != nullptr, tiles, cache.Hkv);
    if (!walk && ws_bytes < attn_decode_kv8_workspace(R, Hq, cache.Hkv, cache.max_pages, false)) return DET_EWORKSPACE;
    kv8_attn_args a{};
    a.q = static_cast<const uint16_t*>(q);
    a.c = cache;
    a.seqlens = seqlens;
    a.slots = slots;
    a.out = static_cast<uint16_t*>(out);
    a.R = R;
    a.Hq = Hq;
    a.G = Hq / cache.Hkv;
    const bool packed = !slots && a.G <= 4;  // rows that share nothing, one to a tile
    a.inverse_G = 65536 / a.G + 1;
    a.rows_per_tile = tile_rows;
    a.len_offset = len_offset;
    a.chunks = (cache.max_pages + kChunkPages - 1) / kChunkPages;
    a.scale_log2 = scale * 1.44269504f;
    const size_t pairs = (size_t)R * Hq * a.chunks;
    a.part_o = static_cast<float*>(ws);
    a.part = reinterpret_cast<float4*>(a.part_o + pairs * kHeadDim);
    if (tiles * cache.Hkv > 0x7FFFFFFFll / 256 || (long long)R * Hq > 0x7FFFFFFFll / 128) return DET_ESHAPE;
    if (walk) {
        hipLaunchKernelGGL(kv8_attn_walk_kernel, dim3((unsigned)((tiles + 3) / 4 * cache.Hkv)), dim3(256), 0, s, a);
        return check_launch();
    }
    if (tiles > 65535) return DET_ESHAPE;
    const long long room = DET_KV8_CHUNK_WGS / (tiles * cache.Hkv);
    a.chunk_step = room < 1 ? 1 : (room < a.chunks ? (int)room : a.chunks);
    const dim3 grid((unsigned)(a.chunk_step * cache.Hkv), (unsigned)tiles);
    if (packed) hipLaunchKernelGGL(kv8_attn_chunk_kernel<true>, grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL(kv8_attn_chunk_kernel<false>, grid, dim3(256), 0, s, a);
    if (a.chunks > 1) hipLaunchKernelGGL(kv8_attn_combine_kernel, dim3((unsigned)(R * Hq)), dim3(128), 0, s, a);
    return check_launch();
}

}  // namespace det

using namespace det;

extern "C" size_t det_attn_decode_kv8_workspace_bytes(int R, int Hq, int Hkv, int D, int max_pages)
{
    if (R < 1 || Hq < 1 || Hkv < 1 || D != kHeadDim || max_pages < 1 || max_pages > DET_KV8_MAX_PAGES || Hq % Hkv != 0) return 0;
    return attn_decode_kv8_workspace(R, Hq, Hkv, max_pages, false);
}

extern "C" size_t det_attn_decode_kv8_rows_workspace_bytes(int R, int Hq, int Hkv, int D, int max_pages)
{
    if (det_attn_decode_kv8_workspace_bytes(R, Hq, Hkv, D, max_pages) == 0 || Hq / Hkv > kPairs) return 0;
    return attn_decode_kv8_workspace(R, Hq, Hkv, max_pages, true);
}

extern "C" int det_attn_decode_kv8(const void* q, const void* pool, const int32_t* page_table, int n_pages, int n_slots, int max_pages,
                                   const int32_t* seqlens, const int32_t* slots, void* out, void* ws, size_t ws_bytes, int R, int Hq, int Hkv,
                                   int D, float scale, void* stream)
{
    const kv8_cache c{static_cast<uint8_t*>(const_cast<void*>(pool)), page_table, n_pages, n_slots, max_pages, Hkv};
    return attn_decode_kv8_impl(q, c, seqlens, slots, 0, out, ws, ws_bytes, R, Hq, D, scale, static_cast<hipStream_t>(stream));
}
