// Attention over the 8-bit paged cache, on the int8 matrix instruction.
//
// Both products are sums of integers, so their order is free and their result exact:
//   scores   q of a (row, head) as a fixed-point number of 23 bits relative to its largest element, in three signed digits of base 256; digit
//            sums are below 2^21 and exact in fp32.
//   values   the weights w_j = e_j d^V_j of a chunk of 256 tokens as fixed-point numbers of 22 bits relative to the chunk's largest, three
//            digits; a chunk's digit sums are below 2^22.  What a weight loses is at most 2^-23 of the largest one, whose own value
//            the cache holds to half a code only.
// Softmax: a chunk's reference m_c is an integer (the ceiling of its largest score in units of log2), so the factors by which chunks are
// brought together are powers of two.  Chunks are folded in ascending order.
#include "kv8.h"

namespace det {

typedef __attribute__((__vector_size__(4 * sizeof(int)))) int v4i;

constexpr int kChunk = 256;               // tokens of a chunk
constexpr int kChunkPages = kChunk / kPage;
constexpr int kPairs = 16;                // (row, head) pairs of a tile
constexpr int kDigitStride = 80;          // bytes of a pair's 64 digits in LDS: padded, so that neither stores nor reads meet in a bank

struct kv8_attn_args {
    const uint16_t* q;  // [R, Hq, 128]
    kv8_cache c;
    const int32_t* seqlens;
    const int32_t* slots;
    uint16_t* out;  // [R, Hq, 128]
    float* part_m;  // [R, Hq, chunks]
    float* part_l;
    float* part_o;  // [R, Hq, chunks, 128]
    int R, Hq, G, rows_per_tile, len_offset, chunks;
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

// Maximum and sum over the sixteen lanes of a row of lanes (rotations: every lane has the result; a sum adds the same pairs in each).
template <int N>
__device__ __forceinline__ float row_ror(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x120 + N, 0xF, 0xF, true));
}
__device__ __forceinline__ float row_max(float v)
{
    v = fmaxf(v, row_ror<8>(v));
    v = fmaxf(v, row_ror<4>(v));
    v = fmaxf(v, row_ror<2>(v));
    return fmaxf(v, row_ror<1>(v));
}
__device__ __forceinline__ float row_sum(float v)
{
    v = v + row_ror<8>(v);
    v = v + row_ror<4>(v);
    v = v + row_ror<2>(v);
    return v + row_ror<1>(v);
}

// The running softmax of a row: weights relative to 2^m, their sum l.  fold_step joins a chunk's (mc, lc) and gives the factors of the
// sums so far (a) and of the chunk's (b).
__device__ __forceinline__ void fold_step(float& m, float& l, float mc, float lc, float& a, float& b)
{
    const float to = fmaxf(m, mc);
    a = pow2_step(m, to);
    b = pow2_step(mc, to);
    l = __builtin_fmaf(lc, b, l * a);
    m = to;
}
// A row that no token reaches has l = 0 and gives zeros.
__device__ __forceinline__ float attn_quotient(float o, float l) { return l == 0.0f ? 0.0f : o / l; }

// ---------------------------------------------------------------- a tile's query

struct tile_q {
    v4i digit[3][2];  // lane: pair lane % 16, columns 32 (lane / 16) + 16 h + 0..15 of the digit (0 the highest)
    float factor[4];  // of the pairs 4 (lane / 16) + 0..3: what an integer score stands for, in units of log2
};

// q: the 128 values of this lane's pair (lane % 16), or null.
__device__ __forceinline__ void load_q(const uint16_t* q, float scale_log2, tile_q& t)
{
    const int lane = threadIdx.x & 63, group = lane >> 4;
    uint32_t w[16] = {};
    if (q) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint4 x = *reinterpret_cast<const uint4*>(q + 32 * group + 8 * k);
            w[4 * k] = x.x, w[4 * k + 1] = x.y, w[4 * k + 2] = x.z, w[4 * k + 3] = x.w;
        }
    }
    float big = 0.0f;
    bool bad = false;
#pragma unroll
    for (int k = 0; k < 16; ++k) {
        const float a = fabsf(bf16lo_to_f32(w[k])), b = fabsf(bf16hi_to_f32(w[k]));
        bad |= !(a < __builtin_inff()) | !(b < __builtin_inff());
        big = fmaxf(big, fmaxf(a, b));
    }
    big = bad ? __builtin_inff() : big;
    big = fmaxf(big, __shfl_xor(big, 16, kWave));
    big = fmaxf(big, __shfl_xor(big, 32, kWave));
    const int e = exponent_above(big);
    const float up = pow2i(22 - e);
    const float factor = big < __builtin_inff() ? scale_log2 * pow2i(e - 22) : __builtin_nanf("");
#pragma unroll
    for (int r = 0; r < 4; ++r) t.factor[r] = __shfl(factor, 4 * group + r, kWave);
#pragma unroll
    for (int k = 0; k < 8; ++k) {  // four columns
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
        t.digit[0][k >> 2][k & 3] = (int)b2;
        t.digit[1][k >> 2][k & 3] = (int)(b1 ^ 0x80808080u);
        t.digit[2][k >> 2][k & 3] = (int)(b0 ^ 0x80808080u);
    }
}

// ---------------------------------------------------------------- one chunk of one slot, one wave

struct chunk_result {
    float m[4], l[4];    // of the pairs 4 (lane / 16) + 0..3
    float o[8][4];       // of the same pairs, column 16 n + lane % 16
};

__device__ __forceinline__ void wave_lds_order()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
}

// len: tokens that each of this lane's four pairs sees of the slot; longest: the largest of the tile's.  digits: 3 * 16 * kDigitStride bytes of LDS
// of this wave.
__device__ __forceinline__ void attend_chunk(const kv8_cache& c, const tile_q& q, int slot, int kvh, int chunk, const int (&len)[4], int longest,
                                             uint8_t* digits, chunk_result& res)
{
    const int lane = threadIdx.x & 63, group = lane >> 4, col = lane & 15;
    const v4i zero = {0, 0, 0, 0};
    const uint8_t* rec[kChunkPages];
#pragma unroll
    for (int p = 0; p < kChunkPages; ++p) {
        const int page = chunk * kChunkPages + p;
        rec[p] = page * kPage < longest ? kv8_record(c, slot, page, kvh) : nullptr;
    }

    float s[kChunkPages][4][4];  // page, token 4 col + t, pair
    float dv[kChunkPages][4];
#pragma unroll
    for (int p = 0; p < kChunkPages; ++p) {
        if (!rec[p]) {
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                dv[p][t] = 0.0f;
#pragma unroll
                for (int r = 0; r < 4; ++r) s[p][t][r] = -__builtin_inff();
            }
            continue;
        }
        const float4 ks = *reinterpret_cast<const float4*>(rec[p] + kRecordKs + 16 * col);
        const float4 vs = *reinterpret_cast<const float4*>(rec[p] + kRecordVs + 16 * col);
        float dk[4] = {ks.x, ks.y, ks.z, ks.w};
        const float dvr[4] = {vs.x, vs.y, vs.z, vs.w};
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            // a V row that is not finite poisons its token's score: the rows that see the token become NaN, the others do not
            dk[t] = dk[t] + 0.0f * dvr[t];
            dv[p][t] = fabsf(dvr[t]) < __builtin_inff() ? dvr[t] : 0.0f;
        }
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const uint8_t* row = rec[p] + (4 * col + t) * kHeadDim + 32 * group;
            const v4i k0 = *reinterpret_cast<const v4i*>(row), k1 = *reinterpret_cast<const v4i*>(row + 16);
            v4i d[3];
#pragma unroll
            for (int g = 0; g < 3; ++g) {
                d[g] = __builtin_amdgcn_mfma_i32_16x16x64_i8(q.digit[g][0], k0, zero, 0, 0, 0);
                d[g] = __builtin_amdgcn_mfma_i32_16x16x64_i8(q.digit[g][1], k1, d[g], 0, 0, 0);
            }
            const int token = chunk * kChunk + p * kPage + 4 * col + t;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float low = (float)(d[1][r] * 256 + d[2][r]) * q.factor[r];
                const float x = __builtin_fmaf((float)d[0][r], 65536.0f * q.factor[r], low) * dk[t];
                s[p][t][r] = token < len[r] ? x : -__builtin_inff();
            }
        }
    }

    // softmax of the chunk relative to an integer power of two; weights against the largest of them
    float safe[4], up[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        float m = -__builtin_inff();
#pragma unroll
        for (int p = 0; p < kChunkPages; ++p)
#pragma unroll
            for (int t = 0; t < 4; ++t) m = fmaxf(m, s[p][t][r]);
        m = __builtin_ceilf(row_max(m));
        res.m[r] = m;
        safe[r] = m == -__builtin_inff() ? 0.0f : m;
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        float sum[kChunkPages], w = 0.0f;
#pragma unroll
        for (int p = 0; p < kChunkPages; ++p) {
            float e[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                e[t] = __builtin_amdgcn_exp2f(s[p][t][r] - safe[r]);
                s[p][t][r] = e[t] * dv[p][t];
                w = fmaxf(w, s[p][t][r]);
            }
            sum[p] = (e[0] + e[1]) + (e[2] + e[3]);
        }
        res.l[r] = row_sum((sum[0] + sum[1]) + (sum[2] + sum[3]));
        const int e = exponent_above(row_max(w));
        up[r] = pow2i(22 - e);
        safe[r] = pow2i(e - 22);
    }

    v4i acc[3][8];
#pragma unroll
    for (int g = 0; g < 3; ++g)
#pragma unroll
        for (int n = 0; n < 8; ++n) acc[g][n] = zero;
#pragma unroll
    for (int p = 0; p < kChunkPages; ++p) {
        if (!rec[p]) continue;
        wave_lds_order();
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            uint32_t y[4], b0, b1, b2;
#pragma unroll
            for (int t = 0; t < 4; ++t) y[t] = __float_as_uint(__builtin_fmaf(s[p][t][r], up[r], 8421504.0f));  // 2^23 + 0x8080
            gather_bytes(y, b0, b1, b2);
            uint8_t* at = digits + (4 * group + r) * kDigitStride + 4 * col;
            *reinterpret_cast<uint32_t*>(at) = b2;
            *reinterpret_cast<uint32_t*>(at + kPairs * kDigitStride) = b1 ^ 0x80808080u;
            *reinterpret_cast<uint32_t*>(at + 2 * kPairs * kDigitStride) = b0 ^ 0x80808080u;
        }
        wave_lds_order();
        v4i w[3];
#pragma unroll
        for (int g = 0; g < 3; ++g) w[g] = *reinterpret_cast<const v4i*>(digits + (g * kPairs + col) * kDigitStride + 16 * group);
#pragma unroll
        for (int n = 0; n < 8; ++n) {
            const v4i v = *reinterpret_cast<const v4i*>(rec[p] + kRecordV + group * (16 * kHeadDim) + (16 * n + col) * 16);
#pragma unroll
            for (int g = 0; g < 3; ++g) acc[g][n] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[g], v, acc[g][n], 0, 0, 0);
        }
    }
#pragma unroll
    for (int n = 0; n < 8; ++n)
#pragma unroll
        for (int r = 0; r < 4; ++r)
            res.o[n][r] = __builtin_fmaf((float)acc[0][n][r], 65536.0f, (float)(acc[1][n][r] * 256 + acc[2][n][r])) * safe[r];
}

// ---------------------------------------------------------------- kernels

// One wave: a tile of up to sixteen (row, head) pairs that read one KV head, one chunk.  Rows of a tile may name different slots: those
// that name the same one go through it together, one slot after the other.  Grid (KV heads, tiles, chunks).
__global__ __launch_bounds__(64, 2) void kv8_attn_chunk_kernel(kv8_attn_args a)
{
    __shared__ __attribute__((aligned(16))) uint8_t digits[3 * kPairs * kDigitStride];
    const int lane = threadIdx.x & 63, group = lane >> 4, col = lane & 15;
    const int kvh = blockIdx.x, chunk = blockIdx.z;
    // this lane's pair: col
    const int row = blockIdx.y * a.rows_per_tile + col / a.G, head = kvh * a.G + col % a.G;
    const bool live = col < a.rows_per_tile * a.G && row < a.R;
    int len = 0, slot = -1;
    if (live) {
        slot = a.slots ? a.slots[row] : row;
        const long long n = (long long)a.seqlens[row] + a.len_offset, most = (long long)a.c.max_pages * kPage;
        len = (unsigned)slot < (unsigned)a.c.n_slots ? (int)(n < 0 ? 0 : (n > most ? most : n)) : 0;
    }
    unsigned todo = (unsigned)(__ballot(len > chunk * kChunk) & 0xFFFFull);
    if (todo == 0) return;
    tile_q q;
    load_q(live ? a.q + ((size_t)row * a.Hq + head) * kHeadDim : nullptr, a.scale_log2, q);
    while (todo != 0) {
        const int now = __builtin_amdgcn_readlane(slot, __builtin_ctz(todo));
        const int mine = slot == now ? len : 0;
        const unsigned members = (unsigned)(__ballot(mine > chunk * kChunk) & 0xFFFFull);
        todo &= ~members;
        int longest = mine;
#pragma unroll
        for (int off = 1; off < 16; off <<= 1) longest = max(longest, __shfl_xor(longest, off, kWave));
        int lens[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) lens[r] = __shfl(mine, 4 * group + r, kWave);
        chunk_result res;
        attend_chunk(a.c, q, now, kvh, chunk, lens, __builtin_amdgcn_readfirstlane(longest), digits, res);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int pair = 4 * group + r;
            if (!((members >> pair) & 1u)) continue;
            const size_t at = ((size_t)(blockIdx.y * a.rows_per_tile + pair / a.G) * a.Hq + kvh * a.G + pair % a.G) * a.chunks + chunk;
            if (col == 0) {
                a.part_m[at] = res.m[r];
                a.part_l[at] = res.l[r];
            }
#pragma unroll
            for (int n = 0; n < 8; ++n) a.part_o[at * kHeadDim + 16 * n + col] = res.o[n][r];
        }
    }
}

// The chunks of one (row, head), folded in ascending order.  Grid (R * Hq), one column a thread.
__global__ __launch_bounds__(128) void kv8_attn_combine_kernel(kv8_attn_args a)
{
    const size_t at = blockIdx.x;
    const int row = (int)(at / a.Hq);
    const int slot = a.slots ? a.slots[row] : row;
    const long long n = (long long)a.seqlens[row] + a.len_offset, most = (long long)a.c.max_pages * kPage;
    const int len = (unsigned)slot < (unsigned)a.c.n_slots ? (int)(n < 0 ? 0 : (n > most ? most : n)) : 0;
    const int chunks = (len + kChunk - 1) / kChunk;
    float m = -__builtin_inff(), l = 0.0f, o = 0.0f;
    for (int c = 0; c < chunks; ++c) {
        float fa, fb;
        fold_step(m, l, a.part_m[at * a.chunks + c], a.part_l[at * a.chunks + c], fa, fb);
        o = __builtin_fmaf(a.part_o[(at * a.chunks + c) * kHeadDim + threadIdx.x], fb, o * fa);
    }
    a.out[at * kHeadDim + threadIdx.x] = f32_to_bf16_rne(attn_quotient(o, l));
}

static size_t workspace_bytes(int R, int Hq, int max_pages)
{
    const size_t chunks = ((size_t)max_pages + kChunkPages - 1) / kChunkPages;
    return (size_t)R * Hq * chunks * (kHeadDim + 2) * sizeof(float);
}

int attn_decode_kv8_impl(const void* q, const kv8_cache& cache, const int32_t* seqlens, const int32_t* slots, int len_offset, void* out,
                         void* ws, size_t ws_bytes, int R, int Hq, int D, float scale, hipStream_t s)
{
    if (!q || !seqlens || !out || !ws || R < 1 || Hq < 1) return DET_EINVAL;
    const int rc = kv8_check(cache.pool, cache.table, cache.n_pages, cache.n_slots, cache.max_pages, cache.Hkv, D);
    if (rc != DET_OK) return rc;
    if (Hq % cache.Hkv != 0 || Hq / cache.Hkv > kPairs || cache.Hkv > 65535) return DET_ESHAPE;
    if (!slots && cache.n_slots < R) return DET_ESHAPE;
    if (!aligned16(q) || !aligned16(out) || !aligned16(ws)) return DET_EALIGN;
    if (ws_bytes < workspace_bytes(R, Hq, cache.max_pages)) return DET_EWORKSPACE;
    kv8_attn_args a{};
    a.q = static_cast<const uint16_t*>(q);
    a.c = cache;
    a.seqlens = seqlens;
    a.slots = slots;
    a.out = static_cast<uint16_t*>(out);
    a.R = R;
    a.Hq = Hq;
    a.G = Hq / cache.Hkv;
    a.rows_per_tile = kPairs / a.G;
    a.len_offset = len_offset;
    a.chunks = (cache.max_pages + kChunkPages - 1) / kChunkPages;
    a.scale_log2 = scale * 1.44269504f;
    const size_t pairs = (size_t)R * Hq * a.chunks;
    a.part_o = static_cast<float*>(ws);
    a.part_m = a.part_o + pairs * kHeadDim;
    a.part_l = a.part_m + pairs;
    const long long tiles = ((long long)R + a.rows_per_tile - 1) / a.rows_per_tile;
    if (tiles > 65535 || a.chunks > 65535 || (long long)R * Hq > 0x7FFFFFFFll / 128) return DET_ESHAPE;
    hipLaunchKernelGGL(kv8_attn_chunk_kernel, dim3(cache.Hkv, (unsigned)tiles, a.chunks), dim3(64), 0, s, a);
    hipLaunchKernelGGL(kv8_attn_combine_kernel, dim3((unsigned)(R * Hq)), dim3(128), 0, s, a);
    return check_launch();
}

}  // namespace det

using namespace det;

extern "C" size_t det_attn_decode_kv8_workspace_bytes(int R, int Hq, int Hkv, int D, int max_pages)
{
    if (R < 1 || Hq < 1 || Hkv < 1 || D != kHeadDim || max_pages < 1 || max_pages > DET_KV8_MAX_PAGES || Hq % Hkv != 0) return 0;
    return workspace_bytes(R, Hq, max_pages);
}

extern "C" int det_attn_decode_kv8(const void* q, const void* pool, const int32_t* page_table, int n_pages, int n_slots, int max_pages,
                                   const int32_t* seqlens, const int32_t* slots, void* out, void* ws, size_t ws_bytes, int R, int Hq, int Hkv,
                                   int D, float scale, void* stream)
{
    const kv8_cache c{static_cast<uint8_t*>(const_cast<void*>(pool)), page_table, n_pages, n_slots, max_pages, Hkv};
    return attn_decode_kv8_impl(q, c, seqlens, slots, 0, out, ws, ws_bytes, R, Hq, D, scale, static_cast<hipStream_t>(stream));
}
