// Rows into and out of the 8-bit paged cache, and copies of its pages.
#include "kv8.h"

#include "geometry.h"

namespace det {

// The quantizer on 128 values that eight neighbouring lanes hold, sixteen each: d = max|v| / 127, codes clamp(rint(v / d)); a row that is not finite
// has no codes and the scale NaN.
__device__ __forceinline__ float quantize_row(const float (&v)[16], uint32_t (&codes)[4])
{
    uint32_t big = 0u;  // magnitudes order like the integers of their bits, NaN and infinities are the largest
#pragma unroll
    for (int k = 0; k < 16; ++k) big = max(big, __float_as_uint(v[k]) & 0x7FFFFFFFu);
#pragma unroll
    for (int off = 1; off < 8; off <<= 1) big = max(big, (uint32_t)__shfl_xor((int)big, off, kWave));
    const float d = big < 0x7F800000u ? __uint_as_float(big) / 127.0f : __builtin_nanf("");
#pragma unroll
    for (int k = 0; k < 4; ++k) codes[k] = 0u;
    if (d > 0.0f) {
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            const float n = rintf(v[k] / d);
            const int code = n < -127.0f ? -127 : (n > 127.0f ? 127 : (int)n);
            codes[k >> 2] |= (uint32_t)(code & 0xFF) << (8 * (k & 3));
        }
    }
    return d;
}
__device__ __forceinline__ void widen(const uint4& lo, const uint4& hi, float (&v)[16])
{
    const uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        v[2 * k] = bf16lo_to_f32(w[k]);
        v[2 * k + 1] = bf16hi_to_f32(w[k]);
    }
}

struct append_args {
    const uint16_t* qkv;
    uint16_t* qbuf;
    kv8_cache c;
    const int32_t* positions;
    const int32_t* slots;
    const float* cos_t;
    const float* sin_t;
    int ldqkv, Hq, Lrope, R;
    uint32_t items, item_blocks;
};

// V heads of 32 rows: their codes meet in LDS, and a thread puts sixteen tokens of one column side by side, as the record has them, so that a run of
// neighbouring tokens is stored in pieces of sixteen bytes (3332 rows of 32/8 heads 30 -> 20 us against a byte at a time and half as many heads a thread).
constexpr int kValueRows = 32;
__device__ __forceinline__ void append_values(const append_args& a, uint32_t block, uint8_t (&codes_of)[kValueRows][kHeadDim + 4],
                                              unsigned long long (&place)[kValueRows])
{
    const int kvh = (int)(block % a.c.Hkv), row0 = (int)(block / a.c.Hkv) * kValueRows, i0 = 8 * (int)(threadIdx.x & 7);
#pragma unroll
    for (int u = 0; u < kValueRows / 32; ++u) {
        const int in = 32 * u + (int)(threadIdx.x >> 3), row = min(row0 + in, a.R - 1);
        const int pos = a.positions[row], slot = a.slots ? a.slots[row] : row;
        const uint16_t* x = a.qkv + (size_t)row * a.ldqkv + (a.Hq + a.c.Hkv + kvh) * kHeadDim;
        float v[16];
        widen(*reinterpret_cast<const uint4*>(x + i0), *reinterpret_cast<const uint4*>(x + 64 + i0), v);
        uint32_t codes[4];
        const float d = quantize_row(v, codes);
        *reinterpret_cast<uint32_t*>(&codes_of[in][i0]) = codes[0];
        *reinterpret_cast<uint32_t*>(&codes_of[in][i0 + 4]) = codes[1];
        *reinterpret_cast<uint32_t*>(&codes_of[in][64 + i0]) = codes[2];
        *reinterpret_cast<uint32_t*>(&codes_of[in][68 + i0]) = codes[3];
        if (i0 == 0) {
            // sixteen tokens' codes are aligned to sixteen bytes: the address of theirs and, in its low bits, the token's place among them
            uint8_t* rec = row0 + in < a.R && pos >= 0 ? kv8_record(a.c, slot, pos / kPage, kvh) : nullptr;
            const int t = pos % kPage;
            place[in] = rec ? (unsigned long long)(rec + kRecordV + (t >> 4) * (16 * kHeadDim)) + (t & 15) : 0ull;
            if (rec) *reinterpret_cast<float*>(rec + kRecordVs + 4 * t) = d;
        }
    }
    __syncthreads();
    const int column = threadIdx.x & 127, half = threadIdx.x >> 7;
    uint32_t piece[4] = {0u, 0u, 0u, 0u}, have = 0u;
    unsigned long long at = 0ull;
    for (int k = 0; k <= kValueRows / 2; ++k) {
        const unsigned long long next = k < kValueRows / 2 ? place[half * (kValueRows / 2) + k] : 0ull;
        if ((next & ~15ull) != at) {
            uint8_t* dst = reinterpret_cast<uint8_t*>(at) + 16 * column;
            if (have == 0xFFFFu) {
                stream_store(dst, make_uint4(piece[0], piece[1], piece[2], piece[3]));
            } else if (have != 0u) {
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const uint32_t bits = (have >> (4 * w)) & 15u;
                    if (bits == 15u) *reinterpret_cast<uint32_t*>(dst + 4 * w) = piece[w];
                    else
                        for (int e = 0; e < 4; ++e)
                            if ((bits >> e) & 1u) dst[4 * w + e] = (uint8_t)(piece[w] >> (8 * e));
                }
            }
            have = 0u;
            at = next & ~15ull;
#pragma unroll
            for (int w = 0; w < 4; ++w) piece[w] = 0u;
        }
        if (next != 0ull) {
            const int t = (int)(next & 15ull);
            const uint32_t byte = (uint32_t)codes_of[half * (kValueRows / 2) + k][column] << (8 * (t & 3));
#pragma unroll
            for (int w = 0; w < 4; ++w) piece[w] |= (t >> 2) == w ? byte : 0u;
            have |= 1u << t;
        }
    }
}

// Heads of projection rows, eight lanes a (row, head): lane i holds the rotation pairs 8i..8i+7, i.e. columns 8i..8i+7 and 64+8i..64+8i+7.
// Query heads are rotated into qbuf; key heads are rotated, rounded to bf16 and quantized, value heads quantized as they are.
// Block (256): 32 heads at a time, append_turns times (few rows once: they are all latency, 5.7 -> 4.6 us against twice), everything that can be asked
// for asked for first: the way is position, then its angles; what bounds a prompt is that chain and the bytes (rows in, queries and codes out).  TILED: the value heads in blocks of their own (append_values), from
// item_blocks on.
constexpr int append_turns(bool tiled) { return tiled ? 4 : 1; }
template <bool TILED>
__global__ __launch_bounds__(256) void kv8_append_kernel(append_args a)
{
    constexpr int kAppendTurns = append_turns(TILED);
    const kv8_cache& c = a.c;
    if constexpr (TILED) {
        __shared__ uint8_t codes_of[kValueRows][kHeadDim + 4];
        __shared__ unsigned long long place[kValueRows];
        if (blockIdx.x >= a.item_blocks) {
            append_values(a, blockIdx.x - a.item_blocks, codes_of, place);
            return;
        }
    }
    const uint32_t heads = a.Hq + (TILED ? 1 : 2) * c.Hkv, first = blockIdx.x * (32 * kAppendTurns) + (threadIdx.x >> 3);
    const int i0 = 8 * (int)(threadIdx.x & 7);
    uint4 lo[kAppendTurns], hi[kAppendTurns];
    int pos[kAppendTurns], slot[kAppendTurns], row[kAppendTurns], head[kAppendTurns];
#pragma unroll
    for (int u = 0; u < kAppendTurns; ++u) {
        const uint32_t item = min(first + 32 * u, a.items - 1);
        row[u] = (int)(item / heads);
        head[u] = (int)(item % heads);
        pos[u] = a.positions[row[u]];
        slot[u] = a.slots ? a.slots[row[u]] : row[u];
        const uint16_t* x = a.qkv + (size_t)row[u] * a.ldqkv + head[u] * kHeadDim;
        lo[u] = *reinterpret_cast<const uint4*>(x + i0);
        hi[u] = *reinterpret_cast<const uint4*>(x + 64 + i0);
    }
#pragma unroll
    for (int u = 0; u < kAppendTurns; ++u) {
        if (first + 32 * u >= a.items) return;
        float v[16];
        widen(lo[u], hi[u], v);
        const bool value = !TILED && head[u] >= a.Hq + c.Hkv;
        if (!value) {
            const int p = pos[u] < 0 ? 0 : (pos[u] >= a.Lrope ? a.Lrope - 1 : pos[u]);
            const float4* cp = reinterpret_cast<const float4*>(a.cos_t + (size_t)p * 64 + i0);
            const float4* sp = reinterpret_cast<const float4*>(a.sin_t + (size_t)p * 64 + i0);
            const float4 c0 = cp[0], c1 = cp[1], s0 = sp[0], s1 = sp[1];
            const float cv[8] = {c0.x, c0.y, c0.z, c0.w, c1.x, c1.y, c1.z, c1.w}, sv[8] = {s0.x, s0.y, s0.z, s0.w, s1.x, s1.y, s1.z, s1.w};
#pragma unroll
            for (int k = 0; k < 8; ++k) {  // rope_pair (common.h) on fp32 operands
                const float l = v[k] * cv[k], h = v[8 + k] * cv[k];
                const float x = __builtin_fmaf(-v[8 + k], sv[k], l), y = __builtin_fmaf(v[k], sv[k], h);
                v[k] = bf16_to_f32(f32_to_bf16_rne(x));
                v[8 + k] = bf16_to_f32(f32_to_bf16_rne(y));
            }
            if (head[u] < a.Hq) {
                uint32_t o[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) o[k] = (__float_as_uint(v[2 * k]) >> 16) | (__float_as_uint(v[2 * k + 1]) & 0xFFFF0000u);
                uint16_t* q = a.qbuf + ((size_t)row[u] * a.Hq + head[u]) * kHeadDim;
                stream_store(q + i0, make_uint4(o[0], o[1], o[2], o[3]));
                stream_store(q + 64 + i0, make_uint4(o[4], o[5], o[6], o[7]));
                continue;
            }
        }
        uint32_t codes[4];
        const float d = quantize_row(v, codes);
        if (pos[u] < 0) continue;
        uint8_t* rec = kv8_record(c, slot[u], pos[u] / kPage, value ? head[u] - a.Hq - c.Hkv : head[u] - a.Hq);
        if (!rec) continue;
        const int t = pos[u] % kPage;
        if (!value) {
            stream_store(rec + t * kHeadDim + i0, make_uint2(codes[0], codes[1]));
            stream_store(rec + t * kHeadDim + 64 + i0, make_uint2(codes[2], codes[3]));
        } else {
            uint8_t* dst = rec + kRecordV + (t >> 4) * (16 * kHeadDim) + (t & 15) + 16 * i0;
#pragma unroll
            for (int k = 0; k < 16; ++k) dst[16 * ((k < 8 ? 0 : 56) + k)] = (uint8_t)(codes[k >> 2] >> (8 * (k & 3)));
        }
        if (i0 == 0) *reinterpret_cast<float*>(rec + (value ? kRecordVs : kRecordKs) + 4 * t) = d;
    }
}

// bf16 values of rows of the cache, sixteen lanes a (row, KV head), lane i the columns 8i..8i+7; zeros where there is no page.
__global__ __launch_bounds__(256) void kv8_read_kernel(kv8_cache c, const int32_t* __restrict__ positions, const int32_t* __restrict__ slots,
                                                       uint4* __restrict__ k, uint4* __restrict__ v, long long heads)
{
    const long long at = (long long)blockIdx.x * 16 + (threadIdx.x >> 4);
    if (at >= heads) return;
    const int r = (int)(at / c.Hkv), kvh = (int)(at % c.Hkv), i = threadIdx.x & 15;
    const int pos = positions[r];
    const uint8_t* rec = pos < 0 ? nullptr : kv8_record(c, slots ? slots[r] : r, pos / kPage, kvh);
    uint32_t o[8] = {};
    if (rec) {
        const int t = pos % kPage;
        const uint2 kc = *reinterpret_cast<const uint2*>(rec + t * kHeadDim + 8 * i);
        const uint8_t* vp = rec + kRecordV + (t >> 4) * (16 * kHeadDim) + (t & 15) + 128 * i;
        const float dk = *reinterpret_cast<const float*>(rec + kRecordKs + 4 * t);
        const float dv = *reinterpret_cast<const float*>(rec + kRecordVs + 4 * t);
        auto code = [](uint32_t word, int e) { return (float)(int8_t)(word >> (8 * e)); };
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t w = e < 2 ? kc.x : kc.y;
            o[e] = pack_bf16x2(code(w, 2 * (e & 1)) * dk, code(w, 2 * (e & 1) + 1) * dk);
            o[4 + e] = pack_bf16x2((float)(int8_t)vp[32 * e] * dv, (float)(int8_t)vp[32 * e + 16] * dv);
        }
    }
    stream_store(k + at * 16 + i, make_uint4(o[0], o[1], o[2], o[3]));
    stream_store(v + at * 16 + i, make_uint4(o[4], o[5], o[6], o[7]));
}

// Pages src[i] -> dst[i] of every layer, 16 KB a workgroup.  Grid (pairs, pieces of a page, layers).
__global__ __launch_bounds__(256) void kv8_copy_kernel(uint4* __restrict__ pool, const int32_t* __restrict__ src, const int32_t* __restrict__ dst,
                                                       int n_pages, int vectors)
{
    const int s = src[blockIdx.x], d = dst[blockIdx.x];
    if ((unsigned)s >= (unsigned)n_pages || (unsigned)d >= (unsigned)n_pages || s == d) return;
    const uint4* from = pool + ((size_t)blockIdx.z * n_pages + s) * vectors;
    uint4* to = pool + ((size_t)blockIdx.z * n_pages + d) * vectors;
    const int first = blockIdx.y * 1024 + threadIdx.x;
    uint4 x[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = from[min(first + 256 * k, vectors - 1)];
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (first + 256 * k < vectors) stream_store(to + first + 256 * k, x[k]);
}

}  // namespace det

using namespace det;

extern "C" size_t det_kv8_pool_bytes(int n_pages, int Hkv, int D)
{
    if (n_pages < 1 || Hkv < 1 || D != kHeadDim) return 0;
    return (size_t)n_pages * Hkv * kRecord;
}

extern "C" int det_kv8_rope_append(const void* qkv, int ldqkv, void* qbuf, void* pool, const int32_t* page_table, int n_pages, int n_slots,
                                   int max_pages, const int32_t* positions, const int32_t* slots, const float* rope_cos,
                                   const float* rope_sin, int R, int Hq, int Hkv, int D, int Lrope, void* stream)
{
    if (!qkv || !qbuf || !positions || !rope_cos || !rope_sin || R < 1 || Hq < 1 || Lrope < 1) return DET_EINVAL;
    const int rc = kv8_check(pool, page_table, n_pages, n_slots, max_pages, Hkv, D);
    if (rc != DET_OK) return rc;
    if (Hq > 65536 || Hkv > 65536) return DET_ESHAPE;
    if (ldqkv < (Hq + 2 * Hkv) * D) return DET_EINVAL;
    if (!aligned16(qkv) || !aligned16(qbuf) || !aligned16(rope_cos) || !aligned16(rope_sin) || ldqkv % 8) return DET_EALIGN;
    const kv8_cache c{static_cast<uint8_t*>(pool), page_table, n_pages, n_slots, max_pages, Hkv};
    const bool tiled = R >= DET_KV8_RUN_ROWS;
    const long long items = (long long)R * (Hq + (tiled ? 1 : 2) * Hkv), per_block = 32 * append_turns(tiled), item_blocks = (items + per_block - 1) / per_block;
    const long long blocks = item_blocks + (tiled ? (long long)((R + kValueRows - 1) / kValueRows) * Hkv : 0);
    if (items > 0x7FFFFFFFll || blocks > 0x7FFFFFFFll / 256) return DET_ESHAPE;
    const append_args a{static_cast<const uint16_t*>(qkv), static_cast<uint16_t*>(qbuf), c, positions, slots, rope_cos, rope_sin, ldqkv, Hq, Lrope, R,
                        (uint32_t)items, (uint32_t)item_blocks};
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (tiled) hipLaunchKernelGGL(kv8_append_kernel<true>, dim3((unsigned)blocks), dim3(256), 0, s, a);
    else hipLaunchKernelGGL(kv8_append_kernel<false>, dim3((unsigned)blocks), dim3(256), 0, s, a);
    return check_launch();
}

extern "C" int det_kv8_read(const void* pool, const int32_t* page_table, int n_pages, int n_slots, int max_pages, const int32_t* positions,
                            const int32_t* slots, void* k, void* v, int R, int Hkv, int D, void* stream)
{
    if (!positions || !k || !v || R < 1) return DET_EINVAL;
    const int rc = kv8_check(pool, page_table, n_pages, n_slots, max_pages, Hkv, D);
    if (rc != DET_OK) return rc;
    if (!aligned16(k) || !aligned16(v)) return DET_EALIGN;
    const long long heads = (long long)R * Hkv;
    if ((heads + 15) / 16 > 0x7FFFFFFFll) return DET_ESHAPE;
    const kv8_cache c{static_cast<uint8_t*>(const_cast<void*>(pool)), page_table, n_pages, n_slots, max_pages, Hkv};
    hipLaunchKernelGGL(kv8_read_kernel, dim3((unsigned)((heads + 15) / 16)), dim3(256), 0, static_cast<hipStream_t>(stream), c, positions, slots,
                       static_cast<uint4*>(k), static_cast<uint4*>(v), heads);
    return check_launch();
}

extern "C" int det_kv8_copy_pages(void* pool, int n_layers, int n_pages, int Hkv, int D, const int32_t* src, const int32_t* dst, int n,
                                  void* stream)
{
    if (!pool || !src || !dst || n_layers < 1 || n_pages < 1 || Hkv < 1 || n < 1) return DET_EINVAL;
    const long long vectors = (long long)Hkv * (kRecord / 16), pieces = (vectors + 1023) / 1024;
    if (D != kHeadDim || n_layers > 65535 || pieces > 65535) return DET_ESHAPE;
    if (!aligned16(pool)) return DET_EALIGN;
    hipLaunchKernelGGL(kv8_copy_kernel, dim3(n, (unsigned)pieces, n_layers), dim3(256), 0, static_cast<hipStream_t>(stream),
                       static_cast<uint4*>(pool), src, dst, n_pages, (int)vectors);
    return check_launch();
}
