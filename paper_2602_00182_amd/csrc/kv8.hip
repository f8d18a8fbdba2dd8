// Rows into and out of the 8-bit paged cache, and copies of its pages.
#include "kv8.h"

namespace det {

// One row's heads of qkv, sixteen lanes a head: lane i holds the rotation pairs 4i..4i+3, i.e. columns 4i..4i+3 and 64+4i..64+4i+3.
// Query heads are rotated into qbuf; key heads are rotated, rounded to bf16 and quantized, value heads quantized as they are.
// Block (256): sixteen heads.  Grid (R, ceil((Hq + 2 Hkv) / 16)).
__global__ __launch_bounds__(256) void kv8_append_kernel(const uint16_t* __restrict__ qkv, int ldqkv, uint16_t* __restrict__ qbuf, kv8_cache c,
                                                         const int32_t* __restrict__ positions, const int32_t* __restrict__ slots,
                                                         const float* __restrict__ cos_t, const float* __restrict__ sin_t, int Hq, int Lrope)
{
    const int r = blockIdx.x, head = blockIdx.y * 16 + (int)(threadIdx.x >> 4), i0 = 4 * (int)(threadIdx.x & 15);
    if (head >= Hq + 2 * c.Hkv) return;
    const int pos = positions[r];
    const uint16_t* x = qkv + (size_t)r * ldqkv + head * kHeadDim;
    const uint2 lo = *reinterpret_cast<const uint2*>(x + i0), hi = *reinterpret_cast<const uint2*>(x + 64 + i0);
    uint16_t y[8] = {(uint16_t)lo.x, (uint16_t)(lo.x >> 16), (uint16_t)lo.y, (uint16_t)(lo.y >> 16),
                     (uint16_t)hi.x, (uint16_t)(hi.x >> 16), (uint16_t)hi.y, (uint16_t)(hi.y >> 16)};
    if (head < Hq + c.Hkv) {
        const int p = pos < 0 ? 0 : (pos >= Lrope ? Lrope - 1 : pos);
        const float4 cs = *reinterpret_cast<const float4*>(cos_t + (size_t)p * 64 + i0);
        const float4 sn = *reinterpret_cast<const float4*>(sin_t + (size_t)p * 64 + i0);
        const float cv[4] = {cs.x, cs.y, cs.z, cs.w}, sv[4] = {sn.x, sn.y, sn.z, sn.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            uint16_t a, b;
            rope_pair(y[k], y[4 + k], cv[k], sv[k], a, b);
            y[k] = a;
            y[4 + k] = b;
        }
    }
    if (head < Hq) {
        uint16_t* q = qbuf + ((size_t)r * Hq + head) * kHeadDim;
        *reinterpret_cast<uint2*>(q + i0) = make_uint2(y[0] | ((uint32_t)y[1] << 16), y[2] | ((uint32_t)y[3] << 16));
        *reinterpret_cast<uint2*>(q + 64 + i0) = make_uint2(y[4] | ((uint32_t)y[5] << 16), y[6] | ((uint32_t)y[7] << 16));
        return;
    }

    // The quantizer: d = max|y| / 127, codes clamp(rint(y / d)); a row that is not finite has no codes and the scale NaN.
    float v[8], amax = 0.0f;
    bool bad = false;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        v[k] = bf16_to_f32(y[k]);
        bad |= !(fabsf(v[k]) < __builtin_inff());
        amax = fmaxf(amax, fabsf(v[k]));
    }
    amax = bad ? __builtin_inff() : amax;
#pragma unroll
    for (int off = 1; off < 16; off <<= 1) amax = fmaxf(amax, __shfl_xor(amax, off, kWave));
    const bool finite = amax < __builtin_inff();
    const float d = finite ? amax / 127.0f : __builtin_nanf("");
    uint32_t codes[2] = {0u, 0u};
    if (d > 0.0f) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float n = rintf(v[k] / d);
            const int code = n < -127.0f ? -127 : (n > 127.0f ? 127 : (int)n);
            codes[k >> 2] |= (uint32_t)(code & 0xFF) << (8 * (k & 3));
        }
    }
    if (pos < 0) return;
    const bool key = head < Hq + c.Hkv;
    uint8_t* rec = kv8_record(c, slots ? slots[r] : r, pos / kPage, key ? head - Hq : head - Hq - c.Hkv);
    if (!rec) return;
    const int t = pos % kPage;
    if (key) {
        *reinterpret_cast<uint32_t*>(rec + t * kHeadDim + i0) = codes[0];
        *reinterpret_cast<uint32_t*>(rec + t * kHeadDim + 64 + i0) = codes[1];
    } else {
        uint8_t* dst = rec + kRecordV + (t >> 4) * (16 * kHeadDim) + (t & 15);
#pragma unroll
        for (int k = 0; k < 8; ++k) dst[16 * ((k < 4 ? 0 : 60) + i0 + k)] = (uint8_t)(codes[k >> 2] >> (8 * (k & 3)));
    }
    if (i0 == 0) *reinterpret_cast<float*>(rec + (key ? kRecordKs : kRecordVs) + 4 * t) = d;
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
    k[at * 16 + i] = make_uint4(o[0], o[1], o[2], o[3]);
    v[at * 16 + i] = make_uint4(o[4], o[5], o[6], o[7]);
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
        if (first + 256 * k < vectors) to[first + 256 * k] = x[k];
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
    hipLaunchKernelGGL(kv8_append_kernel, dim3(R, (Hq + 2 * Hkv + 15) / 16), dim3(256), 0, static_cast<hipStream_t>(stream),
                       static_cast<const uint16_t*>(qkv), ldqkv, static_cast<uint16_t*>(qbuf), c, positions, slots, rope_cos, rope_sin, Hq,
                       Lrope);
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
