// The 8-bit paged cache: the layout of a page's record, and what its kernels share.
//
// A record holds the 64 tokens of a page for one KV head:
//   K codes [64][128] int8, V codes [4][128][16] int8 (sixteen tokens of a column side by side), K scales [64] fp32, V scales [64] fp32.
// Both are the int8 matrix instruction's operands as they lie: the scores' product runs along a token's 128 values, sixteen bytes a
// lane, and the weighted sum runs along the tokens, so a lane needs sixteen tokens of one column.  Nothing is transposed on the way.
#pragma once

#include "internal.h"

namespace det {

constexpr int kPage = DET_KV8_PAGE;          // tokens of a page
constexpr int kRecord = DET_KV8_RECORD;      // bytes of a page and KV head
constexpr int kHeadDim = 128;
constexpr int kRecordV = kPage * kHeadDim;   // offset of the V codes
constexpr int kRecordKs = 2 * kRecordV;      // of the K scales
constexpr int kRecordVs = kRecordKs + 4 * kPage;
static_assert(kRecord == kRecordVs + 4 * kPage && kRecord % 256 == 0);

struct kv8_cache {
    uint8_t* pool;         // [n_pages, Hkv, kRecord]
    const int32_t* table;  // [n_slots, max_pages]
    int n_pages, n_slots, max_pages, Hkv;
};

// Stores of results that this kernel does not read again, past the caches: a line that an XCD's cache holds changed is written back when the kernel ends,
// and the kernel ends no sooner (copies of 16 pages in 8 layers 17.0 -> 5.6 us, of 400 pages 174 -> 167).
typedef __attribute__((__vector_size__(4 * sizeof(uint32_t)))) uint32_t u32x4;
typedef __attribute__((__vector_size__(2 * sizeof(uint32_t)))) uint32_t u32x2;
__device__ __forceinline__ void stream_store(void* to, const uint4& x)
{
    __builtin_nontemporal_store(u32x4{x.x, x.y, x.z, x.w}, static_cast<u32x4*>(to));
}
__device__ __forceinline__ void stream_store(void* to, const uint2& x) { __builtin_nontemporal_store(u32x2{x.x, x.y}, static_cast<u32x2*>(to)); }

// Record of the page that holds position p of a slot (p within the table), or null where the slot is none or the table names no page.
__device__ __forceinline__ uint8_t* kv8_record(const kv8_cache& c, int slot, int page_of_slot, int kvh)
{
    if ((unsigned)slot >= (unsigned)c.n_slots || (unsigned)page_of_slot >= (unsigned)c.max_pages) return nullptr;
    const int page = c.table[(size_t)slot * c.max_pages + page_of_slot];
    if ((unsigned)page >= (unsigned)c.n_pages) return nullptr;
    return c.pool + ((size_t)page * c.Hkv + kvh) * kRecord;
}

// The same for a slot and page that the whole wave asks for: the table's entry comes by the scalar path, the record's address stays in scalar
// registers.
__device__ __forceinline__ const uint8_t* kv8_record_uniform(const kv8_cache& c, int slot, int page_of_slot, int kvh)
{
    typedef const __attribute__((address_space(4))) int32_t* constant_ints;
    slot = __builtin_amdgcn_readfirstlane(slot);
    page_of_slot = __builtin_amdgcn_readfirstlane(page_of_slot);
    if ((unsigned)slot >= (unsigned)c.n_slots || (unsigned)page_of_slot >= (unsigned)c.max_pages) return nullptr;
    const int page = ((constant_ints)(uintptr_t)c.table)[(size_t)slot * c.max_pages + page_of_slot];
    if ((unsigned)page >= (unsigned)c.n_pages) return nullptr;
    return c.pool + ((size_t)page * c.Hkv + kvh) * kRecord;
}

// det_attn_decode_kv8 with the length taken as seqlens[r] + len_offset (a layer passes its positions and 1).
int attn_decode_kv8_impl(const void* q, const kv8_cache& cache, const int32_t* seqlens, const int32_t* slots, int len_offset, void* out,
                         void* ws, size_t ws_bytes, int R, int Hq, int D, float scale, hipStream_t s);

// Workspace for attn_decode_kv8_impl of up to R rows.  named: its rows name slots, and calls of many of them keep nothing there.
size_t attn_decode_kv8_workspace(int R, int Hq, int Hkv, int max_pages, bool named);

// What a step over the cache is told beside its rows: groups of rows whose first pages are the same, and where the pages' weights go (null: nowhere).
struct kv8_step {
    const int32_t* group_rows;  // [n_groups + 1]
    const int32_t* shared;      // [n_groups]: tokens
    int n_groups;
    const float* weights_in;    // [n_slots, max_pages] or null
    float* weights_out;
};
int attn_shared_kv8_impl(const void* q, const kv8_cache& cache, const int32_t* seqlens, const int32_t* slots, int len_offset,
                         const kv8_step& step, void* out, void* ws, size_t ws_bytes, int R, int Hq, int D, float scale, hipStream_t s);
size_t attn_shared_kv8_workspace(int R, int Hq, int max_pages, bool weights);

inline int kv8_check(const void* pool, const int32_t* table, int n_pages, int n_slots, int max_pages, int Hkv, int D)
{
    if (!pool || !table || n_pages < 1 || n_slots < 1 || max_pages < 1 || Hkv < 1) return DET_EINVAL;
    if (D != kHeadDim || max_pages > DET_KV8_MAX_PAGES) return DET_ESHAPE;
    if (!aligned16(pool)) return DET_EALIGN;
    return DET_OK;
}

}  // namespace det
