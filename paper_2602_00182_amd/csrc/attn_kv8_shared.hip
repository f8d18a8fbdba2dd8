// Attention over the 8-bit paged cache for rows whose first pages are the same, and the weight that every page gets.
//
// A group's rows hold their first `shared` tokens in the same pages: those chunks are read once for the group, sixteen (row, head) pairs a tile, and
// what a row has behind them is read for itself.  A chunk's sums are the same numbers whoever computes them, and chunks are folded in ascending order in a
// launch of their own, so the bytes are those of det_attn_decode_kv8.
//
// The weight of a page: what the chunk's softmax sums to over its 64 tokens is kept beside the chunk's sums, and a last launch adds it up over the heads
// once the row's largest score and sum are known.
#include "attn_kv8.h"
#include "geometry.h"

namespace det {

struct kv8_shared_args : kv8_attn_args {
    const int32_t* group_rows;  // [n_groups + 1] or null
    const int32_t* shared;      // [n_groups]
    int n_groups;
    float4* page_sums;          // [R, Hq, chunks]: of each page of a chunk the sum of its e, or null
    float2* row_stats;          // [R, Hq]: m and 1 / l
};

// ---------------------------------------------------------------- groups

struct kv8_group {
    int first, row0, rows, chunks;  // its first row; of a tile its own rows; how many chunks are read once for all of them
};

// A group of one row is read like a row without a group.
__device__ __forceinline__ kv8_group group_at(const kv8_shared_args& a, int g)
{
    kv8_group o{0, 0, 0, 0};
    if (g < 0 || g >= a.n_groups) return o;
    o.first = o.row0 = min(max(a.group_rows[g], 0), a.R);
    o.rows = min(a.group_rows[g + 1], a.R) - o.row0;
    if (o.rows >= 2) o.chunks = min(max(a.shared[g], 0) / kChunk, a.chunks);
    return o;
}

// The group of a row: the last one that begins at or in front of it.
__device__ __forceinline__ kv8_group group_of_row(const kv8_shared_args& a, int row)
{
    int begins = 0;
    for (int base = 0; base <= a.n_groups; base += kWave) {
        const int i = base + (threadIdx.x & 63);
        const int n = __popcll(__ballot(i <= a.n_groups && a.group_rows[min(i, a.n_groups)] <= row));
        begins += n;
        if (n < kWave) break;
    }
    return group_at(a, __builtin_amdgcn_readfirstlane(begins - 1));
}

// Tile number `tile` of all groups' tiles of rows_per_tile rows: its group, and row0 / rows of the tile itself; rows = 0 where there is none.
__device__ __forceinline__ kv8_group tile_of_groups(const kv8_shared_args& a, int tile)
{
    const int lane = threadIdx.x & 63;
    int before = 0;
    for (int base = 0; base < a.n_groups; base += kWave) {
        const kv8_group mine = group_at(a, base + lane);
        const int tiles = mine.chunks > 0 ? (mine.rows + a.rows_per_tile - 1) / a.rows_per_tile : 0;
        int sum = tiles;
#pragma unroll
        for (int off = 1; off < kWave; off <<= 1) {
            const int x = __shfl_up(sum, off, kWave);
            sum += lane >= off ? x : 0;
        }
        const unsigned long long past = __ballot(before + sum > tile);
        if (past != 0) {
            const int at = __builtin_ctzll(past);
            kv8_group o{__builtin_amdgcn_readlane(mine.first, at), 0, __builtin_amdgcn_readlane(mine.rows, at), __builtin_amdgcn_readlane(mine.chunks, at)};
            const int skip = (tile - before - (__builtin_amdgcn_readlane(sum, at) - __builtin_amdgcn_readlane(tiles, at))) * a.rows_per_tile;
            o.row0 = o.first + skip;
            o.rows = min(o.rows - skip, a.rows_per_tile);
            return o;
        }
        before += __builtin_amdgcn_readlane(sum, kWave - 1);
    }
    return kv8_group{0, 0, 0, 0};
}

// ---------------------------------------------------------------- chunks of a tile

// Every step-th chunk from first_chunk on, below end_chunk, for `rows` rows from row0 on, all of which read the pages of slot `now`.  As
// kv8_attn_chunk_kernel takes one (attn_kv8.hip): a page a wave for the scores, 32 columns a wave for the weighted sums.
template <bool PACK, bool WEIGHTS>
__device__ __forceinline__ void chunks_of_tile(const kv8_shared_args& a, int kvh, int row0, int rows, int now, int first_chunk, int end_chunk, int step)
{
    constexpr int NP = PACK ? 1 : 4;                 // pairs of a lane
    constexpr int PAIRS = PACK ? 4 : kPairs, DIGITS = PACK ? 1 : 3;
    __shared__ __attribute__((aligned(1024))) uint8_t digits[DIGITS * kPairs * kChunk];
    __shared__ float top[2][4][PAIRS];               // largest score, largest weight of each wave
    __shared__ float lsum[4][PAIRS][16];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, group = lane >> 4, col = lane & 15;
    int slot, len = 0;
    if (col < rows * a.G) len = row_length(a, row0 + pair_row(a, col), slot);
    int longest = len;
#pragma unroll
    for (int off = 1; off < 16; off <<= 1) longest = max(longest, __shfl_xor(longest, off, kWave));
    longest = __builtin_amdgcn_readfirstlane(longest);
    end_chunk = min(end_chunk, (longest + kChunk - 1) / kChunk);
    if (first_chunk >= end_chunk) return;

    const int qp = PACK ? col >> 2 : col, qrow = pair_row(a, qp);  // the pair of this lane's operand row
    uint32_t words[16];
    ask_query(qp < rows * a.G ? a.q + ((size_t)(row0 + qrow) * a.Hq + kvh * a.G + qp - qrow * a.G) * kHeadDim : nullptr, words);
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
    int lens[NP];
#pragma unroll
    for (int r = 0; r < NP; ++r) lens[r] = __shfl(len, PACK ? group : 4 * group + r, kWave);
    bool first = true;
    for (int chunk = first_chunk; chunk < end_chunk; chunk += step) {
        // the chunk's pages; where one is missing, any record (its tokens weigh nothing)
        const uint8_t *rec[kChunkPages], *keys = nullptr;
#pragma unroll
        for (int p = 0; p < kChunkPages; ++p) {
            const int page = chunk * kChunkPages + p;
            const uint8_t* at = page * kPage < longest ? kv8_record_uniform(a.c, now, page, kvh) : nullptr;
            keys = p == wave ? at : keys;
            rec[p] = at ? at : a.c.pool;
        }
        if (!first) __syncthreads();  // the last chunk's digits have been read

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
        float mc[NP], unit[NP], up[NP], f[NP], own[NP];
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
            own[r] = (e[0] + e[1]) + (e[2] + e[3]);
            lsum[wave][p][col] = own[r];
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
            const float page_sum = WEIGHTS ? row_sum(own[r]) : 0.0f;
            if (p >= rows * a.G || lens[r] <= chunk * kChunk) continue;
            const int row = pair_row(a, p);
            const size_t head = (size_t)(row0 + row) * a.Hq + kvh * a.G + p - row * a.G, at = head * a.chunks + chunk;
            if (WEIGHTS && col == 0) reinterpret_cast<float*>(a.page_sums + at)[wave] = page_sum;
            float o[2];
#pragma unroll
            for (int n = 0; n < 2; ++n) o[n] = PACK ? digits_value(acc[0][n][0], acc[0][n][1], acc[0][n][2]) : digits_value(acc[0][n][r], acc[PACK ? 0 : 1][n][r], acc[PACK ? 0 : 2][n][r]);
            if (lens[r] <= kChunk) {  // the row's only chunk
                float fm = -__builtin_inff(), l = 0.0f, fa, fb;
                fold_step(fm, l, mc[r], lc, unit[r], fa, fb);
                const float by = row_factor(l);
                if (WEIGHTS && wave == 0 && col == 0) {
                    a.part[at] = make_float4(mc[r], lc, unit[r], 0.0f);
                    a.row_stats[head] = make_float2(fm, by);
                }
#pragma unroll
                for (int n = 0; n < 2; ++n) __builtin_nontemporal_store(to_bf16(fold_value(0.0f, o[n], fa, fb) * by), &a.out[head * kHeadDim + 32 * wave + 16 * n + col]);
            } else {
                if (wave == 0 && col == 0) a.part[at] = make_float4(mc[r], lc, unit[r], 0.0f);
#pragma unroll
                for (int n = 0; n < 2; ++n) __builtin_nontemporal_store(o[n], &a.part_o[at * kHeadDim + 32 * wave + 16 * n + col]);
            }
        }
    }
}

// The chunks that a group's rows share.  Grid (KV heads x chunk_step, tiles of all groups).
template <bool WEIGHTS>
__global__ __launch_bounds__(256, 2) void kv8_shared_tile_kernel(kv8_shared_args a)
{
    const int kvh = blockIdx.x % a.c.Hkv, first = blockIdx.x / a.c.Hkv;
    const kv8_group tile = tile_of_groups(a, blockIdx.y);
    if (first >= tile.chunks) return;
    // the pages are those of the group's first row
    const int now = a.slots ? a.slots[tile.first] : tile.first;
    chunks_of_tile<false, WEIGHTS>(a, kvh, tile.row0, tile.rows, now, first, tile.chunks, a.chunk_step);
}

// What a row has behind them.  Grid (KV heads x chunk_step, rows).
template <bool PACK, bool WEIGHTS>
__global__ __launch_bounds__(256, PACK ? 3 : 2) void kv8_shared_row_kernel(kv8_shared_args a)
{
    const int kvh = blockIdx.x % a.c.Hkv, nth = blockIdx.x / a.c.Hkv, row = blockIdx.y;
    int slot;
    const int len = row_length(a, row, slot);
    if (len == 0) {
        if (nth == 0)
            for (int i = threadIdx.x; i < a.G * kHeadDim / 2; i += kBlock)
                reinterpret_cast<uint32_t*>(a.out + ((size_t)row * a.Hq + kvh * a.G) * kHeadDim)[i] = 0u;
        return;
    }
    const int behind = a.group_rows ? group_of_row(a, row).chunks : 0;
    chunks_of_tile<PACK, WEIGHTS>(a, kvh, row, 1, slot, behind + nth, a.chunks, a.chunk_step);
}

// The chunks of one (row, head) of more than one chunk, folded in ascending order: kv8_attn_combine_kernel (attn_kv8.hip) and what the weights need.
template <bool WEIGHTS>
__global__ __launch_bounds__(128) void kv8_shared_combine_kernel(kv8_shared_args a)
{
    constexpr int kBlockChunks = 16;
    const size_t at = blockIdx.x;
    int slot;
    const int len = row_length(a, (int)(at / a.Hq), slot);
    if (len <= kChunk) return;
    const int chunks = (len + kChunk - 1) / kChunk;
    const float4* ps = a.part + at * a.chunks;
    const float* po = a.part_o + at * a.chunks * kHeadDim + threadIdx.x;
    float x[2][kBlockChunks];
    auto ask = [&](float (&to)[kBlockChunks], int c0) {
#pragma unroll
        for (int k = 0; k < kBlockChunks; ++k) to[k] = po[(size_t)min(c0 + k, chunks - 1) * kHeadDim];
    };
    ask(x[0], 0);
    float m = -__builtin_inff(), l = 0.0f, o = 0.0f;
    auto fold = [&](const float (&from)[kBlockChunks], int c0) {
        float4 st[kBlockChunks];
#pragma unroll
        for (int k = 0; k < kBlockChunks; ++k) st[k] = ps[min(c0 + k, chunks - 1)];
#pragma unroll
        for (int k = 0; k < kBlockChunks; ++k) {  // past the last chunk: one without tokens, which changes nothing
            const bool there = c0 + k < chunks;
            float fa, fb;
            fold_step(m, l, there ? st[k].x : -__builtin_inff(), there ? st[k].y : 0.0f, st[k].z, fa, fb);
            o = fold_value(o, there ? from[k] : 0.0f, fa, fb);
        }
    };
    for (int c0 = 0; c0 < chunks; c0 += 2 * kBlockChunks) {
        if (c0 + kBlockChunks < chunks) ask(x[1], c0 + kBlockChunks);
        fold(x[0], c0);
        if (c0 + kBlockChunks >= chunks) break;
        if (c0 + 2 * kBlockChunks < chunks) ask(x[0], c0 + 2 * kBlockChunks);
        fold(x[1], c0 + kBlockChunks);
    }
    const float by = row_factor(l);
    if (WEIGHTS && threadIdx.x == 0) a.row_stats[at] = make_float2(m, by);
    __builtin_nontemporal_store(to_bf16(o * by), &a.out[at * kHeadDim + threadIdx.x]);
}

// ---------------------------------------------------------------- the pages' weights

// weights_out[slot] = weights_in[slot] + what the pages get from the rows that name the slot.  Grid (blocks of 64 chunks, slots); a lane has a chunk, a
// wave a quarter of the heads.  Sums in a fixed order: rows ascending, of a row each quarter's heads ascending, then the four quarters.  A
// row whose softmax is not finite adds nothing.
__global__ __launch_bounds__(256) void kv8_page_weights_kernel(kv8_shared_args a, const float* weights_in, float* weights_out)
{
    __shared__ float4 quarter[3][kWave];
    const int slot = blockIdx.y, wave = threadIdx.x >> 6, lane = threadIdx.x & 63, chunk = blockIdx.x * kWave + lane;
    const int each = (a.Hq + 3) / 4, h0 = wave * each, h1 = min(a.Hq, h0 + each);
    float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    auto add_row = [&](int row) {
        int its;
        const int len = row_length(a, row, its);
        if (its != slot || chunk * kChunk >= len) return;
#pragma unroll 8
        for (int h = h0; h < h1; ++h) {
            const size_t head = (size_t)row * a.Hq + h, at = head * a.chunks + chunk;
            const float2 st = a.row_stats[head];
            const float by = pow2_step(a.part[at].x, st.x) * st.y;
            if (!(by < __builtin_inff())) continue;
            const float4 e = a.page_sums[at];
            sum.x = __builtin_fmaf(e.x, by, sum.x);
            sum.y = __builtin_fmaf(e.y, by, sum.y);
            sum.z = __builtin_fmaf(e.z, by, sum.z);
            sum.w = __builtin_fmaf(e.w, by, sum.w);
        }
    };
    if (!a.slots) {
        if (slot < a.R) add_row(slot);
    } else {
        for (int row = 0; row < a.R; ++row) add_row(row);
    }
    if (wave > 0) quarter[wave - 1][lane] = sum;
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int w = 0; w < 3; ++w) {
        const float4 x = quarter[w][lane];
        sum = make_float4(sum.x + x.x, sum.y + x.y, sum.z + x.z, sum.w + x.w);
    }
    const float of[4] = {sum.x, sum.y, sum.z, sum.w};
#pragma unroll
    for (int p = 0; p < kChunkPages; ++p) {
        const int page = chunk * kChunkPages + p;
        if (page >= a.c.max_pages) continue;
        const size_t at = (size_t)slot * a.c.max_pages + page;
        weights_out[at] = (weights_in ? weights_in[at] : 0.0f) + of[p];
    }
}

// ---------------------------------------------------------------- host

struct kv8_shared_ws {
    size_t part, page_sums, row_stats, total;
};

static kv8_shared_ws shared_ws(int R, int Hq, int max_pages, bool weights)
{
    kv8_shared_ws w{};
    const size_t heads = (size_t)R * Hq, all = heads * (((size_t)max_pages + kChunkPages - 1) / kChunkPages);
    w.part = all * kHeadDim * sizeof(float);
    w.page_sums = w.part + all * sizeof(float4);
    w.row_stats = w.page_sums + (weights ? all * sizeof(float4) : 0);
    w.total = w.row_stats + (weights ? heads * sizeof(float2) : 0);
    return w;
}

size_t attn_shared_kv8_workspace(int R, int Hq, int max_pages, bool weights) { return shared_ws(R, Hq, max_pages, weights).total; }

int attn_shared_kv8_impl(const void* q, const kv8_cache& cache, const int32_t* seqlens, const int32_t* slots, int len_offset,
                         const kv8_step& step, void* out, void* ws, size_t ws_bytes, int R, int Hq, int D, float scale, hipStream_t s)
{
    if (!q || !seqlens || !out || !ws || R < 1 || Hq < 1 || !(scale > 0.0f) || !(scale < __builtin_inff())) return DET_EINVAL;
    if (step.n_groups < 0 || (step.n_groups > 0 && (!step.group_rows || !step.shared))) return DET_EINVAL;
    const int rc = kv8_check(cache.pool, cache.table, cache.n_pages, cache.n_slots, cache.max_pages, cache.Hkv, D);
    if (rc != DET_OK) return rc;
    if (Hq % cache.Hkv != 0 || Hq / cache.Hkv > kPairs || cache.Hkv > 65535 || R > 65535 || step.n_groups > R) return DET_ESHAPE;
    if (!slots && cache.n_slots < R) return DET_ESHAPE;
    const bool weights = step.weights_out != nullptr;
    if (weights && cache.n_slots > 65535) return DET_ESHAPE;
    if (!aligned16(q) || !aligned16(out) || !aligned16(ws)) return DET_EALIGN;
    const kv8_shared_ws w = shared_ws(R, Hq, cache.max_pages, weights);
    if (ws_bytes < w.total) return DET_EWORKSPACE;
    char* base = static_cast<char*>(ws);
    kv8_shared_args a{};
    a.q = static_cast<const uint16_t*>(q);
    a.c = cache;
    a.seqlens = seqlens;
    a.slots = slots;
    a.out = static_cast<uint16_t*>(out);
    a.part_o = reinterpret_cast<float*>(base);
    a.part = reinterpret_cast<float4*>(base + w.part);
    a.page_sums = weights ? reinterpret_cast<float4*>(base + w.page_sums) : nullptr;
    a.row_stats = weights ? reinterpret_cast<float2*>(base + w.row_stats) : nullptr;
    a.R = R;
    a.Hq = Hq;
    a.G = Hq / cache.Hkv;
    a.rows_per_tile = kPairs / a.G;
    a.inverse_G = 65536 / a.G + 1;
    a.len_offset = len_offset;
    a.chunks = (cache.max_pages + kChunkPages - 1) / kChunkPages;
    a.scale_log2 = scale * 1.44269504f;
    a.group_rows = step.n_groups > 0 ? step.group_rows : nullptr;
    a.shared = step.shared;
    a.n_groups = step.n_groups;
    if ((long long)R * Hq > 0x7FFFFFFFll / 128) return DET_ESHAPE;
    auto share_out = [&](long long tiles) {
        const long long room = DET_KV8_CHUNK_WGS / (tiles * cache.Hkv);
        a.chunk_step = room < 1 ? 1 : (room < a.chunks ? (int)room : a.chunks);
        return dim3((unsigned)(a.chunk_step * cache.Hkv), (unsigned)tiles);
    };
    if (step.n_groups > 0) {
        // a group of n rows has at most n / rows_per_tile + 1 tiles, and at most n
        const long long tiles = R / a.rows_per_tile + step.n_groups < R ? R / a.rows_per_tile + step.n_groups : R;
        const dim3 grid = share_out(tiles);
        if (weights) hipLaunchKernelGGL(kv8_shared_tile_kernel<true>, grid, dim3(256), 0, s, a);
        else hipLaunchKernelGGL(kv8_shared_tile_kernel<false>, grid, dim3(256), 0, s, a);
    }
    const dim3 grid = share_out(R);
    if (a.G <= 4) {
        if (weights) hipLaunchKernelGGL((kv8_shared_row_kernel<true, true>), grid, dim3(256), 0, s, a);
        else hipLaunchKernelGGL((kv8_shared_row_kernel<true, false>), grid, dim3(256), 0, s, a);
    } else {
        if (weights) hipLaunchKernelGGL((kv8_shared_row_kernel<false, true>), grid, dim3(256), 0, s, a);
        else hipLaunchKernelGGL((kv8_shared_row_kernel<false, false>), grid, dim3(256), 0, s, a);
    }
    if (a.chunks > 1) {
        if (weights) hipLaunchKernelGGL(kv8_shared_combine_kernel<true>, dim3((unsigned)(R * Hq)), dim3(128), 0, s, a);
        else hipLaunchKernelGGL(kv8_shared_combine_kernel<false>, dim3((unsigned)(R * Hq)), dim3(128), 0, s, a);
    }
    if (weights)
        hipLaunchKernelGGL(kv8_page_weights_kernel, dim3((unsigned)((a.chunks + kWave - 1) / kWave), (unsigned)cache.n_slots), dim3(256), 0, s, a,
                           step.weights_in, step.weights_out);
    return check_launch();
}

}  // namespace det

using namespace det;

static bool shared_sizes_ok(int R, int Hq, int Hkv, int D, int max_pages)
{
    return R >= 1 && Hq >= 1 && Hkv >= 1 && D == kHeadDim && max_pages >= 1 && max_pages <= DET_KV8_MAX_PAGES && Hq % Hkv == 0 && Hq / Hkv <= kPairs;
}

extern "C" size_t det_attn_decode_kv8_shared_workspace_bytes(int R, int Hq, int Hkv, int D, int max_pages)
{
    return shared_sizes_ok(R, Hq, Hkv, D, max_pages) ? attn_shared_kv8_workspace(R, Hq, max_pages, false) : 0;
}

extern "C" size_t det_attn_decode_kv8_weights_workspace_bytes(int R, int Hq, int Hkv, int D, int max_pages)
{
    return shared_sizes_ok(R, Hq, Hkv, D, max_pages) ? attn_shared_kv8_workspace(R, Hq, max_pages, true) : 0;
}

extern "C" int det_attn_decode_kv8_shared(const void* q, const void* pool, const int32_t* page_table, int n_pages, int n_slots, int max_pages,
                                          const int32_t* seqlens, const int32_t* slots, const int32_t* group_rows, const int32_t* shared,
                                          int n_groups, void* out, void* ws, size_t ws_bytes, int R, int Hq, int Hkv, int D, float scale,
                                          void* stream)
{
    const kv8_cache c{static_cast<uint8_t*>(const_cast<void*>(pool)), page_table, n_pages, n_slots, max_pages, Hkv};
    return attn_shared_kv8_impl(q, c, seqlens, slots, 0, kv8_step{group_rows, shared, n_groups, nullptr, nullptr}, out, ws, ws_bytes, R, Hq, D, scale,
                                static_cast<hipStream_t>(stream));
}

extern "C" int det_attn_decode_kv8_weights(const void* q, const void* pool, const int32_t* page_table, int n_pages, int n_slots, int max_pages,
                                           const int32_t* seqlens, const int32_t* slots, const int32_t* group_rows, const int32_t* shared,
                                           int n_groups, const float* weights_in, float* weights_out, void* out, void* ws, size_t ws_bytes, int R,
                                           int Hq, int Hkv, int D, float scale, void* stream)
{
    if (!weights_out) return DET_EINVAL;
    const kv8_cache c{static_cast<uint8_t*>(const_cast<void*>(pool)), page_table, n_pages, n_slots, max_pages, Hkv};
    return attn_shared_kv8_impl(q, c, seqlens, slots, 0, kv8_step{group_rows, shared, n_groups, weights_in, weights_out}, out, ws, ws_bytes, R, Hq,
                                D, scale, static_cast<hipStream_t>(stream));
}
