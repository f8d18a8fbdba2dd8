// Attention over the 8-bit paged cache for rows whose first pages are the same, and the weight that every page gets.
//
// A group's rows hold their first `shared` tokens in the same pages: those chunks are read once for the group, sixteen (row, head) pairs a tile, and
// what a row has behind them is read for itself.  A chunk's sums are the same numbers whoever computes them, and chunks are folded in ascending order in a
// launch of their own, so the bytes are those of det_attn_decode_kv8.
//
// With s a token's score in powers of two, m_c = ceil of a chunk's largest and e = 2^(s - m_c), a chunk leaves m_c, l_c = sum e and o_c = sum e v.  The row's
// output is sum 2^(m_c - m) o_c / l with m = max m_c and l = sum 2^(m_c - m) l_c.  The weight of a page is what e sums to over its 64 tokens, kept beside the
// chunk's sums, times 2^(m_c - m) / l, added up over heads and rows in the second launch.
//
// What bounds it: the partial sums of every (row, head, chunk), which the order of folding asks for (528 bytes, written and read), and, from some rows a
// group on, the digits' products: 96 multiplications of 16 x 16 x 64 codes and what prepares them a (tile, page).  64 rows of 32 heads that share 32000
// tokens: 105 + 25 us; the partial sums are 138 MB each way, the cache 135 MB, and 4400 MB if each row were read for itself.
#include <type_traits>

#include "attn_kv8.h"
#include "geometry.h"
#include "stream.h"

namespace det {

struct kv8_shared_args : kv8_attn_args {
    const int32_t* group_rows;  // [n_groups + 1] or null
    const int32_t* shared;      // [n_groups]
    int n_groups;
    float4* page_sums;          // [R, Hq, chunks]: of each page of a chunk the sum of its e, or null
    const float* weights_in;    // [n_slots, max_pages] or null
    float* weights_out;
    int group_wgs, group_steps; // workgroups of a KV head that take shared chunks (at most 2^15 of runs); of them to a tile
    int part_rows;              // rows of a tile, or of the four that go together
    uint32_t part_inverse;
    int row_steps;              // workgroups of a KV head to a row; or 0: what all rows read for themselves is cut into equal runs,
    int row_wgs;                // for so many; or 0: some of group_wgs take them
};

// ---------------------------------------------------------------- groups

struct kv8_group {
    int first, row0, rows, chunks;  // its first row; of a tile its own rows; how many chunks are read once for all of them
};

// A group of one row is read like a row without a group.
__device__ __forceinline__ kv8_group group_at(const kv8_shared_args& a, int g)
{
    const bool is = g < a.n_groups;
    const int begin = a.group_rows[is ? g : 0], end = a.group_rows[is ? g + 1 : 0], shared = a.shared[is ? g : 0];
    kv8_group o;
    o.first = o.row0 = is ? min(max(begin, 0), a.R) : a.R;
    o.rows = is ? min(end, a.R) - o.row0 : 0;
    o.chunks = o.rows >= 2 ? min(max(shared, 0) / kChunk, a.chunks) : 0;
    return o;
}

// The groups are looked at a wave's width at a time; `mine` is this lane's group of the first 64, which a caller loads once.
__device__ __forceinline__ kv8_group group_of_lane(const kv8_group& from, int lane)
{
    return kv8_group{__builtin_amdgcn_readlane(from.first, lane), __builtin_amdgcn_readlane(from.row0, lane), __builtin_amdgcn_readlane(from.rows, lane),
                     __builtin_amdgcn_readlane(from.chunks, lane)};
}

// Chunks that a row's group reads for it.
__device__ __forceinline__ int chunks_before(const kv8_shared_args& a, kv8_group mine, int row)
{
    for (int base = 0; base < a.n_groups; base += kWave) {
        if (base > 0) mine = group_at(a, base + (threadIdx.x & 63));
        const unsigned long long its = __ballot(row >= mine.first && row < mine.first + mine.rows);
        if (its != 0) return __builtin_amdgcn_readlane(mine.chunks, __builtin_ctzll(its));
    }
    return 0;
}

// The same for this lane's row: the last group that begins at or in front of it, among 64 lanes in ascending order, by halves.
__device__ __forceinline__ int chunks_before_lane(const kv8_shared_args& a, kv8_group mine, int row)
{
    int chunks = 0;
    for (int base = 0; base < a.n_groups; base += kWave) {
        if (base > 0) mine = group_at(a, base + (threadIdx.x & 63));
        int g = 0;
        const int last = min(a.n_groups - base, kWave) - 1;
        for (int step = last > 0 ? 1 << (31 - __builtin_clz(last)) : 0; step > 0; step >>= 1) g += __shfl(mine.first, g + step, kWave) <= row ? step : 0;
        const int first = __shfl(mine.first, g, kWave), rows = __shfl(mine.rows, g, kWave), its = __shfl(mine.chunks, g, kWave);
        chunks = row >= first && row < first + rows ? its : chunks;
    }
    return chunks;
}

// How much of something (a count of each group) lies in front of and in this lane's group.
__device__ __forceinline__ int sum_up(int sum)
{
    // within rows of sixteen lanes, then the row in front's total, then that of the half
    sum += __builtin_amdgcn_update_dpp(0, sum, 0x111, 0xF, 0xF, false);
    sum += __builtin_amdgcn_update_dpp(0, sum, 0x112, 0xF, 0xF, false);
    sum += __builtin_amdgcn_update_dpp(0, sum, 0x114, 0xF, 0xF, false);
    sum += __builtin_amdgcn_update_dpp(0, sum, 0x118, 0xF, 0xF, false);
    sum += __builtin_amdgcn_update_dpp(0, sum, 0x142, 0xA, 0xF, false);
    sum += __builtin_amdgcn_update_dpp(0, sum, 0x143, 0xC, 0xF, false);
    return sum;
}
template <class Count>
__device__ __forceinline__ int count_up(const kv8_group& mine, Count count)
{
    return sum_up(count(mine));
}
// How much of it there is in all; sum: count_up of the first 64 groups.
template <class Count>
__device__ __forceinline__ int count_groups(const kv8_shared_args& a, int sum, Count count)
{
    int all = __builtin_amdgcn_readlane(sum, kWave - 1);
    for (int base = kWave; base < a.n_groups; base += kWave) all += __builtin_amdgcn_readlane(count_up(group_at(a, base + (threadIdx.x & 63)), count), kWave - 1);
    return all;
}
// The group that number `at` of it falls into, and how much lies in front of it there.
template <class Count>
__device__ __forceinline__ kv8_group find_group(const kv8_shared_args& a, kv8_group mine, int sum, int at, int& within, Count count)
{
    int before = 0;
    for (int base = 0; base < a.n_groups; base += kWave) {
        if (base > 0) {
            mine = group_at(a, base + (threadIdx.x & 63));
            sum = count_up(mine, count);
        }
        const unsigned long long past = __ballot(before + sum > at);
        if (past != 0) {
            const int g = __builtin_ctzll(past);
            within = at - before - (g > 0 ? __builtin_amdgcn_readlane(sum, g - 1) : 0);
            return group_of_lane(mine, g);
        }
        before += __builtin_amdgcn_readlane(sum, kWave - 1);
    }
    within = 0;
    return kv8_group{0, 0, 0, 0};
}

// Rows by tiles, or by sets of four tiles, of a group; n / rows by one multiplication (rows <= 64, n below 2^17).
struct parts_of_groups {
    int rows;          // of a part
    uint32_t inverse;  // 2^32 / rows, rounded up
    bool chunks;       // a part counts once for each shared chunk
    __device__ __forceinline__ int operator()(const kv8_group& g) const
    {
        const int parts = rows == 1 ? g.rows : (int)__umulhi((uint32_t)(g.rows + rows - 1), inverse);
        return g.chunks > 0 ? (chunks ? parts * g.chunks : parts) : 0;
    }
};

// Part number `nth` of a group: its rows.
__device__ __forceinline__ void take_part(kv8_group& g, int nth, int rows)
{
    g.row0 = g.first + nth * rows;
    g.rows = min(g.rows - nth * rows, rows);
}

// The slot through whose table a group's shared chunks are read: that of the first of its rows that reaches their end, or, of none, that of its longest.
// (A row that has ended, or ends inside, may stand in front; behind its own pages its table says nothing of the group's.  The first length in front of the
// tables: 16 rows of 2900 shared tokens 15.6 -> 15.8 us.)
__device__ __forceinline__ int slot_of_group(const kv8_shared_args& a, const kv8_group& group)
{
    int slot, most = row_length(a, group.first, slot);
    const int need = group.chunks * kChunk, lane = threadIdx.x & 63;
    for (int base = 1; most < need && base < group.rows; base += kWave) {
        int its = -1, len = -1;
        if (base + lane < group.rows) len = row_length(a, group.first + base + lane, its);
        int longest = min(len, need);
#pragma unroll
        for (int off = 1; off < kWave; off <<= 1) longest = max(longest, __shfl_xor(longest, off, kWave));
        longest = __builtin_amdgcn_readfirstlane(longest);
        if (longest > most) {
            most = longest;
            slot = __builtin_amdgcn_readlane(its, __builtin_ctzll(__ballot(min(len, need) == longest)));
        }
    }
    return slot;
}

// ---------------------------------------------------------------- chunks of a tile

// Every step-th chunk from first_chunk on, below end_chunk, for `rows` rows from row0 on, all of which read the pages of slot `now`: of a group, or (rows =
// 1) a row of length row_len.  As kv8_attn_chunk_kernel takes one (attn_kv8.hip): a page a wave for the scores, 32 columns a wave for the weighted sums.
// Calls may follow one another: what the last one read behind its last barrier is not written in front of the first.
// AHEAD: the next chunk's K codes are asked for once the scores are there, its V codes behind the products.  What rows read for themselves beside kRuns, whose
// registers have room: 64 rows of up to 8000 tokens of their own 176 -> 171 us, 16 prompts of 4 rows with up to 4000 103 -> 98; elsewhere a third workgroup a
// unit gives as much.
template <bool PACK>
struct tile_lds {
    static constexpr int PAIRS = PACK ? 4 : kPairs, DIGITS = PACK ? 1 : 3;
    __attribute__((aligned(1024))) uint8_t digits[DIGITS * kPairs * kChunk];
    float top[2][4][PAIRS];  // largest score, largest weight of each wave
    float lsum[4][PAIRS][16];
};

template <bool PACK, bool WEIGHTS, bool GROUP, bool AHEAD = false>
__device__ __forceinline__ void chunks_of_tile(const kv8_shared_args& a, uint8_t* lds, int kvh, int row0, int rows, int row_len, int now,
                                               int first_chunk, int end_chunk, int step)
{
    constexpr int NP = PACK ? 1 : 4;  // pairs of a lane
    constexpr int DIGITS = tile_lds<PACK>::DIGITS;
    tile_lds<PACK>& shared = *reinterpret_cast<tile_lds<PACK>*>(lds);
    auto& digits = shared.digits;
    auto& top = shared.top;
    auto& lsum = shared.lsum;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, group = lane >> 4, col = lane & 15;
    int len = 0, longest = row_len;
    if constexpr (GROUP) {
        int slot;
        if (col < rows * a.G) len = row_length(a, row0 + pair_row(a, col), slot);
        if (len <= kChunk) len = 0;  // such a row is read for itself
        longest = len;
#pragma unroll
        for (int off = 1; off < 16; off <<= 1) longest = max(longest, __shfl_xor(longest, off, kWave));
        longest = __builtin_amdgcn_readfirstlane(longest);
    } else {
        len = col < a.G ? row_len : 0;
    }
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
    const uint8_t *rec[kChunkPages], *keys = nullptr;
    v4i kc[4][2], vc[kChunkPages][2];
    float dk[4], dv_asked[4] = {};
    // the chunk's pages; where one is missing, any record (its tokens weigh nothing)
    auto look_up = [&](int chunk) {
        keys = nullptr;
#pragma unroll
        for (int p = 0; p < kChunkPages; ++p) {
            const int page = chunk * kChunkPages + p;
            const uint8_t* at = page * kPage < longest && (!AHEAD || chunk < end_chunk) ? kv8_record_uniform(a.c, now, page, kvh) : nullptr;
            keys = p == wave ? at : keys;
            rec[p] = at ? at : a.c.pool;
        }
    };
    auto ask_keys = [&] {
        if (!keys) return;
        ask_scales(keys + kRecordKs, col, dk, dv_asked);
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int h = 0; h < 2; ++h) kc[t][h] = load16(keys, key_at, t * kHeadDim + 64 * h);
    };
    auto ask_values = [&] {
#pragma unroll
        for (int p = 0; p < kChunkPages; ++p)
#pragma unroll
            for (int n = 0; n < 2; ++n) vc[p][n] = load16(rec[p], value_at, 256 * n);
    };
    bool first = true;
    for (int chunk = first_chunk; chunk < end_chunk; chunk += step) {
        if (!AHEAD || first) look_up(chunk);
        if (!first) __syncthreads();  // the last chunk's digits have been read
        if (!AHEAD || first) {
            ask_keys();
            ask_values();
        }
        __builtin_amdgcn_sched_barrier(0);
        if (PACK && first) cut();  // while they are on their way
        first = false;
        float dv[4];
        float s[4][NP];
        if (keys) {
#pragma unroll
            for (int t = 0; t < 4; ++t) dv[t] = dv_asked[t];
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
#pragma unroll
            for (int t = 0; t < 4; ++t) dv[t] = 0.0f;
        }
        if constexpr (AHEAD) {
            __builtin_amdgcn_sched_barrier(0);
            look_up(chunk + step);
            ask_keys();
            __builtin_amdgcn_sched_barrier(0);
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
        if constexpr (AHEAD) {
            __builtin_amdgcn_sched_barrier(0);
            ask_values();
            __builtin_amdgcn_sched_barrier(0);
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
            if (!GROUP && lens[r] <= kChunk) {  // the row's only chunk
                float fm = -__builtin_inff(), l = 0.0f, fa, fb;
                fold_step(fm, l, mc[r], lc, unit[r], fa, fb);
                const float by = row_factor(l);
                if (WEIGHTS && wave == 0 && col == 0) a.part[at] = make_float4(mc[r], lc, unit[r], 0.0f);
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

// ---------------------------------------------------------------- chunks of four tiles

// A wave has a tile, and the four go through a run of chunks together: the codes come by LDS-DMA, two pages of K or of V a step, 16 KB, through a ring of
// three slots, two steps in flight, one barrier a step.  A chunk's sums go to memory, so nothing is kept from chunk to chunk and any run of chunks can be a
// workgroup's.  All 128 columns are summed at once (96 sums a lane), page by page: a page's digits are cut while the page in front of it is multiplied, and
// two pages' of them are all that LDS holds.
//
// K rows and their scales lie in LDS as in kv8_attn_walk_kernel (attn_kv8.hip).  V: column 64 h + 4 c + i of sixteen tokens at [h][i][c], so that a lane
// ends with four neighbouring columns of a pair, twice.  Digits: the 64 bytes of pair p at row 4 (p % 4) + p / 4, their sixteen-byte pieces swizzled by
// p % 4: neither writes nor reads meet in a bank.
//
// A chunk's results are stored in the next one's first step, in front of that step's loads: a wait, which counts the loads behind the step it waits for, then
// waits for no load that was asked for later.
//
// A chunk of four tiles takes a workgroup 10 us, two of them on a unit: 1274 vector instructions and 192 products a wave, which hardly run beside each other
// (a product of 16 cycles holds its SIMD's issue for about ten), 8 us without loads and stores.  Registers: 252, and a spill would wait for every load in
// flight; the pairs' factors, lengths and places lie in LDS therefore, and what the pages' weights cost more with 5 and more heads a KV head is spilled outside
// the loop only.
// Against kTiles: 64 rows that share 32000 tokens 123 us against 245, 16 that share 2900 15.8 against 20, but 4 that share 1000, 4 KV heads, 14.2 against 12.0.
constexpr int kRing = 3, kRingAhead = kRing - 1, kStepBytes = 2 * kRecordV;  // slots, steps in flight, bytes of a slot
constexpr int kSteps = kChunkPages;                                          // of a chunk: two pages each, K codes and then V codes
constexpr int kPageDigits = 3 * kPairs * kPage;                          // bytes
constexpr int kRingScales = 2 * kChunkPages * 512 + 512;                 // two chunks' (K, V of each page); what no one reads
struct pair_notes {  // of a wave's sixteen pairs, kept out of the registers
    float factor[kPairs];
    int len[kPairs], head[kPairs];
};
constexpr int kRingLds = kRing * kStepBytes + 8 * kPageDigits + kRingScales + 4 * sizeof(pair_notes);

// Loads of the step behind step j (three a page for K codes, two for V codes).
constexpr int ring_wait(int j) { return (j + 1) % kSteps < kSteps / 2 ? 6 : 4; }

// Chunks c0 .. c1 - 1 of slot `now` for `rows` rows from row0 on, at most four tiles.
template <bool WEIGHTS>
__device__ __forceinline__ void chunks_of_tiles(const kv8_shared_args& a, uint8_t* lds, int kvh, int row0, int rows, int now, int c0, int c1)
{
    uint8_t* const ring = lds;
    uint8_t* const scales = lds + kRing * kStepBytes + 8 * kPageDigits;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, group = lane >> 4, col = lane & 15;
    uint8_t* const digits = lds + kRing * kStepBytes + 2 * kPageDigits * wave;
    pair_notes& notes = reinterpret_cast<pair_notes*>(scales + kRingScales)[wave];
    const int my_row0 = row0 + wave * a.rows_per_tile, my_rows = min(max(rows - wave * a.rows_per_tile, 0), a.rows_per_tile);
    const int in_tile = pair_row(a, col);
    const bool live = col < my_rows * a.G;
    int slot, len = 0;
    if (live) len = row_length(a, my_row0 + in_tile, slot);
    if (len <= kChunk) len = 0;  // such a row is read for itself
    uint32_t words[16];
    ask_query(live ? a.q + ((size_t)(my_row0 + in_tile) * a.Hq + kvh * a.G + col - in_tile * a.G) * kHeadDim : nullptr, words);
    int mine = len, least = len > 0 ? len : 0x7FFFFFFF;
#pragma unroll
    for (int off = 1; off < 16; off <<= 1) {
        mine = max(mine, __shfl_xor(mine, off, kWave));
        least = min(least, __shfl_xor(least, off, kWave));
    }
    const int my_longest = __builtin_amdgcn_readfirstlane(mine), my_shortest = __builtin_amdgcn_readfirstlane(least);

    // what this wave brings of a step: two blocks of 1 KB; and with K codes one of the page's rows of scales
    const uint32_t ring_at = (uint32_t)(uintptr_t)(lds_char_t*)ring, scales_at = (uint32_t)(uintptr_t)(lds_char_t*)scales;
    uint32_t key_from[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
        const int c = 8 * b + (lane >> 3);  // LDS row 16 wave + c: token 4 c + wave
        key_from[b] = 512 * c + 128 * wave + 16 * ((lane & 7) ^ (c >> 1));
    }
    const uint32_t value_from = kRecordV + 2048 * wave + 64 * (lane & 15) + 16 * (lane >> 4);  // sixteen tokens of 64 columns, of the other 64 too
    const uint32_t scale_from = kRecordKs + 256 * (wave & 1) + 4 * lane;
    // where it reads: a K row's piece, a V operand
    const uint32_t key_at = 128 * col + 16 * (group ^ (col >> 1)), value_at = 2048 * group + 16 * col;

    // records of a chunk; where a page is missing, any (its tokens are masked).  The table's entries of sixteen chunks are asked for at once, one a lane.
    int entries = -1;
    auto look_up = [&](int chunk, const uint8_t* (&rec)[kChunkPages]) {
        if ((chunk - c0) % 16 == 0) {
            const int page = chunk * kChunkPages + lane;
            entries = (unsigned)now < (unsigned)a.c.n_slots && page < min(c1 * kChunkPages, a.c.max_pages) ? a.c.table[(size_t)now * a.c.max_pages + page] : -1;
        }
        unsigned gone = 0;
#pragma unroll
        for (int p = 0; p < kChunkPages; ++p) {
            const int page = __builtin_amdgcn_readlane(entries, (chunk - c0) % 16 * kChunkPages + p);
            const bool there = chunk < c1 && (unsigned)page < (unsigned)a.c.n_pages;
            gone |= there ? 0u : 1u << p;
            rec[p] = a.c.pool + (there ? ((size_t)page * a.c.Hkv + kvh) * kRecord : 0);
        }
        return gone;
    };
    // step j of a chunk with the records rec, into ring slot `to`
    auto bring = [&](int j, const uint8_t* const (&rec)[kChunkPages], int chunk, int to) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int p = 2 * (j % 2) + i;
            const uint8_t* from = rec[p];
            const uint32_t at = ring_at + to * kStepBytes + kRecordV * i + 2048 * wave;
            if (j < kSteps / 2) {
                dma_block(from, key_from[0], at);
                dma_block(from, key_from[1], at + 1024);
                dma_words(from, scale_from, wave < 2 ? scales_at + ((chunk & 1) * kChunkPages + p) * 512 + 256 * wave
                                                     : scales_at + 2 * kChunkPages * 512 + 256 * (wave - 2));
            } else {
                dma_block(from, value_from, at);
                dma_block(from + 1024, value_from, at + 1024);
            }
        }
    };
    const uint8_t *rec[kChunkPages], *next[kChunkPages];
    unsigned gone = look_up(c0, rec);
    int place = 0;  // ring slot of the step at hand
#pragma unroll
    for (int j = 0; j < kRingAhead; ++j) bring(j, rec, c0, j);
    q_digits qd[2];  // while they are on their way
    float factor;
    cut_query(words, a.scale_log2, qd, factor);
    if (lane < kPairs) {
        notes.factor[lane] = factor;
        notes.len[lane] = len;
        notes.head[lane] = (my_row0 + in_tile) * a.Hq + kvh * a.G + lane - in_tile * a.G;
    }
    wave_lds_order();
    const v4i zero = {0, 0, 0, 0};
    float o[4][8];     // held back: two times four columns of each pair
    int o_chunk = -1;  // their chunk
    auto flush = [&](int r) {
        if (o_chunk < 0 || notes.len[4 * group + r] <= o_chunk * kChunk) return;
        float* to = a.part_o + ((size_t)notes.head[4 * group + r] * a.chunks + o_chunk) * kHeadDim + 4 * col;
        *reinterpret_cast<float4*>(to) = make_float4(o[r][0], o[r][1], o[r][2], o[r][3]);
        *reinterpret_cast<float4*>(to + 64) = make_float4(o[r][4], o[r][5], o[r][6], o[r][7]);
    };
    // BUSY: the chunk lies in front of the end of this wave's longest row; else the wave only brings what the others need
    auto pass = [&](int chunk, auto is_busy) {
        constexpr bool busy = decltype(is_busy)::value;
        const unsigned next_gone = look_up(chunk + 1, next);
        int here = lane;  // unknown to the compiler: what follows from it is not kept in registers over the loop
        asm volatile("" : "+v"(here));
        float mc[4], lc[4], up[4], unit[4], sums[kChunkPages][4];
        const uint8_t* codes = ring;
        auto arrive = [&](auto step) {  // the step's codes
            constexpr int j = decltype(step)::value;
            wait_loads_barrier<ring_wait(j)>();
            if constexpr (j == 0) {
#pragma unroll
                for (int r = 0; r < 4; ++r) flush(r);
                o_chunk = -1;
            } else if constexpr (j == 2) {
                if (busy && (here & 15) < 4) {
                    const int r = here & 3;
                    auto of = [&](const float (&x)[4]) { return r < 2 ? (r == 0 ? x[0] : x[1]) : (r == 2 ? x[2] : x[3]); };
                    const int p = 4 * (here >> 4) + r;
                    if (notes.len[p] > chunk * kChunk) {
                        const size_t at = (size_t)notes.head[p] * a.chunks + chunk;
                        a.part[at] = make_float4(of(mc), of(lc), of(unit), 0.0f);
                        if (WEIGHTS) a.page_sums[at] = make_float4(of(sums[0]), of(sums[1]), of(sums[2]), of(sums[3]));
                    }
                }
            }
            const int to = place == 0 ? kRing - 1 : place - 1;
            if constexpr (j + kRingAhead < kSteps) bring(j + kRingAhead, rec, chunk, to);
            else bring(j + kRingAhead - kSteps, next, chunk + 1, to);
            codes = ring + place * kStepBytes;
            place = place + 1 == kRing ? 0 : place + 1;
        };
        const uint8_t* chunk_scales = scales + (chunk & 1) * kChunkPages * 512;
        float s[kChunkPages][4][4];  // page, token 4 col + t, pair
        // K codes half a page at a time: while one half is multiplied the one before it becomes scores
        v4i k[2][4], d[2][2][3];
        float dk[2][4];
        auto ask_keys = [&](auto half) {
            constexpr int i = decltype(half)::value, p = i / 2;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    k[i & 1][2 * t + h] = *reinterpret_cast<const v4i*>(codes + p % 2 * kRecordV + (h ? key_at ^ 64u : key_at) + 2048 * (2 * (i & 1) + t));
        };
        auto ask_page_scales = [&](int p) {
            const float4 ks = *reinterpret_cast<const float4*>(chunk_scales + 512 * p + 16 * col);
            const float4 vs = *reinterpret_cast<const float4*>(chunk_scales + 512 * p + 16 * col + (kRecordVs - kRecordKs));
            // poisoned where the token's V row is not finite, as clean_scales does it
            dk[p & 1][0] = __builtin_fmaf(vs.x, 0.0f, ks.x), dk[p & 1][1] = __builtin_fmaf(vs.y, 0.0f, ks.y);
            dk[p & 1][2] = __builtin_fmaf(vs.z, 0.0f, ks.z), dk[p & 1][3] = __builtin_fmaf(vs.w, 0.0f, ks.w);
        };
        auto scores = [&](auto half) {
            constexpr int i = decltype(half)::value, p = i / 2, two = 2 * (i & 1);
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) s[p][two + t][r] = score_of(d[i & 1][t][0][r], d[i & 1][t][1][r], d[i & 1][t][2][r], dk[p & 1][two + t]);
        };
        auto keys = [&](auto half) {
            constexpr int i = decltype(half)::value, p = i / 2;
            if constexpr (i % 4 == 0) {
                arrive(std::integral_constant<int, i / 4>{});
                if constexpr (busy) ask_keys(half);
            }
            if constexpr (busy) {
                if constexpr (i % 2 == 0) ask_page_scales(p);
                if constexpr (i % 4 != 3) ask_keys(std::integral_constant<int, i + 1>{});
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int t = 0; t < 2; ++t)
#pragma unroll
                        for (int g = 0; g < 3; ++g)
                            d[i & 1][t][g] = __builtin_amdgcn_mfma_i32_16x16x64_i8(qd[h].d[g], k[i & 1][2 * t + h], h ? d[i & 1][t][g] : zero, 0, 0, 0);
                if constexpr (i > 0) {
                    scores(std::integral_constant<int, i - 1>{});
#pragma unroll
                    for (int n = 0; n < 12; ++n) {
                        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                        __builtin_amdgcn_sched_group_barrier(0x002, 4, 0);
                    }
                }
            }
        };
        keys(std::integral_constant<int, 0>{});
        keys(std::integral_constant<int, 1>{});
        keys(std::integral_constant<int, 2>{});
        keys(std::integral_constant<int, 3>{});
        keys(std::integral_constant<int, 4>{});
        keys(std::integral_constant<int, 5>{});
        keys(std::integral_constant<int, 6>{});
        keys(std::integral_constant<int, 7>{});
        if constexpr (busy) scores(std::integral_constant<int, 7>{});
        auto cut_page = [&](int p) {
            uint8_t* at = digits + (p & 1) * kPageDigits + 64 * (here >> 4) + 4 * (here & 3);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                uint32_t b[3];
                cut_weights(s[p], r, up[r], b);
#pragma unroll
                for (int g = 0; g < 3; ++g) *reinterpret_cast<uint32_t*>(at + g * kPairs * kPage + 256 * r + 16 * (((here & 15) >> 2) ^ r)) = b[g];
            }
        };
        if constexpr (busy) {
            if ((chunk + 1) * kChunk > my_shortest || gone != 0) {
                const int4 of = *reinterpret_cast<const int4*>(&notes.len[4 * (here >> 4)]);
                const int lens[4] = {of.x, of.y, of.z, of.w};
#pragma unroll
                for (int p = 0; p < kChunkPages; ++p)
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        const int token = (gone >> p) & 1u ? 0x7FFFFFFF : chunk * kChunk + p * kPage + 4 * (here & 15) + t;
#pragma unroll
                        for (int r = 0; r < 4; ++r) s[p][t][r] = token < lens[r] ? s[p][t][r] : -__builtin_inff();
                    }
            }
            const float4 of_pairs = *reinterpret_cast<const float4*>(&notes.factor[4 * (here >> 4)]);
            const float factors[4] = {of_pairs.x, of_pairs.y, of_pairs.z, of_pairs.w};
            auto value_scales = [&](int p, float (&)[4], float (&dv)[4]) {
                const float4 vs = *reinterpret_cast<const float4*>(chunk_scales + 512 * p + 16 * col + (kRecordVs - kRecordKs));
                const float of[4] = {vs.x, vs.y, vs.z, vs.w};
#pragma unroll
                for (int t = 0; t < 4; ++t) dv[t] = fabsf(of[t]) < __builtin_inff() ? of[t] : 0.0f;
            };
            softmax_weights<WEIGHTS>(s, factors, value_scales, mc, lc, up, unit, sums);
            wave_lds_order();
            cut_page(0);
            wave_lds_order();
        }
        v4i acc[3][8];
        auto values = [&](auto page) {
            constexpr int p = decltype(page)::value;
            if constexpr (p % 2 == 0) arrive(std::integral_constant<int, 2 + p / 2>{});
            if constexpr (!busy) return;
            v4i w[3];
#pragma unroll
            for (int g = 0; g < 3; ++g)
                w[g] = *reinterpret_cast<const v4i*>(digits + (p & 1) * kPageDigits + g * kPairs * kPage + 256 * (here & 3) + 64 * ((here & 15) >> 2) +
                                                     16 * ((here >> 4) ^ (here & 3)));
            v4i v[8];
#pragma unroll
            for (int n = 0; n < 8; ++n) v[n] = *reinterpret_cast<const v4i*>(codes + p % 2 * kRecordV + value_at + 1024 * (n >> 2) + 256 * (n & 3));
            if constexpr (p + 1 < kChunkPages) cut_page(p + 1);
#pragma unroll
            for (int n = 0; n < 8; ++n)
#pragma unroll
                for (int g = 0; g < 3; ++g) acc[g][n] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[g], v[n], p == 0 ? zero : acc[g][n], 0, 0, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 7, 0);
#pragma unroll
            for (int n = 0; n < 24; ++n) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x002, 3, 0);
                if (n % 3 == 2 && n < 12) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            }
            wave_lds_order();
        };
        values(std::integral_constant<int, 0>{});
        values(std::integral_constant<int, 1>{});
        values(std::integral_constant<int, 2>{});
        values(std::integral_constant<int, 3>{});
        if constexpr (busy) {
#pragma unroll
            for (int n = 0; n < 8; ++n)
#pragma unroll
                for (int r = 0; r < 4; ++r) o[r][n] = digits_value(acc[0][n][r], acc[1][n][r], acc[2][n][r]);
            o_chunk = chunk;
        }
        gone = next_gone;
#pragma unroll
        for (int p = 0; p < kChunkPages; ++p) rec[p] = next[p];
    };
    int chunk = c0;
    for (; chunk < c1 && chunk * kChunk < my_longest; ++chunk) pass(chunk, std::true_type{});
    for (; chunk < c1; ++chunk) pass(chunk, std::false_type{});
#pragma unroll
    for (int r = 0; r < 4; ++r) flush(r);
    // the steps asked for past the last chunk have to land before the ring begins anew
    wait_loads_barrier<0>();
}

// ---------------------------------------------------------------- the launches

__device__ __forceinline__ void no_tokens(const kv8_shared_args& a, int kvh, int row)
{
    for (int i = threadIdx.x; i < a.G * kHeadDim / 2; i += kBlock) reinterpret_cast<uint32_t*>(a.out + ((size_t)row * a.Hq + kvh * a.G) * kHeadDim)[i] = 0u;
}

// What this lane's row reads for itself: `count` chunks from `first` on (of a row without tokens one, in which its zeros are written).
struct kv8_own {
    int len, slot, first, count;
};
__device__ __forceinline__ kv8_own own_chunks(const kv8_shared_args& a, const kv8_group& mine, int row)
{
    kv8_own o{0, -1, 0, 0};
    if (row < a.R) o.len = row_length(a, row, o.slot);  // asked for in front of the search
    o.first = chunks_before_lane(a, mine, row);
    o.first = o.len > kChunk ? o.first : 0;
    o.count = row < a.R ? max((max(o.len, 1) + kChunk - 1) / kChunk - o.first, 0) : 0;
    return o;
}

// The nth of `parts` runs, equal but for one, of `all`.
__device__ __forceinline__ void run_of(int all, int nth, int parts, int& at, int& to)
{
    const int each = all / parts, rest = all - each * parts;
    at = each * nth + rest * nth / parts;
    to = each * (nth + 1) + rest * (nth + 1) / parts;
}

// Of all rows.
__device__ __forceinline__ int count_own(const kv8_shared_args& a, const kv8_group& mine)
{
    int all = 0;
    for (int base = 0; base < a.R; base += kWave) all += __builtin_amdgcn_readlane(sum_up(own_chunks(a, mine, base + (threadIdx.x & 63)).count), kWave - 1);
    return all;
}

// How many of `wgs` workgroups take the shared chunks, which count twice, if `own` others are left to the rest (one of them at least): as many as their
// share, or fewer if the longest run stays as long.
__device__ __forceinline__ int wgs_of_groups(int shared, int own, int wgs)
{
    const long long twice = 2ll * shared;
    const int share = min(max((int)(twice * wgs / max(twice + own, 1ll)), 1), wgs - 1), longest = (shared + share - 1) / share;
    return longest > 0 ? (shared + longest - 1) / longest : 0;
}

// Grid: workgroups of shared chunks, then those of what rows read for themselves; neighbours take the KV heads of one page, whose records lie side by side.
// kRuns: four tiles go through a run of chunks together.  All chunks of all groups, one behind the other, are cut into equal runs.
// kTiles: a workgroup takes every group_steps-th chunk of a tile.  PACK: a row's up to four heads a KV head.
// A unit holds two workgroups of kRuns at a time (LDS, registers), empty ones among them: their number is kept near 512.
enum { kNoGroups, kTiles, kRuns };
template <int FORM, bool PACK, bool WEIGHTS>
__global__ __launch_bounds__(256, FORM == kNoGroups && PACK ? 3 : 2) void kv8_shared_kernel(kv8_shared_args a)
{
    constexpr int kTileLds = FORM == kNoGroups ? sizeof(tile_lds<PACK>) : sizeof(tile_lds<false>);
    __shared__ __attribute__((aligned(1024))) uint8_t lds[FORM == kRuns && kRingLds > kTileLds ? kRingLds : kTileLds];
    const int kvh = blockIdx.x % a.c.Hkv;
    int nth = blockIdx.x / a.c.Hkv;
    kv8_group mine{};
    if constexpr (FORM != kNoGroups) mine = group_at(a, threadIdx.x & 63);
    if constexpr (FORM == kRuns) {
        const parts_of_groups parts{a.part_rows, a.part_inverse, true};
        int group_wgs = a.group_wgs, row_wgs = a.row_wgs, at, to;
        if (nth < group_wgs) {
            // the shared chunks of all sets of tiles (below 2^30) in group_wgs runs
            const int sum = count_up(mine, parts), shared = count_groups(a, sum, parts);
            if (a.row_steps == 0 && row_wgs == 0) {
                group_wgs = wgs_of_groups(shared, count_own(a, mine), a.group_wgs);
                row_wgs = a.group_wgs - group_wgs;
            }
            if (nth < group_wgs) {
                run_of(shared, nth, group_wgs, at, to);
                while (at < to) {
                    int in;
                    kv8_group set = find_group(a, mine, sum, at, in, parts);
                    if (set.chunks == 0 || in < 0) return;
                    const int nth_set = in / set.chunks, c0 = in - nth_set * set.chunks, c1 = min(set.chunks, c0 + to - at), slot = slot_of_group(a, set);
                    take_part(set, nth_set, a.part_rows);
                    chunks_of_tiles<WEIGHTS>(a, lds, kvh, set.row0, set.rows, slot, c0, c1);
                    at += c1 - c0;
                }
                return;
            }
        }
        nth -= group_wgs;
        // what all rows read for themselves in row_wgs runs; of a chunk or two each, a row is a run
        const int all = a.row_steps == 0 ? count_own(a, mine) : 0;
        if (a.row_steps == 0 && (row_wgs != a.R || all > 2 * a.R)) {
            run_of(all, nth, row_wgs, at, to);
            int before = 0;
            for (int base = 0; base < a.R && at < to; base += kWave) {
                const kv8_own own = own_chunks(a, mine, base + (threadIdx.x & 63));
                const int sum = before + sum_up(own.count);
                before = __builtin_amdgcn_readlane(sum, kWave - 1);
                while (at < min(to, before)) {
                    const int r = __builtin_ctzll(__ballot(sum > at)), len = __builtin_amdgcn_readlane(own.len, r), last = __builtin_amdgcn_readlane(sum, r);
                    const int end = __builtin_amdgcn_readlane(own.first, r) + __builtin_amdgcn_readlane(own.count, r);
                    if (len == 0) no_tokens(a, kvh, base + r);
                    else chunks_of_tile<PACK, WEIGHTS, false, PACK>(a, lds, kvh, base + r, 1, len, __builtin_amdgcn_readlane(own.slot, r), end - (last - at),
                                                                    end - max(last - to, 0), 1);
                    at = min(to, last);
                }
            }
            return;
        }
    }
    if constexpr (FORM == kTiles) {
        if (nth < a.group_wgs) {
            const parts_of_groups parts{a.part_rows, a.part_inverse, false};
            int in;
            kv8_group tile = find_group(a, mine, count_up(mine, parts), nth / a.group_steps, in, parts);
            const int first = nth % a.group_steps;
            if (first >= tile.chunks) return;
            const int slot = slot_of_group(a, tile);
            take_part(tile, in, a.part_rows);
            chunks_of_tile<false, WEIGHTS, true>(a, lds, kvh, tile.row0, tile.rows, 0, slot, first, tile.chunks, a.group_steps);
            return;
        }
        nth -= a.group_wgs;
    }
    const int row_steps = FORM == kRuns ? max(a.row_steps, 1) : a.row_steps, row = nth / row_steps, first = nth % row_steps;
    int slot;
    const int len = row_length(a, row, slot);
    if (len == 0) {
        if (first == 0) no_tokens(a, kvh, row);
        return;
    }
    int behind = 0;
    if constexpr (FORM != kNoGroups) behind = len > kChunk ? chunks_before(a, mine, row) : 0;
    chunks_of_tile<PACK, WEIGHTS, false, FORM == kRuns && PACK>(a, lds, kvh, row, 1, len, slot, behind + first, a.chunks, row_steps);
}

// The chunks of a (row, head) of more than one chunk, folded in ascending order: the operations of kv8_attn_combine_kernel (attn_kv8.hip), down to the
// empty chunks it ends with (a multiple of sixteen in all).  A wave has a head, a lane two columns.  The factors of 64 chunks come from one load, a chunk a
// lane: the largest score so far is a maximum over the lanes in front (exact in any order), the factors follow from it, and are read from their lane
// while the sums are folded.  That leaves ten instructions a chunk and takes the statistics out of the way between two trips to memory: worked out by every
// lane, a column each, they were the launch.  64 rows of 32 heads and 129 chunks 33 -> 25 us, 133 MB at 5.3 TB/s, which bounds it; 8 rows of 16 heads and up to
// 79 chunks with the pages' weights beside them 10.6 -> 7.2.
constexpr int kFoldChunks = 16, kCombineThreads = 128, kCombineHeads = kCombineThreads / kWave;
__device__ __forceinline__ void combine_heads(const kv8_shared_args& a, size_t block)
{
    const int lane = threadIdx.x & 63;
    const size_t at = block * kCombineHeads + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    if (at >= (size_t)a.R * a.Hq) return;
    int slot;
    const int len = row_length(a, (int)(at / a.Hq), slot);
    if (len <= kChunk) return;
    const int chunks = (len + kChunk - 1) / kChunk, all = (chunks + 15) & ~15;
    const float4* ps = a.part + at * a.chunks;
    const float2* po = reinterpret_cast<const float2*>(a.part_o + at * a.chunks * kHeadDim) + lane;
    float2 x[2][kFoldChunks];
    auto ask = [&](float2 (&to)[kFoldChunks], int c0) {
#pragma unroll
        for (int k = 0; k < kFoldChunks; ++k) to[k] = po[(size_t)min(c0 + k, chunks - 1) * (kHeadDim / 2)];
    };
    auto ask_part = [&](int c) { return c < chunks ? ps[c] : make_float4(-__builtin_inff(), 0.0f, 1.0f, 0.0f); };
    auto lane_of = [](float v, int from) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), from)); };
    float4 st = ask_part(lane);
    ask(x[0], 0);
    float m = -__builtin_inff(), l = 0.0f;
    float2 o = make_float2(0.0f, 0.0f);
    for (int c0 = 0; c0 < all; c0 += kWave) {
        float top = st.x;
#pragma unroll
        for (int off = 1; off < kWave; off <<= 1) {
            const float y = __shfl_up(top, off, kWave);
            top = lane >= off ? fmaxf(top, y) : top;
        }
        top = fmaxf(m, top);
        const float up = __shfl_up(top, 1, kWave);
        const float fa = pow2_step(lane == 0 ? m : up, top), fl = pow2_step(st.x, top), fb = fl * st.z, lc = st.y;
        m = lane_of(top, kWave - 1);
        st = ask_part(c0 + kWave + lane);
#pragma unroll
        for (int q = 0; q < kWave / kFoldChunks; ++q) {
            const int c = c0 + q * kFoldChunks;
            if (c >= all) break;
            if (c + kFoldChunks < all) ask(x[(q + 1) & 1], c + kFoldChunks);
#pragma unroll
            for (int k = 0; k < kFoldChunks; ++k) {  // past the last chunk: one without tokens, which changes nothing
                const int i = q * kFoldChunks + k;
                const bool there = c + k < chunks;
                const float by = lane_of(fa, i), in = lane_of(fb, i);
                l = __builtin_fmaf(lane_of(lc, i), lane_of(fl, i), l * by);
                o.x = fold_value(o.x, there ? x[q & 1][k].x : 0.0f, by, in);
                o.y = fold_value(o.y, there ? x[q & 1][k].y : 0.0f, by, in);
            }
        }
    }
    const float by = row_factor(l);
    __builtin_nontemporal_store((uint32_t)to_bf16(o.x * by) | (uint32_t)to_bf16(o.y * by) << 16, reinterpret_cast<uint32_t*>(a.out + at * kHeadDim) + lane);
}

// ---------------------------------------------------------------- the pages' weights

// weights_out[slot] = weights_in[slot] + what sixteen chunks' pages get from the rows that name the slot.  A thread has one chunk and every eighth
// head; the rows' largest scores and sums are folded here again, beside the heads' own workgroups instead of behind them.  Sums in a fixed order:
// of each eighth the rows ascending and in a row its heads, then the eighths.  A row whose softmax is not finite adds nothing.
// Bound by trips to memory: row, statistics, what is added.  Beside the folding 24 rows of 32 heads and up to 24 chunks 5.9 us, 8 of 16 heads and up to 79 chunks 7.2, with
// the statistics asked for behind one another 7.1 and 9.8.
constexpr int kWeightChunks = 16, kWeightParts = kCombineThreads / kWeightChunks;
constexpr int kWeightHeads = 4, kStatChunks = 32;  // heads of a thread, chunks of a head, that are asked for at once
struct weights_lds {
    float2 stats[kCombineThreads];
    float4 parts[kWeightParts - 1][kWeightChunks];
};
__device__ __forceinline__ void page_weights(const kv8_shared_args& a, weights_lds& lds, int slot, int block)
{
    const int tid = threadIdx.x, part = tid / kWeightChunks, chunk = block * kWeightChunks + tid % kWeightChunks;
    float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    auto add_row = [&](int row) {
        int its;
        const int len = row_length(a, row, its), chunks = (len + kChunk - 1) / kChunk;
        if (its != slot || block * kWeightChunks >= chunks) return;
        for (int h0 = 0; h0 < a.Hq; h0 += kCombineThreads) {
            const int count = min(a.Hq - h0, kCombineThreads);
            // what this thread adds of its first heads is asked for before the statistics are worked out
            float4 e[kWeightHeads];
            float mc[kWeightHeads];
            auto ask = [&](int h) {
#pragma unroll
                for (int k = 0; k < kWeightHeads; ++k) {
                    const size_t at = ((size_t)row * a.Hq + h0 + min(h + k * kWeightParts, count - 1)) * a.chunks + min(chunk, chunks - 1);
                    e[k] = a.page_sums[at];
                    mc[k] = a.part[at].x;
                }
            };
            ask(part);
            __syncthreads();
            if (tid < count) {
                const float4* ps = a.part + ((size_t)row * a.Hq + h0 + tid) * a.chunks;
                float m = -__builtin_inff(), l = 0.0f, fa, fb;
                for (int c0 = 0; c0 < chunks; c0 += kStatChunks) {
                    float2 st[kStatChunks];
#pragma unroll
                    for (int k = 0; k < kStatChunks; ++k) st[k] = *reinterpret_cast<const float2*>(&ps[min(c0 + k, chunks - 1)]);
#pragma unroll
                    for (int k = 0; k < kStatChunks; ++k)
                        if (c0 + k < chunks) fold_step(m, l, st[k].x, st[k].y, 1.0f, fa, fb);
                }
                lds.stats[tid] = make_float2(m, row_factor(l));
            }
            __syncthreads();
            for (int h = part; h < count; h += kWeightHeads * kWeightParts) {
                if (h != part) ask(h);
#pragma unroll
                for (int k = 0; k < kWeightHeads; ++k) {
                    if (h + k * kWeightParts >= count) break;
                    const float2 st = lds.stats[h + k * kWeightParts];
                    const float by = pow2_step(mc[k], st.x) * st.y;
                    const bool fine = by < __builtin_inff() && chunk < chunks;
                    sum.x = fine ? __builtin_fmaf(e[k].x, by, sum.x) : sum.x;
                    sum.y = fine ? __builtin_fmaf(e[k].y, by, sum.y) : sum.y;
                    sum.z = fine ? __builtin_fmaf(e[k].z, by, sum.z) : sum.z;
                    sum.w = fine ? __builtin_fmaf(e[k].w, by, sum.w) : sum.w;
                }
            }
        }
    };
    if (!a.slots) {
        if (slot < a.R) add_row(slot);
    } else {
        for (int r0 = 0; r0 < a.R; r0 += kWave) {
            const int r = r0 + (tid & 63);
            for (unsigned long long some = __ballot(r < a.R && a.slots[r] == slot); some != 0; some &= some - 1) add_row(r0 + __builtin_ctzll(some));
        }
    }
    if (part > 0) lds.parts[part - 1][tid % kWeightChunks] = sum;
    __syncthreads();
    if (part > 0) return;
#pragma unroll
    for (int w = 0; w < kWeightParts - 1; ++w) {
        const float4 x = lds.parts[w][tid];
        sum = make_float4(sum.x + x.x, sum.y + x.y, sum.z + x.z, sum.w + x.w);
    }
    const float of[4] = {sum.x, sum.y, sum.z, sum.w};
#pragma unroll
    for (int p = 0; p < kChunkPages; ++p) {
        const int page = chunk * kChunkPages + p;
        if (page >= a.c.max_pages) continue;
        const size_t at = (size_t)slot * a.c.max_pages + page;
        a.weights_out[at] = (a.weights_in ? a.weights_in[at] : 0.0f) + of[p];
    }
}

// Grid: blocks of kCombineHeads of the R * Hq; before them, if the pages are weighed, (blocks of chunks, slots).
template <bool WEIGHTS>
__global__ __launch_bounds__(kCombineThreads) void kv8_shared_combine_kernel(kv8_shared_args a, int weight_blocks)
{
    if constexpr (WEIGHTS) {
        __shared__ weights_lds lds;
        if ((int)blockIdx.x < weight_blocks * a.c.n_slots) {
            page_weights(a, lds, blockIdx.x / weight_blocks, blockIdx.x % weight_blocks);
            return;
        }
        combine_heads(a, blockIdx.x - (size_t)weight_blocks * a.c.n_slots);
    } else {
        combine_heads(a, blockIdx.x);
    }
}

// ---------------------------------------------------------------- host

static size_t shared_chunks(int R, int Hq, int max_pages) { return (size_t)R * Hq * (((size_t)max_pages + kChunkPages - 1) / kChunkPages); }

size_t attn_shared_kv8_workspace(int R, int Hq, int max_pages, bool weights)
{
    return shared_chunks(R, Hq, max_pages) * (kHeadDim * sizeof(float) + (weights ? 2 : 1) * sizeof(float4));
}

template <int FORM, bool PACK>
static void launch_shared(const kv8_shared_args& a, bool weights, unsigned grid, hipStream_t s)
{
    if (weights) hipLaunchKernelGGL((kv8_shared_kernel<FORM, PACK, true>), dim3(grid), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((kv8_shared_kernel<FORM, PACK, false>), dim3(grid), dim3(256), 0, s, a);
}

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
    if (ws_bytes < attn_shared_kv8_workspace(R, Hq, cache.max_pages, weights)) return DET_EWORKSPACE;
    const size_t all = shared_chunks(R, Hq, cache.max_pages);
    kv8_shared_args a{};
    a.q = static_cast<const uint16_t*>(q);
    a.c = cache;
    a.seqlens = seqlens;
    a.slots = slots;
    a.out = static_cast<uint16_t*>(out);
    a.part_o = static_cast<float*>(ws);
    a.part = reinterpret_cast<float4*>(a.part_o + all * kHeadDim);
    a.page_sums = a.part + all;
    a.R = R;
    a.Hq = Hq;
    a.G = Hq / cache.Hkv;
    a.rows_per_tile = kPairs / a.G;
    a.inverse_G = 65536 / a.G + 1;
    a.len_offset = len_offset;
    a.chunks = (cache.max_pages + kChunkPages - 1) / kChunkPages;
    a.scale_log2 = scale * 1.44269504f;
    a.group_rows = step.group_rows;
    a.shared = step.shared;
    a.n_groups = step.n_groups;
    a.weights_in = step.weights_in;
    a.weights_out = step.weights_out;
    // workgroups between which a row's, or a tile's, chunks are shared out
    auto steps = [&](long long rows, long long wgs) {
        const long long room = wgs / (rows * cache.Hkv);
        return room < 1 ? 1 : (room < a.chunks ? (int)room : a.chunks);
    };
    a.row_steps = steps(R, step.n_groups > 0 ? DET_KV8_OWN_WGS : DET_KV8_CHUNK_WGS);
    bool ring = false;
    if (step.n_groups > 0) {
        auto of_head = [&](long long most, long long wgs) {  // workgroups of a KV head
            const long long n = wgs / cache.Hkv < 1 ? 1 : wgs / cache.Hkv;
            return (int)(most < n ? most : n);
        };
        ring = ((long long)R + a.rows_per_tile - 1) / a.rows_per_tile * a.chunks * cache.Hkv >= DET_KV8_RING_CHUNKS;
        if (ring) {
            const long long sets = ((long long)R + 4 * a.rows_per_tile - 1) / (4 * a.rows_per_tile), most = (sets > step.n_groups ? sets : step.n_groups) * a.chunks;
            // Two workgroups a compute unit.  All of them for runs of several chunks, with those of the rows' own chunks behind them; where the shared chunks
            // need not fill them, they are split between both.  60 rows of 6 prompts of 300 to 4000 tokens 35 -> 32 us (28.5 with the steps since), 32 of 4 prompts of 4000 27.4 -> 23.7;
            // 32 of 8 prompts of 4000 would lose (31.9 -> 34.4).
            // What rows read for themselves, in equal runs.  Few rows: against two to eight workgroups a row 16 rows of up to 16000 tokens behind 512 shared ones
            // 120 -> 70 us, 4 of up to 30000 60 -> 41, 16 of 4 prompts of 1000 with up to 8000 78 -> 44; but 16 of 2900 with up to 500 16.0 -> 16.2, 8 of 20000
            // with up to 100 21.9 -> 22.8: the counting.  Up to 64 rows: as many runs as rows; against a workgroup a row 64 rows of 4000 with up to 8000 171 -> 150,
            // of 2000 with up to 4000 94 -> 76, 32 of 4 prompts of 2000 with up to 2000 32.6 -> 29.1, but of 8000 with a chunk 43.3 -> 44.3 and, if rows of a chunk
            // or two were cut too, 60 of 6 prompts 28.4 -> 32.2.  More rows: a workgroup each; counting 256 costs more than it levels (90 -> 110).
            const bool several = most * cache.Hkv >= 2 * DET_KV8_RUN_WGS, few = (long long)R * cache.Hkv < DET_KV8_RUN_WGS / 2;
            if (few || R <= DET_KV8_EVEN_ROWS) a.row_steps = 0;
            a.row_wgs = !few ? R : several ? of_head((long long)R * a.chunks, DET_KV8_OWN_WGS) : 0;
            a.group_wgs = several ? of_head(most, DET_KV8_RUN_WGS) : few ? of_head(most + (long long)R * a.chunks, DET_KV8_RUN_WGS) : of_head(most, DET_KV8_RUN_WGS / 2);
        } else {
            // a group of n rows has at most n / rows_per_tile + 1 tiles, and at most n
            const long long tiles = R / a.rows_per_tile + step.n_groups < R ? R / a.rows_per_tile + step.n_groups : R;
            a.group_steps = steps(tiles, DET_KV8_CHUNK_WGS);
            if (tiles * a.group_steps > 0x3FFFFFFFll) return DET_ESHAPE;
            a.group_wgs = (int)(tiles * a.group_steps);
        }
    }
    a.part_rows = (ring ? 4 : 1) * a.rows_per_tile;
    a.part_inverse = a.part_rows > 1 ? (uint32_t)((1ull << 32) / a.part_rows + ((1ull << 32) % a.part_rows != 0)) : 0u;
    const long long grid = (a.group_wgs + (a.row_steps > 0 ? (long long)R * a.row_steps : a.row_wgs)) * cache.Hkv, blocks = weights ? (a.chunks + kWeightChunks - 1) / kWeightChunks : 0,
                    second = blocks * cache.n_slots + ((long long)R * Hq + kCombineHeads - 1) / kCombineHeads;
    if (grid > 0x7FFFFFFFll / 256 || second > 0x7FFFFFFFll / kCombineThreads) return DET_ESHAPE;
    auto launch = [&](auto form) {
        if (a.G <= 4) launch_shared<decltype(form)::value, true>(a, weights, (unsigned)grid, s);
        else launch_shared<decltype(form)::value, false>(a, weights, (unsigned)grid, s);
    };
    if (ring) launch(std::integral_constant<int, kRuns>{});
    else if (step.n_groups > 0) launch(std::integral_constant<int, kTiles>{});
    else launch(std::integral_constant<int, kNoGroups>{});
    if (weights) hipLaunchKernelGGL(kv8_shared_combine_kernel<true>, dim3((unsigned)second), dim3(kCombineThreads), 0, s, a, (int)blocks);
    else if (a.chunks > 1) hipLaunchKernelGGL(kv8_shared_combine_kernel<false>, dim3((unsigned)second), dim3(kCombineThreads), 0, s, a, 0);
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
