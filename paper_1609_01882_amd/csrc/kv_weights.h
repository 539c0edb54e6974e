// The weight that every token of an attention memory received.
#pragma once

#include <algorithm>

#include "kv_device.h"

namespace psc {
namespace {

// The weight that every token received, from the scores that the attention left: a thread to four slots.  For up to
// kScoreRows rows (query heads times rows of a sequence): the scores' 4 bytes to a row, written and read, are then less than
// the keys' bytes and what comes with expanding them (32 x 4k tokens, 4 rows: 31 us with the keys once more).  They are kept up to a
// size that a caller can spare (whole calls of 8 rows x 128, kept and not: 8 x 8 x 131k tokens, 0.27 GB of scores, 269 and 355 us;
// 16 x 8 x 262k, 1.1 GB, 1118 and 1426).
constexpr int kScoreRows = 8;
constexpr int64_t kMostScoreBytes = (int64_t)4 << 30;
//
// kHeads = 2: a pair of kv heads holds the same tokens, and each receives what both maps give (differential attention).
template <int N, int kHeads>
__global__ __launch_bounds__(256) void kv_weights_of_scores_kernel(KvView c, KvQueries q, const float *given, float *received)
{
    const int b = (int)blockIdx.z / (c.heads / kHeads), head = (int)blockIdx.z % (c.heads / kHeads) * kHeads;
    const int64_t stride = (int64_t)c.width << c.page_shift, dense = (int64_t)blockIdx.z * kHeads * stride;
    const int64_t first = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (first >= stride) return;
    const int slot = (int)first;
    const RowSet s = rows_of(c, q, b);
    const int m_all = s.rows * q.group;
    f32x4 total[kHeads];
#pragma unroll
    for (int which = 0; which < kHeads; ++which)
        total[which] = given ? *(const f32x4 *)(given + dense + which * stride + slot) : f32x4{0.f, 0.f, 0.f, 0.f};
    if (slot < s.n && m_all > 0) {
        const Blocks blocks = blocks_of(q, s.n, s.first_pos, s.first_pos + s.rows - 1);
        if (slot / 32 < blocks.sink_blocks || (slot / 32 >= blocks.main && slot / 32 < blocks.end)) {
            f32x4 x[kHeads][N], sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int which = 0; which < kHeads; ++which)
#pragma unroll
                for (int m = 0; m < N; ++m)
                    x[which][m] = *(const f32x4 *)(q.scores + (((int64_t)blockIdx.z * kHeads + which) * q.scores_rows + min(m, m_all - 1)) * stride + slot);
#pragma unroll
            for (int which = 0; which < kHeads; ++which)
#pragma unroll
                for (int m = 0; m < N; ++m) {
                    const int mm = min(m, m_all - 1);
                    const float2 st = *(const float2 *)(q.stat + ((int64_t)(s.first_row + mm / q.group) * q.q_heads + (head + which) * q.group + mm % q.group) * 2);
                    const float inv = m < m_all ? st.y : 0.f, most = most_exponent(st.x);
#pragma unroll
                    for (int j = 0; j < 4; ++j)  // (the larger of NaN and 0 is 0: rows that came out NaN add nothing)
                        sum[j] += fmaxf(exp2_fast(fminf(__builtin_fmaf(x[which][m][j], q.factor, -st.x), most)) * inv, 0.f);
                }
#pragma unroll
            for (int which = 0; which < kHeads; ++which)
#pragma unroll
                for (int j = 0; j < 4; ++j) total[which][j] += slot + j < s.n ? sum[j] : 0.f;
        }
    }
#pragma unroll
    for (int which = 0; which < kHeads; ++which) *(f32x4 *)(received + dense + which * stride + slot) = total[which];
}

// Sixteens of tokens of a workgroup that shares out rows for the weights: as many as leave room for two waves' registers.
constexpr int split_tiles(int dim) { return dim == 256 ? 2 : 4; }

// The same with the scores once more, from the same products as in the attention itself, so that with the row's reference and
// sum each probability is the one that was used, before it was rounded.  kSplitRows: a workgroup has 16 kTiles tokens and each wave a quarter of the
// rows that can see one; otherwise a wave has 16 kTiles tokens and all rows.  The next 16 rows are on their way while 16 are worked on,
// their places found by adding, not dividing.  The shares are added in one order.  Rows that came out NaN add nothing.  16 exp2
// and some 90 other vector instructions for 16 rows x 64 tokens: up to 701 rows of 3 x 4 heads x 64 over 5003, 40 us (with 32
// tokens 52), in which a compute unit works 58 % of the time and issues vector instructions in 81 % of the cycles that it works.
//
// Whether rows have a window is asked once for all scores that are compared with positions: two comparisons less for each (624 rows x 8 x 64
// over 6209 that stand in no order, pairs: 114 -> 72 us).
//
// kParts: a pair's two maps, and parts of their rows, go to workgroups of their own (blockIdx.y: the part), each of which leaves its sums for
// kv_pair_weights_kernel (see plan_pair_weights).
template <int D, int DT, bool kSplitRows, int kTiles, int kHeads, bool kParts>
__global__ __launch_bounds__(256, D == 256 && DT == PSC_F32 ? 1 : 2) void kv_weights_kernel(KvView c, KvQueries q, const float *given, float *received)
{
    const int lane = lane_id(), i = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int b = (int)blockIdx.z / (c.heads / kHeads), head0 = (int)blockIdx.z % (c.heads / kHeads) * kHeads;
    const RowSet s = rows_of(c, q, b);
    const int64_t stride = (int64_t)c.width << c.page_shift, dense = (int64_t)blockIdx.z * kHeads * stride;
    const int64_t of_pair = kParts ? ((int64_t)b * c.heads + (head0 & ~1)) * stride : dense;  // whose positions count
    const int64_t block = kSplitRows ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * 4 + wave;
    if (block * 16 * kTiles >= stride) return;  // (with kSplitRows the whole workgroup)
    const int slot = (int)(block * 16 * kTiles), m_all = s.rows * q.group;

    float total[kTiles][4] = {};
#pragma unroll 1
    for (int head = head0; head < head0 + kHeads; ++head) {
        if (!(slot < s.n && m_all > 0)) break;
        int places[kTiles], pos[kTiles][4];
        bool there = true;
        int lowest = 0x7fffffff, highest = -0x7fffffff - 1;  // of the lane's tokens' positions
        u32x4 a[kTiles][D / 32];
#pragma unroll
        for (int h = 0; h < kTiles; ++h) {
            uint32_t k[D / 32], ks;
            places[h] = sixteen_of(c, b, head, s.n, slot + 16 * h);
            there = there && places[h] >= 0 && slot + 16 * h + 16 <= s.n;
            load_keys<D>(c, places[h], i, g, k, ks);
            expand_keys<D, DT>(k, ks, a[h]);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int at = slot + 16 * h + 4 * g + r;
                pos[h][r] = q.positions && at < s.n ? q.positions[of_pair + at] : at;
                lowest = min(lowest, pos[h][r]);
                highest = max(highest, pos[h][r]);
            }
        }
        int64_t m_begin = 0, m_end = m_all;
        if (!q.positions) {
            if (q.causal) m_begin = max((int64_t)0, (int64_t)slot - s.first_pos) * q.group / 16 * 16;
            if (q.window > 0 && slot >= q.sinks)
                m_end = min(m_end, max((int64_t)0, (int64_t)slot + 16 * kTiles - 1 + q.window - s.first_pos) * q.group);
        }
        if constexpr (kParts) {
            const int64_t steps = max((int64_t)0, (m_end - m_begin + 63) / 64), from = m_begin + steps * blockIdx.y / gridDim.y * 64;
            m_end = min(m_end, m_begin + steps * (blockIdx.y + 1) / gridDim.y * 64);
            m_begin = from;
        }
        const int step = kSplitRows ? 64 : 16, more_rows = step / q.group, more_heads = step % q.group;
        int64_t m0 = m_begin + (kSplitRows ? wave * 16 : 0);
        if (m0 < m_end) {
            // the lane's row: place of its sequence, query head of its group
            int place = (int)((m0 + i) / q.group), in_group = (int)((m0 + i) % q.group);
            Rows<D, DT> rows;
            float2 st;
            auto load = [&](int m, int at, int h, Rows<D, DT> &r, float2 &stat) {
                if (m >= m_all) {
                    at = s.rows - 1;
                    h = q.group - 1;
                }
                load_rows<D, DT>(q, s.first_row + at, head * q.group + h, g, r);
                stat = *(const float2 *)(q.stat + ((int64_t)(s.first_row + at) * q.q_heads + head * q.group + h) * 2);
            };
            load((int)m0 + i, place, in_group, rows, st);
            for (; m0 < m_end; m0 += step) {
                const int m = (int)m0 + i, at = place;
                place += more_rows;
                in_group += more_heads;
                if (in_group >= q.group) {
                    in_group -= q.group;
                    ++place;
                }
                Rows<D, DT> next;
                float2 next_st;
                load((int)min(m0 + step, (int64_t)m_all) + i, place, in_group, next, next_st);
                const float inv = m < m_all ? st.y : 0.f;
                f32x4 x[kTiles];
#pragma unroll
                for (int h = 0; h < kTiles; ++h) x[h] = scores_of<D, DT>(a[h], rows);
                const int pos_q = s.first_pos + at;
                const bool coarse = is_coarse(st.x), mine = there && !coarse && (!q.causal || pos_q >= highest) && (q.window <= 0 || (int64_t)pos_q - lowest < q.window || highest < q.sinks);
                if (!__all(mine)) {
                    const RowMask mask = row_mask(q, pos_q);
                    if (q.window <= 0) {
#pragma unroll
                        for (int h = 0; h < kTiles; ++h)
#pragma unroll
                            for (int r = 0; r < 4; ++r)
                                if (!(places[h] >= 0 && slot + 16 * h + 4 * g + r < s.n && pos[h][r] <= mask.pos)) x[h][r] = kNegInf;
                    } else {
#pragma unroll
                        for (int h = 0; h < kTiles; ++h)
#pragma unroll
                            for (int r = 0; r < 4; ++r)
                                if (!(places[h] >= 0 && slot + 16 * h + 4 * g + r < s.n && sees(q, mask, pos[h][r]))) x[h][r] = kNegInf;
                    }
                    if (__any(coarse)) {  // such rows' scores become their exponents over the factor
                        const float inverse = 1.f / q.factor;
#pragma unroll
                        for (int h = 0; h < kTiles; ++h)
#pragma unroll
                            for (int r = 0; r < 4; ++r) x[h][r] = coarse ? fminf(__builtin_fmaf(x[h][r], q.factor, -st.x), kLift) * inverse : x[h][r];
                        st.x = coarse ? 0.f : st.x;
                    }
                }
#pragma unroll
                for (int h = 0; h < kTiles; ++h)
#pragma unroll
                    for (int r = 0; r < 4; ++r) total[h][r] += fmaxf(exp2_fast(__builtin_fmaf(x[h][r], q.factor, -st.x)) * inv, 0.f);
                rows = next;
                st = next_st;
            }
        }
    }
#pragma unroll
    for (int h = 0; h < kTiles; ++h)
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int d = 1; d < 16; d *= 2) total[h][r] += __shfl_xor(total[h][r], d);
    // lane (i, g) of the first 4 kTiles in i: token 4 g + i % 4 of the (i / 4)-th sixteen
    float mine = 0.f;
#pragma unroll
    for (int j = 0; j < 4 * kTiles; ++j) mine = i == j ? total[j >> 2][j & 3] : mine;
    const int in_block = (i & ~3) * 4 + 4 * g + (i & 3);
    const bool one = i < 4 * kTiles;
    if constexpr (kSplitRows) {
        __shared__ float parts[4][16 * kTiles];
        if (one) parts[wave][in_block] = mine;
        __syncthreads();
        if (wave > 0) return;
        if (one) mine = parts[0][in_block] + parts[1][in_block] + parts[2][in_block] + parts[3][in_block];
    }
    if (kParts) {
        if (one && slot + in_block < stride) received[(int64_t)blockIdx.y * gridDim.z * stride + dense + slot + in_block] = mine;
    } else if (one && slot + in_block < stride) {
#pragma unroll
        for (int which = 0; which < kHeads; ++which) {
            const int64_t at = dense + which * stride + slot + in_block;
            received[at] = (given ? given[at] : 0.f) + mine;
        }
    }
}

// Adds up the parts of a pair's two maps, in order: a thread to four slots.
__global__ __launch_bounds__(256) void kv_pair_weights_kernel(KvView c, const float *parts, int splits, const float *given, float *received)
{
    const int64_t stride = (int64_t)c.width << c.page_shift, slot = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (slot >= stride) return;
    const int64_t dense = (int64_t)blockIdx.z * 2 * stride + slot, further = (int64_t)c.batch * c.heads * stride;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    for (int p = 0; p < splits; ++p) sum += *(const f32x4 *)(parts + p * further + dense) + *(const f32x4 *)(parts + p * further + dense + stride);
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        f32x4 x = sum;
        if (given) x += *(const f32x4 *)(given + dense + which * stride);
        *(f32x4 *)(received + dense + which * stride) = x;
    }
}

template <int DT, int D, int kHeads>
int run_weights(const KvView &c, const KvQueries &q, const KvPlan &p, const float *given, float *received, hipStream_t s)
{
    const dim3 grid((uint32_t)p.weights_groups, 1, (uint32_t)(c.batch * c.heads / kHeads));
    if (p.scores_rows > 0) {
        if (p.scores_rows == 1) kv_weights_of_scores_kernel<1, kHeads><<<grid, 256, 0, s>>>(c, q, given, received);
        else if (p.scores_rows <= 4) kv_weights_of_scores_kernel<4, kHeads><<<grid, 256, 0, s>>>(c, q, given, received);
        else kv_weights_of_scores_kernel<kScoreRows, kHeads><<<grid, 256, 0, s>>>(c, q, given, received);
    } else if (kHeads == 2 && p.weight_parts > 0) {
        if constexpr (kHeads == 2) {
            const int64_t slots = (int64_t)c.width << c.page_shift;
            kv_weights_kernel<D, DT, true, split_tiles(D), 1, true>
                <<<dim3((uint32_t)p.weights_groups, (uint32_t)p.weight_parts, (uint32_t)(c.batch * c.heads)), 256, 0, s>>>(c, q, nullptr, q.weight_parts);
            PSC_HIP_TRY(hipGetLastError());
            kv_pair_weights_kernel<<<dim3((uint32_t)((slots + 1023) / 1024), 1, (uint32_t)(c.batch * c.heads / 2)), 256, 0, s>>>(c, q.weight_parts, p.weight_parts, given,
                                                                                                                           received);
        }
    } else if (p.split_rows) {
        kv_weights_kernel<D, DT, true, split_tiles(D), kHeads, false><<<grid, 256, 0, s>>>(c, q, given, received);
    } else {
        kv_weights_kernel<D, DT, false, 2, kHeads, false><<<grid, 256, 0, s>>>(c, q, given, received);
    }
    PSC_HIP_TRY(hipGetLastError());
    return PSC_OK;
}

// What the weights of calls with at most m rows (times query heads) of a kv head need.
inline void plan_weights(const KvView &c, int64_t m, int64_t rows, KvPlan *p)
{
    const int64_t slots = (int64_t)c.width << c.page_shift, scores_bytes = (int64_t)c.batch * c.heads * m * slots * 4;
    const bool keep_scores = rows > 0 && m <= kScoreRows && scores_bytes <= kMostScoreBytes;
    p->split_rows = m > 64;
    const int64_t tokens = keep_scores ? 1024 : p->split_rows ? 16 * split_tiles(c.dim) : 128;
    p->weights_groups = (slots + tokens - 1) / tokens;
    p->stat_bytes = (size_t)(rows * 8 + 255) / 256 * 256;
    if (keep_scores) {
        p->scores_rows = (int)m;
        p->scores_bytes = (size_t)(scores_bytes + 255) / 256 * 256;
    }
}

// The same where two kv heads are a pair.  Where workgroups with all rows of both maps would be few, the maps go to workgroups of their
// own and the rows are cut into parts of at least 256, whose sums kv_pair_weights_kernel adds in order (4 bytes to a slot, head and part, at most
// some 1 MB; it takes 4 to 5 us, where the cut saved 6 and more in all that was measured).  Not cut and cut, both kernels: 3 x 359 rows of 6 x 8 x 128 over
// 395 with a window of 43, 154 and 26 us; 2048 of 8 x 4 x 128 over 2048, 173 and 86; 624 of 4 x 8 x 64 over 6209, 93 and 55; 20 of 4 x 4 x 128
// over 9000, 14.7 and 13.  Up to 1024, 2048 and 4096 workgroups: the second, 92, 86, 90.
constexpr int64_t kWeightGroups = 2048;
inline void plan_pair_weights(const KvView &c, int64_t m, int64_t rows, KvPlan *p)
{
    plan_weights(c, m, rows, p);
    const int64_t groups = p->weights_groups * c.batch * c.heads;
    if (p->scores_rows > 0 || !p->split_rows || rows == 0 || groups >= kWeightGroups) return;
    p->weight_parts = (int)std::min((kWeightGroups + groups - 1) / groups, (m + 255) / 256);
    p->weight_parts_bytes = (size_t)(p->weight_parts * (int64_t)c.batch * c.heads * ((int64_t)c.width << c.page_shift) * 4 + 255) / 256 * 256;
}

}  // namespace
}  // namespace psc
