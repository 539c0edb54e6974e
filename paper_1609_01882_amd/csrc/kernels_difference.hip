// Differential attention over the attention memory in 4 bits (the format: kv_device.h).
//
// kv heads 2j and 2j + 1 are a pair: each has keys of its own, their values lie side by side (2 D wide), and an output head is
//   o = softmax(s q1 K1) V - lam softmax(s q2 K2) V,   then o * rsqrt(mean o^2 + eps) * norm * factor.
// A wave has both maps of its rows, so that the memory is read once, and values are expanded once for both.
//
// What it is bound by.  A few rows: reading the memory, 4.8 TB/s (8 sequences of 40 to 100 thousand tokens x 8 heads x 128, 618 MB in 128 us;
// 146 with the codes through registers and one wave to a SIMD).  Many rows: vector instructions and the way from one product's
// operands to the next product: 2048 rows of 32 query heads over 16384 tokens 925 to 1050 us by card, 740 to 840 TFLOP/s (through registers
// 1768; every wave with expansions of its own 1178).  float32 rows, whose scores take three products and whose values two, have one wave to a SIMD
// and expand for themselves: the same rows 2374 us.
//
// Bits.  Scores, sums and the difference are 32 bits.  The probabilities of 16-bit rows go into the second product as float16 (11 bits: one product,
// where two terms would take two; float32 rows have two, 22 bits).  That error is a share of each map, not of what the maps leave of
// each other: where they cancel to 2 % of themselves, outputs are 0.7 % off, and the head's norm makes it no smaller.
//
// Registers.  Two waves to a SIMD have 256 each, and some kernels need more: with 64 coordinates and 32 rows to a wave 132 to 240 bytes of a lane lie in
// scratch, with 128 coordinates 36 to 52 (none in the rows kernel over a memory in order).
#include <algorithm>
#include <type_traits>

#include "kv_weights.h"

namespace psc {
namespace {

// Codes, scales and positions of a block of 32 tokens on their way through LDS: a wave has kStages places of its own, into which loads write
// past the registers, so that the blocks after the one that is worked on are under way whatever the registers hold.  No other wave
// reads them: no barrier, the wave counts its loads (the first to return are the first asked for).  Each load moves 16 bytes (scales, positions: 4) of every lane to consecutive places; which
// bytes a lane asks for is chosen so that what it reads back lies without conflicts over the banks:
//   keys      in the order in which the lanes read them (coordinates g D/4 ... of token i, as for kv_device.h's load_keys)
//   values    a row of D / 2 bytes to a token, the four tokens of g turned by g (D = 64: g / 2) places
constexpr int kStages = 2;
template <int D, bool kPos>
struct Stage {
    static constexpr int kCodes = 2048 * (D / 64), kScales = 128 * (D / 64);
    static constexpr int kKeys = 0, kValues = kCodes, kKeyScales = 2 * kCodes, kValueScales = kKeyScales + kScales, kPositions = kValueScales + kScales;
    static constexpr int kBytes = kPositions + (kPos ? 256 : 0), kLoads = (D == 64 ? 5 : 10) + (kPos ? 1 : 0);
};

__device__ __forceinline__ void load_to_lds(const void *from, uint32_t to)  // 16 bytes of every lane
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(to), "v"(from) : "memory", "m0");
}
__device__ __forceinline__ void load_word_to_lds(const void *from, uint32_t to)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(to), "v"(from) : "memory", "m0");
}
template <int N>
__device__ __forceinline__ void wait_for_loads()  // but for the last N
{
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ void wait_for_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// Scores of 32 tokens x 16 rows: as scores_of, with the two sums in turn, since a product waits for the one whose sum it goes on.
template <int D, int DT>
__device__ __forceinline__ void scores_of_two(const u32x4 (&a)[2][D / 32], const Rows<D, DT> &rows, f32x4 (&s)[2])
{
    s[0] = s[1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int term = Rows<D, DT>::kTerms - 1; term >= 0; --term)  // the smallest first
#pragma unroll
        for (int j = 0; j < D / 32; ++j)
#pragma unroll
            for (int h = 0; h < 2; ++h) s[h] = mfma_scores<DT>(a[h][j], rows.x[term][j], s[h]);
}

// What a lane reads of a stage.
template <int D, bool kPos>
struct StageReader {
    typedef Stage<D, kPos> S;
    PSC_LDS const uint8_t *keys, *key_scales, *values, *value_scales, *positions;  // of the lane, in stage 0
    int g;
    __device__ StageReader(PSC_LDS const uint8_t *base, int i, int lane_g) : g(lane_g)
    {
        keys = base + S::kKeys + (D == 128 ? (g * 16 + i) * 16 : ((g >> 1) * 16 + i) * 16 + (g & 1) * 8);
        key_scales = base + S::kKeyScales + (D == 128 ? i * 4 + g : i * 2 + (g >> 1));
        values = base + S::kValues + 4 * g * (D / 2) + i * (D / 32);
        value_scales = base + S::kValueScales + g * (D / 8);
        positions = base + S::kPositions + 16 * g;
    }
    __device__ __forceinline__ void read_keys(int stage, int w, int h, uint32_t (&k)[D / 32], uint32_t &ks) const
    {
        PSC_LDS const uint8_t *p = keys + stage * S::kBytes;
        if constexpr (D == 128) {
            const u32x4 t = *(PSC_LDS const u32x4 *)(p + (w * 2 + h) * 1024);
#pragma unroll
            for (int j = 0; j < 4; ++j) k[j] = t[j];
            ks = (key_scales + stage * S::kBytes)[(w * 2 + h) * 64];
        } else {
            const u32x2 t = *(PSC_LDS const u32x2 *)(p + w * 1024 + h * 512);
            k[0] = t.x;
            k[1] = t.y;
            ks = (key_scales + stage * S::kBytes)[(w * 2 + h) * 32];
        }
    }
    __device__ __forceinline__ void read_values(int stage, int w, uint32_t (&v)[8], uint32_t (&vs)[2][4]) const
    {
        PSC_LDS const uint8_t *p = values + stage * S::kBytes, *s = value_scales + stage * S::kBytes;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                PSC_LDS const uint8_t *token = p + (D == 128 ? (w * 2 + h) * 1024 : w * 1024 + h * 512) + ((r + (D == 128 ? g : g >> 1)) & 3) * (D / 2);
                if constexpr (D == 128) v[4 * h + r] = *(PSC_LDS const uint32_t *)token;
                else v[4 * h + r] = *(PSC_LDS const uint16_t *)token;
            }
            if constexpr (D == 128) {
                const u32x4 t = *(PSC_LDS const u32x4 *)(s + (w * 2 + h) * 64);
#pragma unroll
                for (int r = 0; r < 4; ++r) vs[h][r] = t[r];
            } else {
                const u32x2 t = *(PSC_LDS const u32x2 *)(s + (w * 2 + h) * 32);
                vs[h][0] = t.x;
                vs[h][1] = t.y;
            }
        }
    }
    __device__ __forceinline__ void read_positions(int stage, int (&pos)[8]) const
    {
        if constexpr (kPos) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const u32x4 t = *(PSC_LDS const u32x4 *)(positions + stage * S::kBytes + h * 64);
#pragma unroll
                for (int r = 0; r < 4; ++r) pos[4 * h + r] = (int)t[r];
            }
        }
    }
};

// Whether all rows of a wave see all 32 tokens of a block that stands in no order: mostly so, for what an eviction kept lies mostly
// behind all rows; the comparisons and selections for every score and row are then passed over.
template <int RT>
__device__ __forceinline__ bool all_seen(const KvQueries &q, const RowMask (&mask)[RT], const int (&pos)[8], int slot, int lim0, int lim1)
{
    int lo = pos[0], hi = pos[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) {
        lo = min(lo, pos[e]);
        hi = max(hi, pos[e]);
    }
    bool all = slot + 16 <= lim0 && slot + 32 <= lim1;
#pragma unroll
    for (int t = 0; t < RT; ++t) all = all && hi <= mask[t].pos && (q.window <= 0 || lo > mask[t].after || hi < q.sinks);
    return __all(all);
}

// One wave attends with 16 RT rows, in both maps, over every fourth of the workgroup's blocks.  As in kv_attention_kernel: scores K Q^T leave
// 8 scores of one row in a lane, which are the operand of V^T P^T as they are; maximum, sum and rescaling are the lane's own.
// Tile t of map w is number w RT + t.  Accumulator (h D / 16 + j) of a tile has coordinate (4 g + r) D / 16 + j of value half h.
template <int D, int DT, int RT, bool kPos>
struct Difference {
    f32x4 acc[2 * RT][D / 8];
    float top[2 * RT], sum[2 * RT];  // of the scaled scores in units of log 2, the maximum less kLift; the sum is the lane's own share
    Rows<D, DT> rows[2 * RT];

    // kFar: rows whose scores are coarse may be among them.  `refill` is called when the stage has been read.
    template <bool kFar, class Refill>
    __device__ __forceinline__ void block(const KvQueries &q, const StageReader<D, kPos> &from, int stage, const RowMask (&mask)[RT], int slot, int lim0, int lim1,
                                          int n, bool whole, float factor, int i, int g, float *scores, int64_t scores_stride, const Refill &refill)
    {
        f32x4 s[2 * RT][2];
#pragma unroll
        for (int w = 0; w < 2; ++w)
        {
            u32x4 a[2][D / 32];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint32_t k[D / 32], ks;
                from.read_keys(stage, w, h, k, ks);
                expand_keys<D, DT>(k, ks, a[h]);
            }
#pragma unroll
            for (int t = 0; t < RT; ++t) scores_of_two<D, DT>(a, rows[w * RT + t], s[w * RT + t]);
        }
        int positions[8];
        if (kPos) from.read_positions(stage, positions);
        if (!(whole || (kPos && all_seen<RT>(q, mask, positions, slot, lim0, lim1)))) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int at = slot + 16 * h + 4 * g + r;
                    const bool there = at < (h ? lim1 : lim0);
                    const int pos = kPos ? positions[4 * h + r] : at;
#pragma unroll
                    for (int t = 0; t < RT; ++t)
                        if (!(there && sees(q, mask[t], pos))) s[t][h][r] = s[RT + t][h][r] = kNegInf;
                }
        }
        if constexpr (RT == 1) {
            if (scores) {
#pragma unroll
                for (int w = 0; w < 2; ++w)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        if (slot + 16 * h < n) *(f32x4 *)(scores + w * scores_stride + slot + 16 * h + 4 * g) = s[w][h];
            }
        }
        uint32_t p[2 * RT][2][4];  // float16 pairs (the second array: what the first leaves of float32 rows' probabilities)
#pragma unroll
        for (int t = 0; t < 2 * RT; ++t) {
            float m = kNegInf;  // (NaN where a score is: the row is lost then, whatever the maximum)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int r = 0; r < 4; ++r) m = __builtin_elementwise_maximum(m, s[t][h][r]);
            m = __builtin_fmaf(column_max(m), factor, -kLift);
            if (__any(m > top[t])) {
                const float now = fmaxf(top[t], kFar ? reference_below(m) : m);
                const float shrink = now == kNegInf ? 1.f : exp2_fast(top[t] - now);
                top[t] = now;
                sum[t] *= shrink;
#pragma unroll
                for (int j = 0; j < D / 8; ++j) acc[t][j] *= shrink;
            }
            const float base = top[t] == kNegInf ? 0.f : top[t];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int r = 0; r < 4; r += 2) {
                    float e0 = __builtin_fmaf(s[t][h][r], factor, -base), e1 = __builtin_fmaf(s[t][h][r + 1], factor, -base);
                    if constexpr (kFar) {
                        const float most = most_exponent(base);
                        e0 = __builtin_elementwise_minimum(e0, most);  // (NaN stays)
                        e1 = __builtin_elementwise_minimum(e1, most);
                    }
                    e0 = exp2_fast(e0);
                    e1 = exp2_fast(e1);
                    sum[t] += e0 + e1;
                    const h16x2 hi = {(_Float16)e0, (_Float16)e1};
                    p[t][0][h * 2 + r / 2] = __builtin_bit_cast(uint32_t, hi);
                    if constexpr (DT == PSC_F32) {
                        const h16x2 lo = {(_Float16)(e0 - (float)hi.x), (_Float16)(e1 - (float)hi.y)};
                        p[t][1][h * 2 + r / 2] = __builtin_bit_cast(uint32_t, lo);
                    }
                }
        }
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            uint32_t v[8], vs[2][4];
            from.read_values(stage, half, v, vs);
            if (half == 1) refill();
            // tokens 0..7 of the lane: 4 g + r, then 16 + 4 g + r
            uint32_t held[8];
#pragma unroll
            for (int t = 0; t < 8; ++t) held[t] = value_scale<D>(vs[t >> 2], t & 3, i);
            if (!whole) {  // what lies past the end may be NaN: with the scale 2^-127 it is zeros in float16
#pragma unroll
                for (int t = 0; t < 8; ++t) held[t] = slot + (t < 4 ? 4 * g + t : 12 + 4 * g + t) < (t < 4 ? lim0 : lim1) ? held[t] : 0u;
            }
            constexpr int kBytes = D / 32;  // code bytes of a token in this lane
#pragma unroll
            for (int y = 0; y < kBytes; ++y) {
                uint32_t w[8];
#pragma unroll
                for (int t = 0; t < 8; ++t) {
                    const float sc = __uint_as_float(held[t]);
                    const uint32_t x = v[t];
                    w[t] = y == 0 ? two_h16<0>(x, sc) : y == 1 ? two_h16<1>(x, sc) : y == 2 ? two_h16<2>(x, sc) : two_h16<3>(x, sc);
                }
                u32x4 lo, hi;
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    lo[t] = __builtin_amdgcn_perm(w[2 * t + 1], w[2 * t], 0x05040100u);
                    hi[t] = __builtin_amdgcn_perm(w[2 * t + 1], w[2 * t], 0x07060302u);
                }
#pragma unroll
                for (int t = 0; t < 2 * RT; ++t) {
#pragma unroll
                    for (int term = DT == PSC_F32 ? 1 : 0; term >= 0; --term) {
                        const h16x8 pr = __builtin_bit_cast(h16x8, (u32x4){p[t][term][0], p[t][term][1], p[t][term][2], p[t][term][3]});
                        f32x4 &a = acc[t][half * (D / 16) + 2 * y], &b = acc[t][half * (D / 16) + 2 * y + 1];
                        a = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h16x8, lo), pr, a, 0, 0, 0);
                        b = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h16x8, hi), pr, b, 0, 0, 0);
                    }
                }
            }
        }
    }
};

// Waves of a SIMD that the registers are to leave room for (D = 64 with 16 rows: three waves spill, 1 x 700 tokens 15.5 us instead of 12.7).
constexpr int difference_waves(int dim, int dtype, int row_tiles)
{
    if (dtype == PSC_F32) return dim == 64 ? 2 : 1;
    return 2;
}

// From a row's sums over both maps, D / 16 coordinates of both value halves to each of 16 lanes that stand in a row: the output.  A row that sees
// nothing (both `inv` are 0) is 0 whatever lam, norm and eps are, here and at both other ends: 0 / 0 and 0 times infinity would be NaN.
template <int D, int DT>
__device__ __forceinline__ void finish_row(const KvQueries &q, const KvDifference &d, int row, int out_head, int run, const float (&x)[2][2][D / 16], const float (&inv)[2])
{
    const float lam = d.lam[(int64_t)row * d.lam_stride + out_head];
    const bool nothing = inv[0] == 0.f && inv[1] == 0.f;
    float o[2][D / 16], squares = 0.f;
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int j = 0; j < D / 16; ++j) {
            o[half][j] = x[0][half][j] * inv[0] - lam * (x[1][half][j] * inv[1]);
            squares += o[half][j] * o[half][j];
        }
    float scale = d.factor;
    if (d.norm) {
#pragma unroll
        for (int k = 1; k < 16; k *= 2) squares += __shfl_xor(squares, k);
        scale *= 1.f / sqrtf(squares * (1.f / (2 * D)) + d.eps);
    }
    typename Element<DT>::type *out = (typename Element<DT>::type *)q.out + ((int64_t)row * (q.q_heads / 2) + out_head) * (2 * D);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const int at = half * D + run * (D / 16);
#pragma unroll
        for (int j = 0; j < D / 16; ++j) o[half][j] = nothing ? 0.f : o[half][j] * (d.norm ? d.norm[at + j] * scale : scale);
        store_row<DT, D / 16>(out + at, o[half]);
    }
}

// The output of rows from .. to - 1, NaN: no sequence has them.
template <int D, int DT>
__device__ void difference_of_nobody(const KvQueries &q, int pair, int from, int to)
{
    for (int64_t x = (int64_t)max(from, 0) * q.group + (threadIdx.x >> 4); x < (int64_t)min(to, q.nrows) * q.group; x += blockDim.x >> 4) {
        const int64_t row = x / q.group;
        const int in_group = (int)(x % q.group), run = (int)threadIdx.x & 15;
        float nan[D / 16];
#pragma unroll
        for (int j = 0; j < D / 16; ++j) nan[j] = __builtin_nanf("");
        typename Element<DT>::type *out = (typename Element<DT>::type *)q.out + (row * (q.q_heads / 2) + pair * q.group + in_group) * (2 * D) + run * (D / 16);
        store_row<DT, D / 16>(out, nan);
        store_row<DT, D / 16>(out + D, nan);
        if (run < 2 && q.lse) q.lse[row * q.q_heads + (2 * pair + run) * q.group + in_group] = nan[0];
    }
}

template <int D, int RT>
struct JoinedPair {  // of a workgroup's four waves
    static constexpr int kStride = 2 * D + 4;
    float acc[4][16 * kStride];
    float tops[4][32 * RT], sums[4][32 * RT];
};
template <int D, int RT, bool kPos>
union PairLds {  // first the stages, then the join
    JoinedPair<D, RT> joined;
    uint8_t stages[4][kStages][Stage<D, kPos>::kBytes];
};

// Blocks begin .. end - 1 of the rows from m0 on of (b, pair): the workgroup's four waves take every fourth each and are joined in LDS.
// part < 0: these are all blocks, and the result is final.
template <int D, int DT, int RT, bool kPos>
__device__ __forceinline__ void attend_pair(const KvView &c, const KvQueries &q, const KvDifference &d, const RowSet &s, int b, int pair, int m0, const Blocks &blocks,
                                            int begin, int end, int64_t part, PairLds<D, RT, kPos> &lds)
{
    const int lane = lane_id(), i = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int m_all = s.rows * q.group, m_end = min(m0 + 16 * RT, m_all);
    const int lo_pos = s.first_pos + m0 / q.group, hi_pos = s.first_pos + (m_end - 1) / q.group;
    constexpr int step = 4;

    Difference<D, DT, RT, kPos> a;
    RowMask mask[RT];
    const auto start = [&] {
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            const int m = min(m0 + t * 16 + i, m_all - 1), place = m / q.group;  // (rows past the last: the last one again)
            mask[t] = row_mask(q, s.first_pos + place);
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                const int n = w * RT + t;
                load_rows<D, DT>(q, s.first_row + place, (2 * pair + w) * q.group + m - place * q.group, g, a.rows[n]);
                a.top[n] = kNegInf;
                a.sum[n] = 0.f;
#pragma unroll
                for (int j = 0; j < D / 8; ++j) a.acc[n][j] = f32x4{0.f, 0.f, 0.f, 0.f};
            }
        }
    };
    start();
    const int64_t slots = (int64_t)c.width << c.page_shift, dense = ((int64_t)b * c.heads + 2 * pair) * slots;
    const int next_head = 1 << (c.page_shift - 4);  // sixteens from a head's slots to the next head's

    // The places of 32 of the wave's blocks are held across the lanes; the codes of the blocks after the one that is worked on
    // are on their way, without a branch around their loads (past the last block: of a page that is there).
    const int own = begin + wave, mine = end > own ? (end - own + step - 1) / step : 0;
    auto pages_from = [&](int k) {
        return sixteen_of(c, b, 2 * pair, s.n, blocks.block(min(own + (k + (lane >> 1)) * step, end - 1)) * 32 + (lane & 1) * 16);
    };
    typedef Stage<D, kPos> S;
    PSC_LDS uint8_t *const base = (PSC_LDS uint8_t *)lds.stages[wave];
    const uint32_t base_at = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(uintptr_t)base);
    const StageReader<D, kPos> reader(base, i, g);
    // what the lane asks for: of keys, values and scales (see Stage)
    const int key_token = D == 128 ? i * 64 + g * 16 : i * 32 + (g & 1) * 16;
    const int row = D == 128 ? lane >> 2 : lane >> 1 & 15, value_token = (row & ~3) + ((row - (D == 128 ? row >> 2 : row >> 3)) & 3);
    const int value_at = value_token * (D / 2) + (D == 128 ? lane & 3 : lane & 1) * 16;
    const auto load = [&](int k, const int (&pg)[2], int stage) {
        const uint32_t to = base_at + stage * S::kBytes;
        const int p0 = max(pg[0], 0), p1 = max(pg[1], 0);
        if constexpr (D == 128) {
#pragma unroll
            for (int w = 0; w < 2; ++w)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int64_t at = (int64_t)((h ? p1 : p0) + w * next_head) * 1024;
                    load_to_lds(c.k_codes + at + key_token, to + S::kKeys + (w * 2 + h) * 1024);
                    load_to_lds(c.v_codes + at + value_at, to + S::kValues + (w * 2 + h) * 1024);
                }
            const int64_t at = (int64_t)((lane & 16 ? p1 : p0) + (lane >> 5) * next_head) * 64 + (lane & 15) * 4;
            load_word_to_lds(c.k_scales + at, to + S::kKeyScales);
            load_word_to_lds(c.v_scales + at, to + S::kValueScales);
        } else {
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                const int64_t at = (int64_t)((lane & 32 ? p1 : p0) + w * next_head) * 512;
                load_to_lds(c.k_codes + at + key_token, to + S::kKeys + w * 1024);
                load_to_lds(c.v_codes + at + value_at, to + S::kValues + w * 1024);
            }
            const int64_t at = (int64_t)((lane & 8 ? p1 : p0) + (lane >> 4 & 1) * next_head) * 32 + (lane & 7) * 4;
            load_word_to_lds((lane & 32 ? c.v_scales : c.k_scales) + at, to + S::kKeyScales);
        }
        if constexpr (kPos) {
            const int sl = blocks.block(min(own + k * step, end - 1)) * 32;
            load_word_to_lds(q.positions + dense + min(sl + (lane & 31), (int)slots - 1), to + S::kPositions);
        }
    };
    // where the scores of the lane's row are left for kv_weights_of_scores_kernel
    float *scores = nullptr;
    if constexpr (RT == 1)
        if (q.scores && i < m_all) scores = q.scores + (((int64_t)b * c.heads + 2 * pair) * q.scores_rows + i) * slots;
    const auto work = [&](auto far, int k, int stage, const int (&pg)[2], const auto &refill) {
        const int slot = blocks.block(own + k * step) * 32;
        const bool there = slot + 32 <= s.n && pg[0] >= 0 && pg[1] >= 0 && !kPos;
        const bool whole = there && (!q.causal || slot + 31 <= lo_pos) &&
                           (q.window <= 0 || (int64_t)hi_pos - slot < q.window || slot + 32 <= q.sinks);
        a.template block<far.value>(q, reader, stage, mask, slot, pg[0] >= 0 ? s.n : 0, pg[1] >= 0 ? s.n : 0, s.n, whole, q.factor, i, g, scores, q.scores_rows * slots,
                                    refill);
    };
    if (mine > 0) {
        int ids = pages_from(0), pages[kStages + 1][2], stage = 0;  // pages of the block that is worked on, and of those under way
#pragma unroll
        for (int k = 0; k < kStages; ++k) {
            pages[k][0] = __builtin_amdgcn_readlane(ids, 2 * k);
            pages[k][1] = __builtin_amdgcn_readlane(ids, 2 * k + 1);
            load(k, pages[k], k);
        }
        int ids_then = pages_from(32);
        for (int k = 0; k < mine; ++k) {
            const int ahead = (k & 31) + kStages, from = ahead < 32 ? ids : ids_then;
            pages[kStages][0] = __builtin_amdgcn_readlane(from, 2 * (ahead & 31));
            pages[kStages][1] = __builtin_amdgcn_readlane(from, 2 * (ahead & 31) + 1);
            wait_for_loads<(kStages - 1) * S::kLoads>();
            work(std::false_type(), k, stage, pages[0], [&] {
                wait_for_lds();
                load(k + kStages, pages[kStages], stage);
            });
            stage = stage + 1 < kStages ? stage + 1 : 0;
#pragma unroll
            for (int j = 0; j < kStages; ++j) {
                pages[j][0] = pages[j + 1][0];
                pages[j][1] = pages[j + 1][1];
            }
            if ((k & 31) == 31) {
                ids = ids_then;
                ids_then = pages_from(k + 33);
            }
        }
    }
    wait_for_loads<0>();  // (of blocks past the last too: their places are used again)
    // Decided at the end, and all done again, as in kv_attention_kernel.
    bool far = false;
#pragma unroll
    for (int t = 0; t < 2 * RT; ++t) far = far || is_coarse(a.top[t]);
    if (__any(far)) {
        asm volatile("" ::: "memory");  // (the rows are read again: kept, they would cost the pass above registers)
        start();
#pragma unroll 1
        for (int k = 0; k < mine; ++k) {
            const int ids = pages_from(k), pages[2] = {__builtin_amdgcn_readlane(ids, 0), __builtin_amdgcn_readlane(ids, 1)};
            wait_for_lds();
            load(k, pages, 0);
            wait_for_loads<0>();
            work(std::true_type(), k, 0, pages, [] {});
        }
    }
    JoinedPair<D, RT> &joined = lds.joined;
    __syncthreads();
#pragma unroll
    for (int t = 0; t < 2 * RT; ++t) a.sum[t] = column_sum(a.sum[t]);
    if (g == 0) {
#pragma unroll
        for (int t = 0; t < 2 * RT; ++t) {
            joined.tops[wave][t * 16 + i] = a.top[t];
            joined.sums[wave][t * 16 + i] = a.sum[t];
        }
    }
    __syncthreads();
    const int local = (int)threadIdx.x >> 4, run = (int)threadIdx.x & 15;
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        const int m = m0 + t * 16 + local;
        float x[2][2][D / 16], inv[2];
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            const int n = w * RT + t;
            float top = kNegInf;
#pragma unroll
            for (int k = 0; k < 4; ++k) top = fmaxf(top, joined.tops[k][n * 16 + i]);
            const float shrink = top == kNegInf ? 1.f : exp2_fast(a.top[n] - top);
            if (t > 0 || w > 0) __syncthreads();
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    float y[D / 16];
#pragma unroll
                    for (int j = 0; j < D / 16; ++j) y[j] = a.acc[n][half * (D / 16) + j][r] * shrink;
                    store_row<PSC_F32, D / 16>(&joined.acc[wave][i * joined.kStride + half * D + (g * 4 + r) * (D / 16)], y);
                }
            __syncthreads();
            float best = kNegInf, sum = 0.f;
#pragma unroll
            for (int k = 0; k < 4; ++k) best = fmaxf(best, joined.tops[k][n * 16 + local]);
#pragma unroll
            for (int k = 0; k < 4; ++k) sum += joined.sums[k][n * 16 + local] * (best == kNegInf ? 1.f : exp2_fast(joined.tops[k][n * 16 + local] - best));
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int j = 0; j < D / 16; ++j) {
                    x[w][half][j] = 0.f;
#pragma unroll
                    for (int k = 0; k < 4; ++k) x[w][half][j] += joined.acc[k][local * joined.kStride + half * D + run * (D / 16) + j];
                }
            inv[w] = sum == 0.f ? 0.f : 1.f / sum;
            if (m >= m_all) continue;
            if (part >= 0) {
                const int64_t at = (part * 2 + w) * (16 * RT) + t * 16 + local;
                if (run == 0) *(float2 *)(q.part_stat + at * 2) = make_float2(best, sum);
#pragma unroll
                for (int half = 0; half < 2; ++half) store_row<PSC_F32, D / 16>(q.part_acc + at * (2 * D) + half * D + run * (D / 16), x[w][half]);
            } else if (run == 0) {
                const int64_t row = (int64_t)(s.first_row + m / q.group) * q.q_heads + (2 * pair + w) * q.group + m % q.group;
                if (q.lse) q.lse[row] = sum == 0.f ? kNegInf : log_sum(best, sum);
                if (q.stat) *(float2 *)(q.stat + row * 2) = make_float2(best == kNegInf ? 0.f : best, inv[w]);
            }
        }
        if (part < 0 && m < m_all) finish_row<D, DT>(q, d, s.first_row + m / q.group, pair * q.group + m % q.group, run, x, inv);
    }
}

template <int D, int DT, int RT, bool kPos, bool kParts>
__global__ __launch_bounds__(256, difference_waves(D, DT, RT)) void kv_difference_kernel(KvView c, KvQueries q, KvDifference d)
{
    __shared__ __attribute__((aligned(16))) PairLds<D, RT, kPos> lds;
    const int pairs = c.heads / 2;
    if constexpr (!kParts) {
        // (the last rows first: they see the most)
        const int b = (int)blockIdx.z / pairs, pair = (int)blockIdx.z % pairs, m0 = ((int)gridDim.x - 1 - (int)blockIdx.x) * 16 * RT;
        const RowSet s = rows_of(c, q, b);
        if (q.offsets && m0 == 0) {
            if (b == 0) difference_of_nobody<D, DT>(q, pair, 0, s.first_row);
            difference_of_nobody<D, DT>(q, pair, s.first_row + s.rows, b + 1 < c.batch ? q.offsets[b + 1] : q.nrows);
        }
        if (m0 >= s.rows * q.group || s.rows * q.group > d.most) return;
        const Blocks blocks = blocks_of(q, s.n, s.first_pos + m0 / q.group, s.first_pos + (min(m0 + 16 * RT, s.rows * q.group) - 1) / q.group);
        attend_pair<D, DT, RT, kPos>(c, q, d, s, b, pair, m0, blocks, 0, blocks.count(), -1, lds);
    } else {
        Parts all(c, q);
        if (blockIdx.x >= all.total) return;
        uint32_t first;
        const int b = all.find(c, q, blockIdx.x, &first);
        const RowSet s = rows_of(c, q, b);
        const uint32_t each = Parts::blocks_of_unit(q, s), parts = all.parts_of_unit(each);
        const uint32_t unit = (blockIdx.x - first) / parts, part = blockIdx.x - first - unit * parts;
        const int pair = (int)unit % pairs, m0 = (int)unit / pairs * 16 * RT;
        const Blocks blocks = blocks_of(q, s.n, s.first_pos + m0 / q.group, s.first_pos + (min(m0 + 16 * RT, s.rows * q.group) - 1) / q.group);
        const int count = blocks.count(), from = (int)((uint64_t)part * each / parts), to = (int)((uint64_t)(part + 1) * each / parts);
        attend_pair<D, DT, RT, kPos>(c, q, d, s, b, pair, m0, blocks, min(count, from), min(count, to), parts == 1 ? -1 : (int64_t)blockIdx.x, lds);
    }
}

// ------------------------------------------------------------------------------------------- many rows
// Where there are rows for it, a wave has 16 RT rows of its own and a workgroup's four waves take every block together: each expands a
// quarter of the block's keys and values -- sixteen tokens of a head -- into LDS as the operands of the products, and all four read them.  Two
// buffers in turn: one barrier to a block.  A wave's expansions (192 vector instructions to a block of 128 coordinates, of 390
// altogether) become 48.  Vector instructions are then issued in 48 % of the cycles, the matrix cores busy in 36 %, LDS in 48 %: none of them, but
// the way through them bounds it, with the two waves to a SIMD that the registers leave room for.  32 rows of 128 coordinates
// to a wave do not fit (6296 us).
template <int D>
struct Operands {
    u32x4 keys[2][2][D / 32][64];      // [map][sixteen][32 coordinates]: a lane's operand of a product
    u32x2 values[2][D / 16][2][64];    // [half][16 coordinates][sixteen]: half of one
};
template <int D>
struct Quarter {  // of a block, as it lies in memory
    uint32_t k[D / 32], ks, v[4][1], vs[4];
};

template <int D, int DT, int RT, bool kPos>
struct RowsDifference {
    f32x4 acc[2 * RT][D / 8];  // as in Difference
    float top[2 * RT], sum[2 * RT];
    Rows<D, DT> rows[2 * RT];

    // `keys` and `values` expand what the wave has of the next block, where the matrix units are at work on this one.
    template <bool kFar, class Keys, class Values>
    __device__ __forceinline__ void block(const KvQueries &q, const Operands<D> &from, const RowMask (&mask)[RT], const int (&pos)[8], int slot, int lim0, int lim1,
                                          bool whole, float factor, int lane, const Keys &keys, const Values &values)
    {
        const int g = lane >> 4;
        f32x4 s[2 * RT][2];
#pragma unroll
        for (int w = 0; w < 2; ++w)
        {
            u32x4 a[2][D / 32];
#pragma unroll
            for (int j = 0; j < D / 32; ++j)
#pragma unroll
                for (int h = 0; h < 2; ++h) a[h][j] = from.keys[w][h][j][lane];
#pragma unroll
            for (int t = 0; t < RT; ++t) scores_of_two<D, DT>(a, rows[w * RT + t], s[w * RT + t]);
        }
        keys();
        if (!(whole || (kPos && all_seen<RT>(q, mask, pos, slot, lim0, lim1)))) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int at = slot + 16 * h + 4 * g + r;
                    const bool there = at < (h ? lim1 : lim0);
                    const int p = kPos ? pos[4 * h + r] : at;
#pragma unroll
                    for (int t = 0; t < RT; ++t)
                        if (!(there && sees(q, mask[t], p))) s[t][h][r] = s[RT + t][h][r] = kNegInf;
                }
        }
        uint32_t p[2 * RT][4];  // float16 pairs
#pragma unroll
        for (int t = 0; t < 2 * RT; ++t) {
            float m = kNegInf;  // (NaN where a score is: the row is lost then, whatever the maximum)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int r = 0; r < 4; ++r) m = __builtin_elementwise_maximum(m, s[t][h][r]);
            m = __builtin_fmaf(column_max(m), factor, -kLift);
            if (__any(m > top[t])) {
                const float now = fmaxf(top[t], kFar ? reference_below(m) : m);
                const float shrink = now == kNegInf ? 1.f : exp2_fast(top[t] - now);
                top[t] = now;
                sum[t] *= shrink;
#pragma unroll
                for (int j = 0; j < D / 8; ++j) acc[t][j] *= shrink;
            }
            const float base = top[t] == kNegInf ? 0.f : top[t];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int r = 0; r < 4; r += 2) {
                    float e0 = __builtin_fmaf(s[t][h][r], factor, -base), e1 = __builtin_fmaf(s[t][h][r + 1], factor, -base);
                    if constexpr (kFar) {
                        const float most = most_exponent(base);
                        e0 = __builtin_elementwise_minimum(e0, most);  // (NaN stays)
                        e1 = __builtin_elementwise_minimum(e1, most);
                    }
                    e0 = exp2_fast(e0);
                    e1 = exp2_fast(e1);
                    sum[t] += e0 + e1;
                    p[t][h * 2 + r / 2] = __builtin_bit_cast(uint32_t, (h16x2){(_Float16)e0, (_Float16)e1});
                }
        }
        values();
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int j = 0; j < D / 16; ++j) {
                const u32x2 x = from.values[half][j][0][lane], y = from.values[half][j][1][lane];
                const h16x8 v = __builtin_bit_cast(h16x8, (u32x4){x.x, x.y, y.x, y.y});
#pragma unroll
                for (int t = 0; t < 2 * RT; ++t) {
                    const h16x8 pr = __builtin_bit_cast(h16x8, (u32x4){p[t][0], p[t][1], p[t][2], p[t][3]});
                    acc[t][half * (D / 16) + j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, pr, acc[t][half * (D / 16) + j], 0, 0, 0);
                }
            }
    }
};

// kParts: what a workgroup's rows see is cut into parts as in kv_difference_kernel, for kv_difference_join_kernel.
template <int D, int DT, int RT, bool kPos, bool kParts>
__global__ __launch_bounds__(256, 2) void kv_difference_rows_kernel(KvView c, KvQueries q, KvDifference d)
{
    __shared__ Operands<D> operands[2];
    const int pairs = c.heads / 2, lane = lane_id(), i = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    int b, pair, group0;
    uint32_t part = 0, parts = 1, each = 0;
    if constexpr (kParts) {
        Parts all(c, q);
        if (blockIdx.x >= all.total) return;
        uint32_t first;
        b = all.find(c, q, blockIdx.x, &first);
        each = Parts::blocks_of_unit(q, rows_of(c, q, b));
        parts = all.parts_of_unit(each);
        const uint32_t unit = (blockIdx.x - first) / parts;
        part = blockIdx.x - first - unit * parts;
        pair = (int)unit % pairs;
        group0 = (int)unit / pairs * 64 * RT;
    } else {
        // (the last rows first: they see the most)
        b = (int)blockIdx.z / pairs;
        pair = (int)blockIdx.z % pairs;
        group0 = ((int)gridDim.x - 1 - (int)blockIdx.x) * 64 * RT;
    }
    const RowSet s = rows_of(c, q, b);
    const int m_all = s.rows * q.group, group_end = min(group0 + 64 * RT, m_all);
    if constexpr (!kParts) {
        if (q.offsets && group0 == 0) {
            if (b == 0) difference_of_nobody<D, DT>(q, pair, 0, s.first_row);
            difference_of_nobody<D, DT>(q, pair, s.first_row + s.rows, b + 1 < c.batch ? q.offsets[b + 1] : q.nrows);
        }
        if (group0 >= m_all || m_all <= d.few) return;  // (few: left to kv_difference_kernel)
    }
    const int m0 = group0 + wave * 16 * RT, m_end = min(m0 + 16 * RT, m_all);
    const bool some = m0 < m_all;
    const int lo_pos = s.first_pos + min(m0, m_all - 1) / q.group, hi_pos = s.first_pos + (m_end - 1) / q.group;
    const Blocks blocks = blocks_of(q, s.n, s.first_pos + group0 / q.group, s.first_pos + (group_end - 1) / q.group);
    const int begin = kParts ? min(blocks.count(), (int)((uint64_t)part * each / parts)) : 0;
    const int count = (kParts ? min(blocks.count(), (int)((uint64_t)(part + 1) * each / parts)) : blocks.count()) - begin;
    const int64_t slots = (int64_t)c.width << c.page_shift, dense = ((int64_t)b * c.heads + 2 * pair) * slots;
    const int next_head = 1 << (c.page_shift - 4);  // sixteens from a head's slots to the next head's

    RowsDifference<D, DT, RT, kPos> a;
    RowMask mask[RT];
    const auto start = [&] {
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            const int m = min(m0 + t * 16 + i, m_all - 1), place = m / q.group;  // (rows past the last: the last one again)
            mask[t] = row_mask(q, s.first_pos + place);
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                const int n = w * RT + t;
                load_rows<D, DT>(q, s.first_row + place, (2 * pair + w) * q.group + m - place * q.group, g, a.rows[n]);
                a.top[n] = kNegInf;
                a.sum[n] = 0.f;
#pragma unroll
                for (int j = 0; j < D / 8; ++j) a.acc[n][j] = f32x4{0.f, 0.f, 0.f, 0.f};
            }
        }
    };
    // The places of 32 blocks are held across the lanes, a sixteen to each; a wave's quarter is sixteen `mine` of head `head`.
    const int head = wave >> 1, mine = wave & 1;
    const auto pages_from = [&](int k) { return sixteen_of(c, b, 2 * pair, s.n, blocks.block(begin + min(k + (lane >> 1), count - 1)) * 32 + (lane & 1) * 16); };
    const auto load = [&](int page, Quarter<D> &x) {
        const int at = max(page, 0) + head * next_head;
        load_keys<D>(c, at, i, g, x.k, x.ks);
        load_values<D>(c, at, i, g, x.v, x.vs);
    };
    const auto expand_k = [&](const Quarter<D> &x, Operands<D> &to) {
        u32x4 k[D / 32];
        expand_keys<D, DT>(x.k, x.ks, k);
#pragma unroll
        for (int j = 0; j < D / 32; ++j) to.keys[head][mine][j][lane] = k[j];
    };
    const auto expand_v = [&](const Quarter<D> &x, int slot, int page, Operands<D> &to) {
        uint32_t held[4];
        // what lies past the end may be NaN: with the scale 2^-127 it is zeros in float16
        const int lim = page < 0 ? 0 : s.n - slot - 16 * mine - 4 * g;
#pragma unroll
        for (int r = 0; r < 4; ++r) held[r] = r < lim ? value_scale<D>(x.vs, r, i) : 0u;
#pragma unroll
        for (int y = 0; y < D / 32; ++y) {
            uint32_t w[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float sc = __uint_as_float(held[r]);
                w[r] = y == 0 ? two_h16<0>(x.v[r][0], sc) : y == 1 ? two_h16<1>(x.v[r][0], sc) : y == 2 ? two_h16<2>(x.v[r][0], sc) : two_h16<3>(x.v[r][0], sc);
            }
            to.values[head][2 * y][mine][lane] = u32x2{__builtin_amdgcn_perm(w[1], w[0], 0x05040100u), __builtin_amdgcn_perm(w[3], w[2], 0x05040100u)};
            to.values[head][2 * y + 1][mine][lane] = u32x2{__builtin_amdgcn_perm(w[1], w[0], 0x07060302u), __builtin_amdgcn_perm(w[3], w[2], 0x07060302u)};
        }
    };
    // The block that is worked on lies in one buffer; the next one's codes are here and go into the other while the products run, and those of
    // the one after that are asked for then.  (Past the last block: the last one again.)
    const auto pass = [&](auto far) {
        start();
        if (count == 0) return;
        int ids = pages_from(0), ids_then = pages_from(32);
        const auto page_of_block = [&](int in, int h) { return __builtin_amdgcn_readlane(in < 32 ? ids : ids_then, 2 * (in & 31) + h); };
        const auto slot_of = [&](int k) { return blocks.block(begin + min(k, count - 1)) * 32; };
        Quarter<D> next;
        load(page_of_block(0, mine), next);
        expand_k(next, operands[0]);
        expand_v(next, slot_of(0), page_of_block(0, mine), operands[0]);
        load(page_of_block(1, mine), next);
        __syncthreads();
        for (int k = 0; k < count; ++k) {
            const int in = k & 31, page0 = page_of_block(in, 0), page1 = page_of_block(in, 1), page_next = page_of_block(in + 1, mine);
            const int page_then = page_of_block(in + 2, mine);
            const int slot = slot_of(k), slot_next = slot_of(k + 1);
            int pos[8];
            if constexpr (kPos) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int4 x = *(const int4 *)(q.positions + dense + min(slot + 16 * h, (int)slots - 16) + 4 * g);
                    pos[4 * h] = x.x;
                    pos[4 * h + 1] = x.y;
                    pos[4 * h + 2] = x.z;
                    pos[4 * h + 3] = x.w;
                }
            }
            const Operands<D> &buffer = operands[k & 1];
            Operands<D> &other = operands[(k & 1) ^ 1];
            const bool there = slot + 32 <= s.n && page0 >= 0 && page1 >= 0 && !kPos;
            const bool whole = there && (!q.causal || slot + 31 <= lo_pos) && (q.window <= 0 || (int64_t)hi_pos - slot < q.window || slot + 32 <= q.sinks);
            a.template block<far.value>(q, buffer, mask, pos, slot, page0 >= 0 ? s.n : 0, page1 >= 0 ? s.n : 0, whole, q.factor, lane,
                                        [&] { expand_k(next, other); },
                                        [&] {
                                            expand_v(next, slot_next, page_next, other);
                                            load(page_then, next);
                                        });
            __syncthreads();
            if (in == 31) {
                ids = ids_then;
                ids_then = pages_from(k + 33);
            }
        }
    };
    pass(std::false_type());
    // Decided at the end, and all done again, as in kv_attention_kernel.
    bool coarse = false;
#pragma unroll
    for (int t = 0; t < 2 * RT; ++t) coarse = coarse || is_coarse(a.top[t]);
    if (__syncthreads_or(coarse && some)) {
        asm volatile("" ::: "memory");  // (the rows are read again: kept, they would cost the pass above registers)
        pass(std::true_type());
    }
    if (!some) return;
    if (kParts && parts > 1) {
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                const int n = w * RT + t;
                const float sum = column_sum(a.sum[n]);
                if (m0 + t * 16 + i >= m_all) continue;
                const int64_t at = ((int64_t)blockIdx.x * 2 + w) * (64 * RT) + (wave * RT + t) * 16 + i;
                if (g == 0) *(float2 *)(q.part_stat + at * 2) = make_float2(a.top[n], sum);
#pragma unroll
                for (int half = 0; half < 2; ++half)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        float o[D / 16];
#pragma unroll
                        for (int j = 0; j < D / 16; ++j) o[j] = a.acc[n][half * (D / 16) + j][r];
                        store_row<PSC_F32, D / 16>(q.part_acc + at * (2 * D) + half * D + (4 * g + r) * (D / 16), o);
                    }
            }
        return;
    }
    typedef typename Element<DT>::type T;
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        const int m = m0 + t * 16 + i;
        float inv[2], squares = 0.f;
        const bool there = m < m_all;
        const int row = s.first_row + min(m, m_all - 1) / q.group, in_group = min(m, m_all - 1) % q.group, out_head = pair * q.group + in_group;
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            const int n = w * RT + t;
            const float sum = column_sum(a.sum[n]);
            inv[w] = sum == 0.f ? 0.f : 1.f / sum;
            if (g == 0 && there) {
                const int64_t at = (int64_t)row * q.q_heads + (2 * pair + w) * q.group + in_group;
                if (q.lse) q.lse[at] = sum == 0.f ? kNegInf : log_sum(a.top[n], sum);
                if (q.stat) *(float2 *)(q.stat + at * 2) = make_float2(a.top[n] == kNegInf ? 0.f : a.top[n], inv[w]);
            }
        }
        const float lam = d.lam[(int64_t)row * d.lam_stride + out_head];
        const bool nothing = inv[0] == 0.f && inv[1] == 0.f;
#pragma unroll
        for (int j = 0; j < D / 8; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float o = a.acc[t][j][r] * inv[0] - lam * (a.acc[RT + t][j][r] * inv[1]);
                a.acc[t][j][r] = o;
                squares += o * o;
            }
        float scale = d.factor;
        if (d.norm) scale *= 1.f / sqrtf(column_sum(squares) * (1.f / (2 * D)) + d.eps);
        T *out = (T *)q.out + ((int64_t)row * (q.q_heads / 2) + out_head) * (2 * D);
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int at = half * D + (4 * g + r) * (D / 16);
                float o[D / 16];
#pragma unroll
                for (int j = 0; j < D / 16; ++j) o[j] = nothing ? 0.f : a.acc[t][half * (D / 16) + j][r] * (d.norm ? d.norm[at + j] * scale : scale);
                if (there) store_row<DT, D / 16>(out + at, o);
            }
    }
}

// Joins the parts of an output head's two maps, a wave to each: its lanes take a part's maximum and sum each (64 parts at a time), then
// 2 D / 64 coordinates of every part, sixteen parts on their way; the second map's wave hands its row to the first's.  Sequences
// without a block have no part: zeros.  What bounds it is the way from load to load and through its instructions, which no workgroup runs
// twice.  8 x 16 heads of 128 with 16 parts to each: 8.7 us (with few
// parts as many as there are: 5 parts of 624 x 32 heads of 64, 28 us; sixteen all the same, 32); a wave with both maps, and every fourth part to a quarter of its lanes, 13.7 one
// map after the other, 17.0 side by side; four parts on their way 13.0.
template <int D, int DT>
__global__ __launch_bounds__(256) void kv_difference_join_kernel(KvView c, KvQueries q, KvDifference d)
{
    constexpr int N = D / 32;  // coordinates of a lane
    __shared__ float second[2][2 * D], second_inv[2];
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), which = wave & 1, lane = lane_id(), out_heads = q.q_heads / 2;
    const int64_t items = (int64_t)q.nrows * out_heads, item = min((int64_t)blockIdx.x * 2 + (wave >> 1), items - 1);  // (past the last: it again)
    const int r = (int)(item / out_heads), out_head = (int)(item % out_heads), pair = out_head / q.group, in_group = out_head % q.group;
    const int b = __builtin_amdgcn_readfirstlane(sequence_of_row(q.offsets, c.batch, q.each, r));
    const RowSet s = rows_of(c, q, b);
    const int place = r - s.first_row;
    const bool nobodys = place < 0 || place >= s.rows;
    const int m = nobodys ? 0 : place * q.group + in_group, in_unit = m % q.unit_rows;
    const uint32_t unit = (uint32_t)(m / q.unit_rows * q.unit_heads + pair);
    Parts all(c, q);
    const int parts = nobodys ? 0 : (int)all.parts_of_unit(Parts::blocks_of_unit(q, s));  // 1: final already
    const int64_t at = (((int64_t)all.first_of(c, q, b) + (int64_t)unit * parts) * 2 + which) * q.unit_rows + in_unit;  // and every 2 unit_rows further
    const int64_t further = 2 * q.unit_rows, row = (int64_t)r * q.q_heads + (2 * pair + which) * q.group + in_group;
    float x[N], top = kNegInf, sum = 0.f;
#pragma unroll
    for (int j = 0; j < N; ++j) x[j] = 0.f;
    for (int p0 = 0; p0 < (parts == 1 ? 0 : parts); p0 += 64) {
        float2 st = make_float2(kNegInf, 0.f);
        if (p0 + lane < parts) st = *(const float2 *)(q.part_stat + (at + (p0 + lane) * further) * 2);
        float now = top;
        if (st.y != 0.f) now = fmaxf(now, st.x);
#pragma unroll
        for (int k = 1; k < 64; k *= 2) now = fmaxf(now, __shfl_xor(now, k));
        const float shrink = now == kNegInf ? 1.f : exp2_fast(top - now);
        const float theirs = st.y == 0.f ? 0.f : now == kNegInf ? 1.f : exp2_fast(st.x - now);
        float add = st.y * theirs;  // (a part that saw nothing: 0)
#pragma unroll
        for (int k = 1; k < 64; k *= 2) add += __shfl_xor(add, k);
        sum = __builtin_fmaf(sum, shrink, add);
        top = now;
#pragma unroll
        for (int j = 0; j < N; ++j) x[j] *= shrink;
        const int last = min(64, parts - p0);
        const auto add_parts = [&](auto ahead) {
            for (int p = 0; p < last; p += ahead.value) {  // (past the last: the last again, times 0)
                float y[ahead.value][N];
#pragma unroll
                for (int u = 0; u < ahead.value; ++u) load_row<PSC_F32, N>(q.part_acc + (at + (p0 + min(p + u, last - 1)) * further) * (2 * D) + lane * N, y[u]);
#pragma unroll
                for (int u = 0; u < ahead.value; ++u) {
                    const float weight = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(theirs), p + u));
#pragma unroll
                    for (int j = 0; j < N; ++j) x[j] = __builtin_fmaf(y[u][j], weight, x[j]);
                }
            }
        };
        if (last <= 2) add_parts(std::integral_constant<int, 2>());
        else if (last <= 6) add_parts(std::integral_constant<int, 6>());
        else add_parts(std::integral_constant<int, 16>());
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    if (lane == 0 && parts != 1) {
        if (q.lse) q.lse[row] = nobodys ? __builtin_nanf("") : sum == 0.f ? kNegInf : log_sum(top, sum);
        if (q.stat && !nobodys) *(float2 *)(q.stat + row * 2) = make_float2(top == kNegInf ? 0.f : top, inv);
    }
#pragma unroll
    for (int j = 0; j < N; ++j) x[j] *= inv;
    if (which == 1) {
        store_row<PSC_F32, N>(&second[wave >> 1][lane * N], x);
        if (lane == 0) second_inv[wave >> 1] = inv;
    }
    __syncthreads();
    if (which == 1 || parts == 1) return;
    const float lam = d.lam[(int64_t)r * d.lam_stride + out_head];
    const bool nothing = inv == 0.f && second_inv[wave >> 1] == 0.f;
    float y[N], squares = 0.f, scale = d.factor;
    load_row<PSC_F32, N>(&second[wave >> 1][lane * N], y);
#pragma unroll
    for (int j = 0; j < N; ++j) {
        x[j] -= lam * y[j];
        squares += x[j] * x[j];
    }
    if (d.norm) {
#pragma unroll
        for (int k = 1; k < 64; k *= 2) squares += __shfl_xor(squares, k);
        scale *= 1.f / sqrtf(squares * (1.f / (2 * D)) + d.eps);
    }
#pragma unroll
    for (int j = 0; j < N; ++j) x[j] = nobodys ? __builtin_nanf("") : nothing ? 0.f : x[j] * (d.norm ? d.norm[lane * N + j] * scale : scale);
    store_row<DT, N>((typename Element<DT>::type *)q.out + item * (2 * D) + lane * N, x);
}

// Blocks of a part at least, and blocks of a memory up to which a unit stays whole (a block is 32 tokens of both heads: half of what they are
// for kv_attention_kernel).
constexpr int64_t kLeastBlocks = 8, kFewBlocks = 32;

// Rows of a wave, in sixteens, at most.
constexpr int most_row_tiles(int dtype, int dim) { return dtype == PSC_F32 || dim == 128 ? 1 : 2; }

// Workgroups from which on a wave's rows are its own (kv_difference_rows_kernel): two to a compute unit, as many as run at
// a time.  With just so many it gains 8 to 12 % or loses 1, with half as many again it lost 5 %, with four times as many it gains 17 %.  8 heads x
// 128, us with rows of their own and without: 512 rows x 4 over 8000 tokens (512 workgroups) 444 and 485, 2048 over 8000 (512) 509 and 578, 8192 of
// 8192 (2048) 1102 and 1320; 2048 of 2048 (512) 140 and 138, 3000 over 8000 (752) 830 and 790; 1024 over 8000 (256) 385 and 315, 256 x 4 over 8000
// (256) 382 and 287.
constexpr int64_t kRowGroups = 512;

// 64 coordinates: where workgroups with rows of their own would be fewer, what they see is cut into parts, as many workgroups as those, if there are
// kRowUnits units and kRowBlocks blocks to a part at least.  4 heads x 64, float16, 8 query heads to each, us so cut and with waves that share out the
// tokens, joins with both: 624 rows over 6209 tokens 138 and 193, in any order 170 and 246; 3 x 300 over 3000 (21 blocks to a part) 99 and 127, 400 over
// 6000 (18) 103 and 137, 900 over 3000 (21) 128 and 122 (lost: more rows and short memories), 1200 over 1900 (14) 105 and 90; 100 over 40000 (14 units) 136 and 140, 40 over 60000 (6 units) 103 and 97.
// (128 coordinates, a part's sums twice as long: 256 rows over 8000 120 and 112, over 30000 292 and 310; 1024 over 4000 203 and 167: never taken.)
constexpr int64_t kRowUnits = 16, kRowBlocks = 16;

template <int DT, int D>
int run_difference(const KvView &c, const KvQueries &q, const KvDifference &d, const KvPlan &p, const float *given, float *received, hipStream_t s)
{
    constexpr int kMost = most_row_tiles(DT, D);
    if (q.nrows > 0) {
        const uint32_t groups = (uint32_t)(c.batch * (c.heads / 2));
        const auto launch = [&](auto rt, auto pos) {
            if constexpr (DT != PSC_F32) {
                if constexpr (D == 64) {
                    if (p.own_rows && p.workgroups) {
                        kv_difference_rows_kernel<D, DT, kMost, pos.value, true><<<(uint32_t)p.most_parts, 256, 0, s>>>(c, q, d);
                        return;
                    }
                }
                if (p.own_rows) {
                    // of a batch with rows of any number, sequences of one tile go to a workgroup whose waves share out the tokens
                    KvDifference mine = d;
                    mine.few = q.offsets && c.batch > 1 ? 16 : 0;
                    kv_difference_rows_kernel<D, DT, kMost, pos.value, false><<<dim3((uint32_t)p.row_groups, 1, groups), 256, 0, s>>>(c, q, mine);
                    mine.most = mine.few;
                    if (mine.few) kv_difference_kernel<D, DT, 1, pos.value, false><<<dim3(1, 1, groups), 256, 0, s>>>(c, q, mine);
                    return;
                }
            }
            if (p.workgroups) kv_difference_kernel<D, DT, rt.value, pos.value, true><<<(uint32_t)p.most_parts, 256, 0, s>>>(c, q, d);
            else kv_difference_kernel<D, DT, rt.value, pos.value, false><<<dim3((uint32_t)p.row_groups, 1, groups), 256, 0, s>>>(c, q, d);
        };
        const auto launch_rows = [&](auto pos) {
            if (p.row_tiles == 1) launch(std::integral_constant<int, 1>(), pos);
            else launch(std::integral_constant<int, kMost>(), pos);
        };
        if (q.positions) launch_rows(std::true_type());
        else launch_rows(std::false_type());
        PSC_HIP_TRY(hipGetLastError());
        if (p.workgroups) {
            kv_difference_join_kernel<D, DT><<<(uint32_t)(((int64_t)q.nrows * (q.q_heads / 2) + 1) / 2), 256, 0, s>>>(c, q, d);
            PSC_HIP_TRY(hipGetLastError());
        }
    }
    if (received) return run_weights<DT, D, 2>(c, q, p, given, received, s);
    return PSC_OK;
}

}  // namespace

KvPlan plan_kv_difference(const KvView &c, int dtype, int group, int64_t nrows, int max_rows, int window, int sinks, bool ordered, bool weights)
{
    KvPlan p;
    const int64_t m = (int64_t)max_rows * group, slots = (int64_t)c.width << c.page_shift, pairs = c.heads / 2;
    p.row_tiles = m <= 16 ? 1 : most_row_tiles(dtype, c.dim);
    p.row_groups = (m + 16 * p.row_tiles - 1) / (16 * p.row_tiles);
    // blocks of 32 tokens that a unit's rows can see at most
    const auto blocks_of_rows = [&](int64_t unit_rows) {
        const int64_t all = (slots + 31) / 32;
        return ordered && window > 0 ? std::min(all, ((int64_t)window + unit_rows / group + 1) / 32 + 2 + ((int64_t)sinks + 31) / 32) : all;
    };
    int64_t blocks = blocks_of_rows(16 * p.row_tiles);
    const int most = 64 * most_row_tiles(dtype, c.dim);
    const int64_t groups = (m + most - 1) / most;
    // (By the rows that there are, not by the most that a sequence may have: single tokens beside a prompt do not fill workgroups.  Whether units are
    // cut into parts does go by the most, for all sequences: long memories with a row or two beside a sequence with many rows are not cut.  31
    // tokens over 8 to 98 thousand, 8 heads x 128: 359 us in a call of their own; with a chunk over 16 thousand, of 2048 rows 1991 us where that
    // takes 926 alone, of 512 rows 6625 where that takes 336, of 300 rows 1158 where that takes 256.)
    p.own_rows = dtype != PSC_F32 && nrows * group * pairs >= kRowGroups * most && m > most / 2;
    if (p.own_rows) p.row_groups = groups;
    int64_t units = p.row_groups * c.batch * pairs;
    const int waves = difference_waves(c.dim, dtype, p.row_tiles);  // workgroups to a compute unit
    p.unit_rows = 16 * p.row_tiles;
    // units of workgroups with rows of their own: as many as there can be, and about as many as there are
    const int64_t most_units = groups * c.batch * pairs, some_units = std::min(most_units, (nrows * group / most + c.batch) * pairs), row_blocks = blocks_of_rows(most);
    if (!p.own_rows && dtype != PSC_F32 && c.dim == 64 && m > most / 2 && nrows * group >= (int64_t)c.batch * most / 2 && some_units >= kRowUnits &&
        most_units <= kRowGroups && some_units * row_blocks >= kRowGroups * kRowBlocks && most_units * row_blocks < (int64_t)1 << 31) {
        p.own_rows = true;
        p.unit_rows = most;
        p.workgroups = (int)kRowGroups;
        units = most_units;
        blocks = row_blocks;
    } else if (!p.own_rows && units > 0 && units < 256 * waves && blocks > kFewBlocks && units * blocks < (int64_t)1 << 31) {
        p.workgroups = 256 * waves;
    }
    if (p.workgroups) {
        // at most one part more to a unit than `wanted` of Parts, which is half of the workgroups or more
        p.most_parts = std::min(p.workgroups + units, units * ((blocks + kLeastBlocks - 1) / kLeastBlocks));
        p.part_stat_bytes = (size_t)(p.most_parts * 2 * p.unit_rows * 8 + 255) / 256 * 256;
        p.part_acc_bytes = (size_t)(p.most_parts * 2 * p.unit_rows * 2 * c.dim * 4 + 255) / 256 * 256;
    }
    p.least_blocks = kLeastBlocks;
    if (weights) plan_pair_weights(c, m, nrows * group * c.heads, &p);
    return p;
}

int launch_kv_difference(const KvView &c, int dtype, const KvQueries &q, const KvDifference &d, const KvPlan &p, const float *given, float *received, hipStream_t s)
{
    return c.dim == 64 ? (dtype == PSC_BF16  ? run_difference<PSC_BF16, 64>(c, q, d, p, given, received, s)
                          : dtype == PSC_F16 ? run_difference<PSC_F16, 64>(c, q, d, p, given, received, s)
                                             : run_difference<PSC_F32, 64>(c, q, d, p, given, received, s))
                       : (dtype == PSC_BF16  ? run_difference<PSC_BF16, 128>(c, q, d, p, given, received, s)
                          : dtype == PSC_F16 ? run_difference<PSC_F16, 128>(c, q, d, p, given, received, s)
                                             : run_difference<PSC_F32, 128>(c, q, d, p, given, received, s));
}

}  // namespace psc
