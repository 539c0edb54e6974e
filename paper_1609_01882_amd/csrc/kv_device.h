// Device code that the kernels over the attention memory in 4 bits share: the format, where tokens and rows lie, rows and keys as
// operands, which tokens a row sees, how long memories are cut into parts.
//
// Format.  A token's head has head_dim coordinates, two to a byte (even coordinates in the low half), as E2M1
// floats: 0, 1/2, 1, 3/2, 2, 3, 4, 6 and a sign.  32 consecutive coordinates share the scale 2^e, e + 127 in a byte.
// With a the largest of the 32 magnitudes, e = floor(log2 a) - 2, one more where a > 7 * 2^e (there the error of
// cutting a to 6 and that of the coarser grid are the same; on normal, Laplace and heavy-tailed data this rule has
// the smallest mean square error of all thresholds on a's mantissa, 1.25 % of the normal data's), clamped to
// -23 .. 13: every held value is then exact in float16 as well as in bfloat16, which the products rely on.
// A token with a value that is not finite gets 255 in all scale bytes of its key, and a value of zeros: its scores
// are NaN, so every row that sees it comes out NaN, and no other row does (a NaN in the value would reach masked
// rows too, as 0 * NaN).
#pragma once

#include <cmath>

#include "common.h"
#include "entry.h"

// Calls fn<type, head_dim>.
#define PSC_KV_DISPATCH(fn, dtype, dim, ...)                                   \
    (dim == 64    ? (dtype == PSC_BF16  ? fn<PSC_BF16, 64>(__VA_ARGS__)        \
                     : dtype == PSC_F16 ? fn<PSC_F16, 64>(__VA_ARGS__)         \
                                        : fn<PSC_F32, 64>(__VA_ARGS__))        \
     : dim == 128 ? (dtype == PSC_BF16  ? fn<PSC_BF16, 128>(__VA_ARGS__)       \
                     : dtype == PSC_F16 ? fn<PSC_F16, 128>(__VA_ARGS__)        \
                                        : fn<PSC_F32, 128>(__VA_ARGS__))       \
                  : (dtype == PSC_BF16  ? fn<PSC_BF16, 256>(__VA_ARGS__)       \
                     : dtype == PSC_F16 ? fn<PSC_F16, 256>(__VA_ARGS__)        \
                                        : fn<PSC_F32, 256>(__VA_ARGS__)))

namespace psc {
namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 h16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 h16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 b16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 b16x8 __attribute__((ext_vector_type(8)));

constexpr uint32_t kNanScale = 255u;
constexpr int kMinScale = 127 - 23, kMaxScale = 127 + 13;
constexpr float kNegInf = -__builtin_huge_valf();
constexpr float kLn2 = 0.693147180559945f;

// A row's probabilities are held as 2^kLift p / (the largest p so far) until the row is done: float16 keeps 11 bits of those down
// to 2^-29 of the largest, and steps of 2^-39 of it below, where 1 as the largest would leave 2^-14 and 2^-24 (a long
// tail that far below one token was lost from the output and not from the sum).  What a row is referred to (its maximum less
// kLift) takes the lift into sums and accumulators alike, and quotients are free of it.
constexpr float kLift = 15.f;

// Scaled scores so large that neighbouring floats lie 2 or more apart.  A row's maximum is then rounded by so much that the
// exponents of its probabilities come out above kLift without limit, or all so low that nothing is left.  Such a row is referred
// to a step or two further down, and exponents above kLift are cut to it: scores that 32 bits hardly tell apart share the row.
constexpr float kCoarse = 16777216.f;
__device__ __forceinline__ bool is_coarse(float top) { return fabsf(top) >= kCoarse && fabsf(top) <= __FLT_MAX__; }
__device__ __forceinline__ float reference_below(float top)  // (coarse as well)
{
    return is_coarse(top) ? fmaxf(__builtin_fmaf(fabsf(top), -0x1p-23f, top), top > 0.f ? kCoarse : -__FLT_MAX__) : top;
}
__device__ __forceinline__ float most_exponent(float reference) { return is_coarse(reference) ? kLift : -kNegInf; }
// log(sum of exp s) from a row's reference and the sum over it (the lift leaves both first: near 0 it would cost bits).
__device__ __forceinline__ float log_sum(float reference, float sum) { return (reference + kLift + __log2f(sum * 0x1p-15f)) * kLn2; }

template <int DT>
struct Element;  // what a row's coordinates are stored as
template <>
struct Element<PSC_BF16> {
    typedef uint16_t type;
    static __device__ float load(type x) { return __uint_as_float((uint32_t)x << 16); }
    static __device__ type store(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }
};
template <>
struct Element<PSC_F16> {
    typedef uint16_t type;
    static __device__ float load(type x) { return (float)__builtin_bit_cast(_Float16, x); }
    static __device__ type store(float x) { return __builtin_bit_cast(uint16_t, (_Float16)x); }
};
template <>
struct Element<PSC_F32> {
    typedef float type;
    static __device__ float load(type x) { return x; }
    static __device__ type store(float x) { return x; }
};

// N consecutive coordinates (16-byte aligned for N * size >= 16) as floats, and back.
template <int DT, int N>
__device__ __forceinline__ void load_row(const void *p, float (&x)[N])
{
    typedef typename Element<DT>::type T;
    T t[N];
    __builtin_memcpy(t, __builtin_assume_aligned(p, N * sizeof(T) < 16 ? N * sizeof(T) : 16), sizeof t);
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = Element<DT>::load(t[i]);
}
template <int DT, int N>
__device__ __forceinline__ void store_row(void *p, const float (&x)[N])
{
    typedef typename Element<DT>::type T;
    T t[N];
#pragma unroll
    for (int i = 0; i < N; ++i) t[i] = Element<DT>::store(x[i]);
    __builtin_memcpy(__builtin_assume_aligned(p, N * sizeof(T) < 16 ? N * sizeof(T) : 16), t, sizeof t);
}

// The larger of the values, and the sum of them, that the four lanes lane % 16 + 0, 16, 32, 48 hold.
__device__ __forceinline__ float column_max(float x)
{
    typedef uint32_t u2 __attribute__((ext_vector_type(2)));
    u2 y = __builtin_bit_cast(u2, __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false));
    x = __builtin_elementwise_maximum(__uint_as_float(y.x), __uint_as_float(y.y));
    y = __builtin_bit_cast(u2, __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false));
    return __builtin_elementwise_maximum(__uint_as_float(y.x), __uint_as_float(y.y));
}
__device__ __forceinline__ float column_sum(float x)
{
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}

__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// Two held values: byte B of `codes`.
template <int B>
__device__ __forceinline__ uint32_t two_b16(uint32_t codes, float scale)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, B));
}
template <int B>
__device__ __forceinline__ uint32_t two_h16(uint32_t codes, float scale)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, B));
}

// The sequence a row belongs to: offsets [batch + 1] ascending, or `each` rows for every sequence.
__device__ __forceinline__ int sequence_of_row(const int32_t *offsets, int batch, int each, int row)
{
    if (!offsets) return row / each;
    int lo = 0, hi = batch;  // offsets[lo] <= row < offsets[hi], where offsets are as they should be
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (offsets[mid] <= row) lo = mid;
        else hi = mid;
    }
    return lo;
}

// The page of a slot, -1 where the table has none.
__device__ __forceinline__ int page_of(const KvView &c, int b, int64_t slot)
{
    if (slot < 0 || slot >= (int64_t)c.width << c.page_shift) return -1;
    const int p = c.table[(int64_t)b * c.width + (int)(slot >> c.page_shift)];
    return p >= 0 && p < c.pages ? p : -1;
}

// Number of the 16 slots that begin at `slot` in a buffer taken as [pages * heads * page / 16] of them (under 2^31: checked by
// the host); -1 where there are none: past the n tokens, or no page.
__device__ __forceinline__ int sixteen_of(const KvView &c, int b, int head, int n, int slot)
{
    const int p = c.table[(int64_t)b * c.width + min(slot >> c.page_shift, c.width - 1)];
    if (slot >= n || (uint32_t)p >= (uint32_t)c.pages) return -1;
    return ((p * c.heads + head) << (c.page_shift - 4)) + ((slot & ((1 << c.page_shift) - 1)) >> 4);
}

// Where a row that is written or read lies: slot lengths[b] + place of its sequence; page -1 where it has none (or nobody has the row).
struct RowPlace {
    int b, place, page;
    int64_t slot;
};
__device__ __forceinline__ RowPlace place_of(const KvView &c, const KvRows &r, int row)
{
    RowPlace p;
    p.b = sequence_of_row(r.offsets, c.batch, r.each, row);
    p.place = row - (r.offsets ? r.offsets[p.b] : p.b * r.each);
    p.slot = (int64_t)c.lengths[p.b] + p.place;
    const bool nobodys = p.place < 0 || (r.offsets && row >= r.offsets[c.batch]);
    p.page = nobodys ? -1 : page_of(c, p.b, p.slot);
    return p;
}

// Writes a token's key x[0] and value x[1], 8 coordinates of each to a lane, D / 8 lanes to a head; four lanes share a scale, whose
// largest magnitude they find as integers.
template <int D>
__device__ __forceinline__ void write_token(const KvView &c, const KvRows &r, const RowPlace &p, int head, int part, const float (&x)[2][8])
{
    constexpr int L = D / 8;
    float top[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        uint32_t bits = 0u;  // the largest magnitude as an integer: NaN and infinity are above all others
#pragma unroll
        for (int i = 0; i < 8; ++i) bits = max(bits, __float_as_uint(x[t][i]) & 0x7fffffffu);
        bits = max(bits, (uint32_t)__shfl_xor((int)bits, 1));
        bits = max(bits, (uint32_t)__shfl_xor((int)bits, 2));
        top[t] = __uint_as_float(bits);
    }
    uint32_t odd = max(__float_as_uint(top[0]), __float_as_uint(top[1]));
#pragma unroll
    for (int d = 4; d < L; d *= 2) odd = max(odd, (uint32_t)__shfl_xor((int)odd, d));
    const bool finite = odd < 0x7f800000u;
    if (p.page < 0) return;
    const int64_t at = ((int64_t)p.page * c.heads + head) << c.page_shift | (p.slot & ((1 << c.page_shift) - 1));
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const uint32_t bits = __float_as_uint(top[t]);
        int e = (int)(bits >> 23) - 2 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
        e = min(max(e, kMinScale), kMaxScale);
        uint32_t codes = 0u;
        if (finite) {
            const float s = scale_of((uint32_t)e);
            codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[t][0], x[t][1], s, 0);
            codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[t][2], x[t][3], s, 1);
            codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[t][4], x[t][5], s, 2);
            codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[t][6], x[t][7], s, 3);
        } else {
            e = t == 0 ? (int)kNanScale : kMinScale;
        }
        uint8_t *to = t == 0 ? c.k_codes : c.v_codes, *scales = t == 0 ? c.k_scales : c.v_scales;
        *(uint32_t *)(to + at * (D / 2) + part * 4) = codes;
        if (part % 4 == 0) scales[at * (D / 32) + part / 4] = (uint8_t)e;
    }
    if (part == 0) {
        const int64_t dense = ((int64_t)p.b * c.heads + head) * ((int64_t)c.width << c.page_shift) + p.slot;
        if (r.positions) r.positions[dense] = (r.first ? r.first[p.b] : c.lengths[p.b]) + p.place;
        if (r.weights) r.weights[dense] = 0.f;
    }
}

// ------------------------------------------------------------------------------------------- attention
// The rows of a (sequence, kv head): row m of it is query head m % group of the sequence's row m / group.
struct RowSet {
    int first_row, rows;  // the sequence's rows, in the caller's array
    int first_pos;        // position of its first row
    int n;                // tokens of the sequence
};
__device__ __forceinline__ RowSet rows_of(const KvView &c, const KvQueries &q, int b)
{
    RowSet s;
    s.first_row = q.offsets ? q.offsets[b] : b * q.each;
    int all = q.offsets ? q.offsets[b + 1] - s.first_row : q.each;
    if (s.first_row < 0 || s.first_row > q.nrows) all = 0;
    all = max(0, min(all, q.nrows - s.first_row));
    s.rows = min(all, q.max_rows);
    s.n = (int)max((int64_t)0, min((int64_t)c.lengths[b], (int64_t)c.width << c.page_shift));
    s.first_pos = q.first ? q.first[b] : s.n - all;
    return s;
}

// The output of rows from .. to - 1, NaN: no sequence has them, and what the memory held is not to pass for a result.
template <int D, int DT>
__device__ void rows_of_nobody(const KvQueries &q, int head, int from, int to)
{
    for (int64_t x = (int64_t)max(from, 0) * q.group + (threadIdx.x >> 4); x < (int64_t)min(to, q.nrows) * q.group; x += blockDim.x >> 4) {
        const int64_t row = x / q.group * q.q_heads + head * q.group + x % q.group;
        const int run = (int)threadIdx.x & 15;
        float nan[D / 16];
#pragma unroll
        for (int j = 0; j < D / 16; ++j) nan[j] = __builtin_nanf("");
        store_row<DT, D / 16>((typename Element<DT>::type *)q.out + row * D + run * (D / 16), nan);
        if (run == 0 && q.lse) q.lse[row] = nan[0];
    }
}

// Blocks of 32 slots that some row at positions lo_pos .. hi_pos can see: those below `sink_blocks`, then
// `main` ... end.  With positions of their own the slots are in no order: all blocks.
struct Blocks {
    int sink_blocks, main, end;
    __device__ int count() const { return sink_blocks + end - main; }
    __device__ int block(int i) const { return i < sink_blocks ? i : i - sink_blocks + main; }
};
__device__ __forceinline__ Blocks blocks_of(const KvQueries &q, int n, int lo_pos, int hi_pos)
{
    Blocks k;
    k.sink_blocks = 0;
    k.main = 0;
    int end = n;
    if (!q.positions && q.causal) end = (int)max((int64_t)0, min((int64_t)n, (int64_t)hi_pos + 1));
    k.end = (end + 31) / 32;
    if (!q.positions && q.window > 0) {
        const int from = (int)max((int64_t)0, min((int64_t)end, (int64_t)lo_pos - q.window + 1));
        k.sink_blocks = (min(q.sinks, end) + 31) / 32;
        k.main = max(k.sink_blocks, from / 32);
        if (k.main > k.end) k.main = k.end;
    }
    return k;
}

// What a lane holds of a block of 32 tokens as it lies in memory.  With i = lane % 16 and g = lane / 16:
// keys of the tokens i and 16 + i, coordinates g D/4 ... (a run of D/8 bytes; whole scale blocks or halves of one);
// values of the tokens 4 g + r and 16 + 4 g + r (r = 0..3), coordinates i D/16 ... (a run of D/32 bytes).
template <int D>
struct Raw {
    uint32_t k[2][D / 32], ks[2];
    uint32_t v[8][D == 256 ? 2 : 1];
    uint32_t vs[2][4];  // of the tokens' scale bytes the words that hold the lane's (value_scale)
};
// The lane's scale byte of token r of four, in the place of a float's exponent.  The conversions look at these eight bits
// alone, so the others may hold what they like.
template <int D>
__device__ __forceinline__ uint32_t value_scale(const uint32_t (&vs)[4], int r, int i)
{
    if constexpr (D == 64) return __builtin_amdgcn_alignbit(vs[r >> 1], vs[r >> 1], (9 + (r & 1) * 16 + (i >> 3) * 8) & 31);
    else if constexpr (D == 128) return __builtin_amdgcn_alignbit(vs[r], vs[r], (9 + (i >> 2) * 8) & 31);
    else return vs[r] << 23;
}

template <int D>
__device__ __forceinline__ void load_keys(const KvView &c, int sixteen, int i, int g, uint32_t (&k)[D / 32], uint32_t &ks)
{
    const int64_t at = (int64_t)max(sixteen, 0) << 4;  // uniform
    const uint8_t *p = c.k_codes + at * (D / 2), *s = c.k_scales + at * (D / 32);
    const uint32_t off = (uint32_t)(i * (D / 2) + g * (D / 8));
    if constexpr (D == 64) {
        const u32x2 t = *(const u32x2 *)(p + off);
        k[0] = t.x;
        k[1] = t.y;
        ks = s[(uint32_t)(i * 2 + (g >> 1))];
    } else {
#pragma unroll
        for (int j = 0; j < D / 128; ++j) {
            const u32x4 t = *(const u32x4 *)(p + off + j * 16);
            k[j * 4 + 0] = t.x;
            k[j * 4 + 1] = t.y;
            k[j * 4 + 2] = t.z;
            k[j * 4 + 3] = t.w;
        }
        if constexpr (D == 128) ks = s[(uint32_t)(i * 4 + g)];
        else ks = *(const uint16_t *)(s + (uint32_t)(i * 8 + g * 2));
    }
}

template <int D>
__device__ __forceinline__ void load_values(const KvView &c, int sixteen, int i, int g, uint32_t (*v)[D == 256 ? 2 : 1], uint32_t (&vs)[4])
{
    const int64_t at = (int64_t)max(sixteen, 0) << 4;
    const uint8_t *p = c.v_codes + at * (D / 2), *s = c.v_scales + at * (D / 32);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const uint32_t off = (uint32_t)((g * 4 + r) * (D / 2) + i * (D / 32));
        if constexpr (D == 64) v[r][0] = *(const uint16_t *)(p + off);
        else if constexpr (D == 128) v[r][0] = *(const uint32_t *)(p + off);
        else {
            const u32x2 t = *(const u32x2 *)(p + off);
            v[r][0] = t.x;
            v[r][1] = t.y;
        }
        if constexpr (D == 256) vs[r] = s[(uint32_t)((g * 4 + r) * 8 + (i >> 1))];
    }
    if constexpr (D == 64) {
        const u32x2 t = *(const u32x2 *)(s + (uint32_t)(g * 8));
        vs[0] = t.x;
        vs[1] = t.y;
    } else if constexpr (D == 128) {
        const u32x4 t = *(const u32x4 *)(s + (uint32_t)(g * 16));
#pragma unroll
        for (int r = 0; r < 4; ++r) vs[r] = t[r];
    }
}

// Keys of 16 tokens as operands of D / 32 products (bfloat16, or float16 for float16 rows): both exact.
template <int D, int DT>
__device__ __forceinline__ void expand_keys(const uint32_t (&k)[D / 32], uint32_t ks, u32x4 (&a)[D / 32])
{
#pragma unroll
    for (int j = 0; j < D / 32; ++j) {
        const float s = scale_of(D == 256 ? (j < 4 ? ks & 255u : ks >> 8) : ks);
        if constexpr (DT == PSC_F16) a[j] = u32x4{two_h16<0>(k[j], s), two_h16<1>(k[j], s), two_h16<2>(k[j], s), two_h16<3>(k[j], s)};
        else a[j] = u32x4{two_b16<0>(k[j], s), two_b16<1>(k[j], s), two_b16<2>(k[j], s), two_b16<3>(k[j], s)};
    }
}

template <int DT>
__device__ __forceinline__ f32x4 mfma_scores(u32x4 a, u32x4 b, f32x4 acc)
{
    if constexpr (DT == PSC_F16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h16x8, a), __builtin_bit_cast(h16x8, b), acc, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b16x8, a), __builtin_bit_cast(b16x8, b), acc, 0, 0, 0);
}

// Sixteen rows as operands: lane (i, g) holds of row i the coordinates g D/4 ..., 8 to a product.  float32 rows are the
// sum of three bfloat16 (24 bits of mantissa): three products each.
template <int D, int DT>
struct Rows {
    static constexpr int kTerms = DT == PSC_F32 ? 3 : 1;
    u32x4 x[kTerms][D / 32];
};
template <int D, int DT>
__device__ __forceinline__ void load_rows(const KvQueries &q, int row, int q_head, int g, Rows<D, DT> &rows)
{
    typedef typename Element<DT>::type T;
    const T *p = (const T *)q.q + (int64_t)row * q.row_stride + (int64_t)q_head * q.head_stride + g * (D / 4);
#pragma unroll
    for (int j = 0; j < D / 32; ++j) {
        if constexpr (DT != PSC_F32) rows.x[0][j] = *(const u32x4 *)(p + j * 8);
        else {
            float x[8];
            load_row<DT, 8>(p + j * 8, x);
#pragma unroll
            for (int term = 0; term < 3; ++term) {
                uint32_t w[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const __bf16 a = (__bf16)x[2 * i], b = (__bf16)x[2 * i + 1];
                    w[i] = (uint32_t)__builtin_bit_cast(uint16_t, a) | (uint32_t)__builtin_bit_cast(uint16_t, b) << 16;
                    x[2 * i] -= (float)a;
                    x[2 * i + 1] -= (float)b;
                }
                rows.x[term][j] = u32x4{w[0], w[1], w[2], w[3]};
            }
        }
    }
}

// Scores of 16 tokens x 16 rows: token 4 g + r in register r, row i.
template <int D, int DT>
__device__ __forceinline__ f32x4 scores_of(const u32x4 (&a)[D / 32], const Rows<D, DT> &rows)
{
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int term = Rows<D, DT>::kTerms - 1; term >= 0; --term)  // the smallest first
#pragma unroll
        for (int j = 0; j < D / 32; ++j) s = mfma_scores<DT>(a[j], rows.x[term][j], s);
    return s;
}

// Which of a lane's 8 tokens (16 h + 4 g + r of the block) its row sees.
struct RowMask {
    int pos, after;  // position; tokens must lie after this one (or be among the first)
};
__device__ __forceinline__ RowMask row_mask(const KvQueries &q, int pos)
{
    RowMask m;
    m.pos = q.causal ? pos : 0x7fffffff;
    m.after = q.window > 0 ? (int)max((int64_t)pos - q.window, (int64_t)-0x80000000ll) : (int)-0x80000000ll;
    return m;
}
__device__ __forceinline__ bool sees(const KvQueries &q, const RowMask &m, int pos_k)
{
    return pos_k <= m.pos && (q.window <= 0 || pos_k > m.after || pos_k < q.sinks);
}

// exp2 of the probability's exponent; values below 2^-126 come out as 0 or denormal, nothing depends on which.
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// A unit of work is 16 RT rows of a (sequence, kv head) and all blocks that they see.  Where there are enough units, a
// workgroup has one.  Where there are few, each is cut into equal parts of at most `per` blocks, a part to a workgroup, with
// `per` such that about as many workgroups come out as run at a time, whatever the lengths of the sequences; kv_join_kernel
// joins the parts.  The units of a sequence count alike, as the widest of them.  (8 sequences of 53 to 131 thousand tokens
// 156 us; every sequence cut into as many parts 175; all units' blocks cut into equal shares, which may end inside units, 162,
// and 32 sequences of 2 to 4 thousand 47 instead of 42, for what a second unit costs a workgroup.)
__device__ __forceinline__ uint32_t scan64(uint32_t x)  // inclusive sums over the wave
{
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xf, 0xf, false);  // row_shr 1, 2, 4, 8
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xf, 0xf, false);
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xf, 0xf, false);
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xf, 0xf, false);
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xa, 0xf, false);  // row_bcast 15, 31
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xc, 0xf, false);
    return x;
}

struct Parts {
    uint32_t parts, upto;  // workgroups of the lane's sequence of 64, and of those up to it
    uint32_t total, per;   // workgroups; blocks of each

    __device__ static uint32_t units_of(const KvView &c, const KvQueries &q, const RowSet &s) { return (uint32_t)((s.rows * q.group + q.unit_rows - 1) / q.unit_rows * q.unit_heads); }
    __device__ static uint32_t blocks_of_unit(const KvQueries &q, const RowSet &s)
    {
        if (s.rows == 0) return 0u;
        const Blocks k = blocks_of(q, s.n, s.first_pos, s.first_pos + s.rows - 1);
        const int most = q.positions || q.window <= 0 ? k.count() : (int)min((int64_t)k.count(), k.sink_blocks + ((int64_t)q.window + q.unit_rows / q.group + 1) / 32 + 2);
        return (uint32_t)most;
    }
    __device__ uint32_t parts_of_unit(uint32_t blocks) const { return (blocks + per - 1) / per; }
    __device__ void load(const KvView &c, const KvQueries &q, int b0)
    {
        const int b = b0 + lane_id();
        parts = 0u;
        if (b < c.batch) {
            const RowSet s = rows_of(c, q, b);
            parts = units_of(c, q, s) * parts_of_unit(blocks_of_unit(q, s));
        }
        upto = scan64(parts);
    }
    __device__ Parts(const KvView &c, const KvQueries &q)
    {
        uint32_t blocks = 0u, units = 0u;
        for (int b = lane_id(); b < c.batch; b += 64) {
            const RowSet s = rows_of(c, q, b);
            const uint32_t n = units_of(c, q, s);
            blocks += n * blocks_of_unit(q, s);
            units += n;
        }
        blocks = (uint32_t)__builtin_amdgcn_readlane((int)scan64(blocks), 63);
        units = (uint32_t)__builtin_amdgcn_readlane((int)scan64(units), 63);
        // rounding up leaves half a part too many per unit
        const uint32_t wanted = max(q.workgroups / 2, q.workgroups - min(q.workgroups, units / 2));
        per = max((uint32_t)q.least_blocks, (blocks + wanted - 1) / wanted);
        total = 0u;
        for (int b0 = 0; b0 < c.batch; b0 += 64) {
            load(c, q, b0);
            total += (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
        }
    }
    // The sequence of workgroup `at` < total, and its first workgroup.
    __device__ int find(const KvView &c, const KvQueries &q, uint32_t at, uint32_t *first)
    {
        uint32_t base = 0u;
        for (int b0 = 0; b0 < c.batch; b0 += 64) {
            if (c.batch > 64) load(c, q, b0);
            const uint64_t behind = ballot64(at - base < upto);
            if (behind) {
                const int l = __builtin_ctzll(behind);
                *first = base + (uint32_t)__builtin_amdgcn_readlane((int)(upto - parts), l);
                return b0 + l;
            }
            base += (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
        }
        return c.batch - 1;  // (not reached)
    }
    // The first workgroup of sequence b.
    __device__ uint32_t first_of(const KvView &c, const KvQueries &q, int b)
    {
        uint32_t base = 0u;
        for (int b0 = 0; b0 < c.batch; b0 += 64) {
            if (c.batch > 64) load(c, q, b0);
            if (b < b0 + 64) return base + (uint32_t)__builtin_amdgcn_readlane((int)(upto - parts), b - b0);
            base += (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
        }
        return base;
    }
};

}  // namespace
}  // namespace psc
