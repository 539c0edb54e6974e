// Attention memory in 4 bits: writing it, attending over it, cutting it to a budget.
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
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "common.h"
#include "entry.h"

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

// ------------------------------------------------------------------------------------------- append, read
// D / 8 lanes to a (row, head), 8 coordinates of its key and of its value to a lane; four lanes share a scale, whose largest
// magnitude they find as integers.  Bound by HBM: 27 thousand rows of 8 heads x 128 float16 (141 MB) in 33 us, 4.3 TB/s;
// kv_read_kernel gives the same back in 30 us, 4.7 TB/s.
template <int DT, int D>
__global__ __launch_bounds__(256) void kv_append_kernel(KvView c, KvRows r)
{
    constexpr int L = D / 8;
    const int64_t item = ((int64_t)blockIdx.x * 256 + threadIdx.x) / L;
    const int part = (int)(threadIdx.x % L);
    if (item >= (int64_t)r.nrows * c.heads) return;
    const int row = (int)(item / c.heads), head = (int)(item % c.heads);
    const int b = sequence_of_row(r.offsets, c.batch, r.each, row);
    const int place = row - (r.offsets ? r.offsets[b] : b * r.each);
    const int64_t slot = (int64_t)c.lengths[b] + place;
    const bool nobodys = place < 0 || (r.offsets && row >= r.offsets[c.batch]);
    const int page = nobodys ? -1 : page_of(c, b, slot);
    typedef typename Element<DT>::type T;
    float x[2][8];
    load_row<DT, 8>((const T *)r.k + row * r.k_stride + head * r.k_head_stride + part * 8, x[0]);
    load_row<DT, 8>((const T *)r.v + row * r.v_stride + head * r.v_head_stride + part * 8, x[1]);
    float top[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        top[t] = 0.f;
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
    if (page < 0) return;
    const int64_t at = ((int64_t)page * c.heads + head) << c.page_shift | (slot & ((1 << c.page_shift) - 1));
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
        const int64_t dense = ((int64_t)b * c.heads + head) * ((int64_t)c.width << c.page_shift) + slot;
        if (r.positions) r.positions[dense] = (r.first ? r.first[b] : c.lengths[b]) + place;
        if (r.weights) r.weights[dense] = 0.f;
    }
}

template <int DT, int D>
__global__ __launch_bounds__(256) void kv_read_kernel(KvView c, KvRows r, void *k_out, void *v_out)
{
    constexpr int L = D / 8;
    const int64_t item = ((int64_t)blockIdx.x * 256 + threadIdx.x) / L;
    const int part = (int)(threadIdx.x % L);
    if (item >= (int64_t)r.nrows * c.heads) return;
    const int row = (int)(item / c.heads), head = (int)(item % c.heads);
    const int b = sequence_of_row(r.offsets, c.batch, r.each, row);
    const int place = row - (r.offsets ? r.offsets[b] : b * r.each);
    const int64_t slot = (int64_t)c.lengths[b] + place;
    const bool nobodys = place < 0 || (r.offsets && row >= r.offsets[c.batch]);
    const int page = nobodys ? -1 : page_of(c, b, slot);
    typedef typename Element<DT>::type T;
    const int64_t at = page < 0 ? 0 : ((int64_t)page * c.heads + head) << c.page_shift | (slot & ((1 << c.page_shift) - 1));
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const uint8_t *from = t == 0 ? c.k_codes : c.v_codes, *scales = t == 0 ? c.k_scales : c.v_scales;
        uint32_t codes = 0u, e = kMinScale;
        if (page >= 0) {
            codes = *(const uint32_t *)(from + at * (D / 2) + part * 4);
            e = scales[at * (D / 32) + part / 4];
        }
        const float s = scale_of(e);
        const uint32_t two[4] = {two_b16<0>(codes, s), two_b16<1>(codes, s), two_b16<2>(codes, s), two_b16<3>(codes, s)};
        float x[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(two[i] << 16);
            x[2 * i + 1] = __uint_as_float(two[i] & 0xffff0000u);
        }
        store_row<DT, 8>((T *)(t == 0 ? k_out : v_out) + item * D + part * 8, x);
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

// One wave attends with 16 RT rows over every fourth of the workgroup's blocks.
//
// The transposed products keep everything of a row in the lanes of its column: scores K Q^T have the tokens in rows and
// the rows in columns, so a lane holds 8 scores of one row; they are the operand of V^T P^T as they are, since the
// order of the tokens inside a product is free as long as both sides agree; and the running maximum, which rescales
// a column of the output, is the lane's own.  Values have to be transposed for that: a lane takes a run of
// coordinates of 8 tokens and pairs up the tokens' values of one coordinate with one permutation each.
// What it is bound by: a few rows read the cache at 5.7 TB/s (8 sequences of 53 to 131 thousand tokens x 8 heads x 128, 825 MB
// in 145 us); many rows are bound by vector instructions (32 rows x 32 tokens: 16 exp2 of four issue slots each, 64 conversions,
// 32 permutations, 110 others for 32 products): 2048 rows of 4 x 8 heads over 16384 tokens 656 us, 795 TFLOP/s.
// Scores, maximum, sum and output are 32-bit floats.  Probabilities are rounded to float16: by at most 2^-11 of each, an
// eighth of what the output's own rounding to bfloat16 may add (float32 rows: two float16, 2^-22 of each down to 2^-18 of the
// largest), and never by more than 2^-40 of the row's largest beyond that (kLift).
template <int D, int DT, int RT, bool kPos>
struct Attention {
    f32x4 acc[RT][D / 16];
    float top[RT], sum[RT];  // of the scaled scores in units of log 2, the maximum less kLift; the sum is the lane's own share
    Rows<D, DT> rows[RT];

    // kFar: rows whose scores are coarse may be among them
    template <bool kFar>
    __device__ void block(const KvView &c, const KvQueries &q, const Raw<D> &raw, const int (&positions)[8], const RowMask (&mask)[RT], int slot, int lim0,
                          int lim1, int n, bool whole, float factor, int i, int g, float *scores)
    {
        f32x4 s[RT][2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            u32x4 a[D / 32];
            expand_keys<D, DT>(raw.k[h], raw.ks[h], a);
#pragma unroll
            for (int t = 0; t < RT; ++t) s[t][h] = scores_of<D, DT>(a, rows[t]);
        }
        if (!whole) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int at = slot + 16 * h + 4 * g + r;
                    const bool there = at < (h ? lim1 : lim0);
                    const int pos = kPos ? positions[4 * h + r] : at;
#pragma unroll
                    for (int t = 0; t < RT; ++t)
                        if (!(there && sees(q, mask[t], pos))) s[t][h][r] = kNegInf;
                }
        }
        if constexpr (RT == 1) {
            if (scores) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    if (slot + 16 * h < n) *(f32x4 *)(scores + slot + 16 * h + 4 * g) = s[0][h];
            }
        }
        uint32_t p[RT][2][4];  // float16 pairs (the second array: what the first leaves of float32 rows' probabilities)
#pragma unroll
        for (int t = 0; t < RT; ++t) {
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
                for (int j = 0; j < D / 16; ++j) acc[t][j] *= shrink;
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
        // tokens 0..7 of the lane: 4 g + r, then 16 + 4 g + r
        uint32_t held[8];
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            held[t] = value_scale<D>(raw.vs[t >> 2], t & 3, i);
        }
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
                const uint32_t x = raw.v[t][y / 4];
                w[t] = y % 4 == 0 ? two_h16<0>(x, sc) : y % 4 == 1 ? two_h16<1>(x, sc) : y % 4 == 2 ? two_h16<2>(x, sc) : two_h16<3>(x, sc);
            }
            u32x4 lo, hi;
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                lo[t] = __builtin_amdgcn_perm(w[2 * t + 1], w[2 * t], 0x05040100u);
                hi[t] = __builtin_amdgcn_perm(w[2 * t + 1], w[2 * t], 0x07060302u);
            }
#pragma unroll
            for (int t = 0; t < RT; ++t) {
#pragma unroll
                for (int term = DT == PSC_F32 ? 1 : 0; term >= 0; --term) {
                    const h16x8 pr = __builtin_bit_cast(h16x8, (u32x4){p[t][term][0], p[t][term][1], p[t][term][2], p[t][term][3]});
                    acc[t][2 * y] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h16x8, lo), pr, acc[t][2 * y], 0, 0, 0);
                    acc[t][2 * y + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h16x8, hi), pr, acc[t][2 * y + 1], 0, 0, 0);
                }
            }
        }
    }
};

// Waves of a SIMD that the registers are to leave room for.  (8 x 128k tokens, one row, 128 coordinates: 191 us without a
// bound, 175 with 2 or 3, 317 with 4; 2048 rows over 16k tokens, 32 rows to a wave: 1336, 792 with 2, 2477 with 3.)
template <int D, int DT, int RT>
constexpr int attention_waves()
{
    if (D == 256) return DT == PSC_F32 ? 1 : 2;
    return RT == 1 ? (DT == PSC_F32 ? 2 : D == 64 ? 4 : 3) : DT == PSC_F32 ? 1 : 2;
}

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

    __device__ static uint32_t units_of(const KvView &c, const KvQueries &q, const RowSet &s) { return (uint32_t)((s.rows * q.group + q.unit_rows - 1) / q.unit_rows * c.heads); }
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

template <int D, int RT>
struct Joined {  // of a workgroup's four waves
    static constexpr int kStride = D + 4;
    float acc[4][16 * kStride];
    float tops[4][16 * RT], sums[4][16 * RT];
};

// Blocks begin .. end - 1 of the rows from m0 on of (b, head): the workgroup's four waves take every fourth each and are
// joined in LDS.  part < 0: these are all blocks, and the result is final.
template <int D, int DT, int RT, bool kPos>
__device__ __forceinline__ void attend_unit(const KvView &c, const KvQueries &q, const RowSet &s, int b, int head, int m0, const Blocks &blocks, int begin,
                                            int end, int64_t part, Joined<D, RT> &joined)
{
    const int lane = lane_id(), i = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int m_all = s.rows * q.group, m_end = min(m0 + 16 * RT, m_all);
    const int lo_pos = s.first_pos + m0 / q.group, hi_pos = s.first_pos + (m_end - 1) / q.group;
    constexpr int step = 4;

    Attention<D, DT, RT, kPos> a;
    RowMask mask[RT];
    const auto start = [&] {
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            const int m = min(m0 + t * 16 + i, m_all - 1), place = m / q.group;  // (rows past the last: the last one again)
            load_rows<D, DT>(q, s.first_row + place, head * q.group + m - place * q.group, g, a.rows[t]);
            mask[t] = row_mask(q, s.first_pos + place);
            a.top[t] = kNegInf;
            a.sum[t] = 0.f;
#pragma unroll
            for (int j = 0; j < D / 16; ++j) a.acc[t][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    };
    start();
    const int64_t dense = ((int64_t)b * c.heads + head) * ((int64_t)c.width << c.page_shift);

    // The places of 32 of the wave's blocks are held across the lanes; the codes of the block after the one that is worked on
    // are on their way, without a branch around their loads (past the last block: of a page that is there).
    const int own = begin + wave, mine = end > own ? (end - own + step - 1) / step : 0;
    auto pages_from = [&](int k) {
        return sixteen_of(c, b, head, s.n, blocks.block(min(own + (k + (lane >> 1)) * step, end - 1)) * 32 + (lane & 1) * 16);
    };
    auto load = [&](int k, const int (&pg)[2], Raw<D> &r) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            load_keys<D>(c, pg[h], i, g, r.k[h], r.ks[h]);
            load_values<D>(c, pg[h], i, g, &r.v[4 * h], r.vs[h]);
        }
    };
    // positions of the value tokens of a block, where they have some of their own (asked for when the block is worked on: held
    // for the next one too they would not fit the registers)
    auto load_positions = [&](int k, int (&pos)[8]) {
        if constexpr (kPos) {
            const int sl = blocks.block(min(own + k * step, end - 1)) * 32;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int4 x = *(const int4 *)(q.positions + dense + min(sl + 16 * h, (c.width << c.page_shift) - 16) + 4 * g);
                pos[4 * h] = x.x;
                pos[4 * h + 1] = x.y;
                pos[4 * h + 2] = x.z;
                pos[4 * h + 3] = x.w;
            }
        }
    };
    // where the scores of the lane's row are left for kv_weights_of_scores_kernel
    float *scores = nullptr;
    if constexpr (RT == 1)
        if (q.scores && i < m_all) scores = q.scores + (((int64_t)b * c.heads + head) * q.scores_rows + i) * ((int64_t)c.width << c.page_shift);
    const auto work = [&](auto far, int k, const Raw<D> &raw, const int (&pos)[8], const int (&pg)[2]) {
        const int slot = blocks.block(own + k * step) * 32;
        const bool there = slot + 32 <= s.n && pg[0] >= 0 && pg[1] >= 0 && !kPos;
        const bool whole = there && (!q.causal || slot + 31 <= lo_pos) &&
                           (q.window <= 0 || (int64_t)hi_pos - slot < q.window || slot + 32 <= q.sinks);
        a.template block<far.value>(c, q, raw, pos, mask, slot, pg[0] >= 0 ? s.n : 0, pg[1] >= 0 ? s.n : 0, s.n, whole, q.factor, i, g, scores);
    };
    if (mine > 0) {
        // (two sets of registers in turn: copying the next block's costs 8 % of a block of 32 rows)
        Raw<D> raw[2];
        int ids = pages_from(0), pages[2][2] = {{__builtin_amdgcn_readlane(ids, 0), __builtin_amdgcn_readlane(ids, 1)}, {-1, -1}};
        load(0, pages[0], raw[0]);
        for (int k0 = 0; k0 < mine; k0 += 32) {
            const int ids_then = pages_from(k0 + 32), k_end = min(32, mine - k0);
            const auto turn = [&](int k, const Raw<D> &now, const int (&now_pages)[2], Raw<D> &next, int (&next_pages)[2]) {
                if (k < 31) {
                    next_pages[0] = __builtin_amdgcn_readlane(ids, 2 * k + 2);
                    next_pages[1] = __builtin_amdgcn_readlane(ids, 2 * k + 3);
                } else {
                    next_pages[0] = __builtin_amdgcn_readlane(ids_then, 0);
                    next_pages[1] = __builtin_amdgcn_readlane(ids_then, 1);
                }
                int pos[8];
                load_positions(k0 + k, pos);
                load(k0 + k + 1, next_pages, next);
                work(std::false_type(), k0 + k, now, pos, now_pages);
            };
            for (int k = 0; k < k_end; k += 2) {  // (32 is even: a set's turn does not change from one 32 to the next)
                turn(k, raw[0], pages[0], raw[1], pages[1]);
                if (k + 1 < k_end) turn(k + 1, raw[1], pages[1], raw[0], pages[0]);
            }
            ids = ids_then;
        }
    }
    // Decided at the end, and all done again: a look at every block costs 2 to 3 % of a large chunk.
    bool far = false;
#pragma unroll
    for (int t = 0; t < RT; ++t) far = far || is_coarse(a.top[t]);
    if (__any(far)) {
        asm volatile("" ::: "memory");  // (the rows are read again: kept, they would cost the pass above registers)
        start();
#pragma unroll 1
        for (int k = 0; k < mine; ++k) {
            const int ids = pages_from(k), pages[2] = {__builtin_amdgcn_readlane(ids, 0), __builtin_amdgcn_readlane(ids, 1)};
            int pos[8];
            load_positions(k, pos);
            Raw<D> raw;
            load(k, pages, raw);
            work(std::true_type(), k, raw, pos, pages);
        }
    }
#pragma unroll
    for (int t = 0; t < RT; ++t) a.sum[t] = column_sum(a.sum[t]);
    if (g == 0) {
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            joined.tops[wave][t * 16 + i] = a.top[t];
            joined.sums[wave][t * 16 + i] = a.sum[t];
        }
    }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        float top = kNegInf;
#pragma unroll
        for (int w = 0; w < 4; ++w) top = fmaxf(top, joined.tops[w][t * 16 + i]);
        const float shrink = top == kNegInf ? 1.f : exp2_fast(a.top[t] - top);
        if (t) __syncthreads();
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            float x[D / 16];
#pragma unroll
            for (int j = 0; j < D / 16; ++j) x[j] = a.acc[t][j][r] * shrink;
            store_row<PSC_F32, D / 16>(&joined.acc[wave][i * joined.kStride + (g * 4 + r) * (D / 16)], x);
        }
        __syncthreads();
        const int local = (int)threadIdx.x >> 4, run = (int)threadIdx.x & 15, m = m0 + t * 16 + local;
        if (m < m_all) {
            float best = kNegInf, sum = 0.f;
#pragma unroll
            for (int w = 0; w < 4; ++w) best = fmaxf(best, joined.tops[w][t * 16 + local]);
#pragma unroll
            for (int w = 0; w < 4; ++w) sum += joined.sums[w][t * 16 + local] * (best == kNegInf ? 1.f : exp2_fast(joined.tops[w][t * 16 + local] - best));
            float x[D / 16];
#pragma unroll
            for (int j = 0; j < D / 16; ++j) {
                x[j] = 0.f;
#pragma unroll
                for (int w = 0; w < 4; ++w) x[j] += joined.acc[w][local * joined.kStride + run * (D / 16) + j];
            }
            if (part >= 0) {
                const int64_t at = part * (16 * RT) + t * 16 + local;
                if (run == 0) *(float2 *)(q.part_stat + at * 2) = make_float2(best, sum);
                store_row<PSC_F32, D / 16>(q.part_acc + at * D + run * (D / 16), x);
            } else {
                const int64_t row = (int64_t)(s.first_row + m / q.group) * q.q_heads + head * q.group + m % q.group;
                const float inv = sum == 0.f ? 0.f : 1.f / sum;
                if (run == 0) {
                    if (q.lse) q.lse[row] = sum == 0.f ? kNegInf : log_sum(best, sum);
                    if (q.stat) *(float2 *)(q.stat + row * 2) = make_float2(best == kNegInf ? 0.f : best, inv);
                }
#pragma unroll
                for (int j = 0; j < D / 16; ++j) x[j] *= inv;
                store_row<DT, D / 16>((typename Element<DT>::type *)q.out + row * D + run * (D / 16), x);
            }
        }
    }
}

template <int D, int DT, int RT, bool kPos, bool kParts>
__global__ __launch_bounds__(256, (attention_waves<D, DT, RT>())) void kv_attention_kernel(KvView c, KvQueries q)
{
    __shared__ Joined<D, RT> joined;
    if constexpr (!kParts) {
        const int b = (int)blockIdx.z / c.heads, head = (int)blockIdx.z % c.heads, m0 = (int)blockIdx.x * 16 * RT;
        const RowSet s = rows_of(c, q, b);
        if (q.offsets && m0 == 0) {
            if (b == 0) rows_of_nobody<D, DT>(q, head, 0, s.first_row);
            rows_of_nobody<D, DT>(q, head, s.first_row + s.rows, b + 1 < c.batch ? q.offsets[b + 1] : q.nrows);
        }
        if (m0 >= s.rows * q.group) return;
        const Blocks blocks = blocks_of(q, s.n, s.first_pos + m0 / q.group, s.first_pos + (min(m0 + 16 * RT, s.rows * q.group) - 1) / q.group);
        attend_unit<D, DT, RT, kPos>(c, q, s, b, head, m0, blocks, 0, blocks.count(), -1, joined);
    } else {
        Parts all(c, q);
        if (blockIdx.x >= all.total) return;
        uint32_t first;
        const int b = all.find(c, q, blockIdx.x, &first);
        const RowSet s = rows_of(c, q, b);
        const uint32_t each = Parts::blocks_of_unit(q, s), parts = all.parts_of_unit(each);
        const uint32_t unit = (blockIdx.x - first) / parts, part = blockIdx.x - first - unit * parts;
        const int head = (int)unit % c.heads, m0 = (int)unit / c.heads * 16 * RT;
        const Blocks blocks = blocks_of(q, s.n, s.first_pos + m0 / q.group, s.first_pos + (min(m0 + 16 * RT, s.rows * q.group) - 1) / q.group);
        const int count = blocks.count(), from = (int)((uint64_t)part * each / parts), to = (int)((uint64_t)(part + 1) * each / parts);
        attend_unit<D, DT, RT, kPos>(c, q, s, b, head, m0, blocks, min(count, from), min(count, to), parts == 1 ? -1 : (int64_t)blockIdx.x, joined);
    }
}

// Joins a row's parts, a wave to a row: each lane takes a part's maximum and sum (64 parts at a time), then the lanes take
// D / 16 coordinates of every fourth part each.  Sequences without a block have no part: zeros.
template <int D, int DT>
__global__ __launch_bounds__(256) void kv_join_kernel(KvView c, KvQueries q)
{
    const int lane = lane_id(), run = lane & 15, quarter = lane >> 4;
    const int64_t row = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    if (row >= (int64_t)q.nrows * q.q_heads) return;
    const int r = (int)(row / q.q_heads), q_head = (int)(row % q.q_heads), b = __builtin_amdgcn_readfirstlane(sequence_of_row(q.offsets, c.batch, q.each, r));
    const RowSet s = rows_of(c, q, b);
    const int place = r - s.first_row;
    if (place < 0 || place >= s.rows) {  // nobody's
        float nan[D / 16];
#pragma unroll
        for (int j = 0; j < D / 16; ++j) nan[j] = __builtin_nanf("");
        if (quarter == 0) store_row<DT, D / 16>((typename Element<DT>::type *)q.out + row * D + run * (D / 16), nan);
        if (lane == 0 && q.lse) q.lse[row] = nan[0];
        return;
    }
    const int m = place * q.group + q_head % q.group, in_unit = m % q.unit_rows;
    const uint32_t unit = (uint32_t)(m / q.unit_rows * c.heads + q_head / q.group);
    Parts all(c, q);
    const int parts = (int)all.parts_of_unit(Parts::blocks_of_unit(q, s));
    if (parts == 1) return;  // (final already)
    const int64_t at = ((int64_t)all.first_of(c, q, b) + (int64_t)unit * parts) * q.unit_rows + in_unit;  // and every unit_rows further
    float top = kNegInf, sum = 0.f, x[D / 16];
#pragma unroll
    for (int j = 0; j < D / 16; ++j) x[j] = 0.f;
    for (int p0 = 0; p0 < parts; p0 += 64) {
        float2 st = make_float2(kNegInf, 0.f);
        if (p0 + lane < parts) st = *(const float2 *)(q.part_stat + (at + (int64_t)(p0 + lane) * q.unit_rows) * 2);
        float now = top;
        if (st.y != 0.f) now = fmaxf(now, st.x);
#pragma unroll
        for (int d = 1; d < 64; d *= 2) now = fmaxf(now, __shfl_xor(now, d));
        const float shrink = now == kNegInf ? 1.f : exp2_fast(top - now);
        const float theirs = st.y == 0.f ? 0.f : now == kNegInf ? 1.f : exp2_fast(st.x - now);
        float add = st.y * theirs;  // (a part that saw nothing: 0)
#pragma unroll
        for (int d = 1; d < 64; d *= 2) add += __shfl_xor(add, d);
        sum = __builtin_fmaf(sum, shrink, add);
        top = now;
#pragma unroll
        for (int j = 0; j < D / 16; ++j) x[j] *= shrink;
        const int last = min(64, parts - p0);
        for (int k = 0; k < last; k += 4) {  // (all lanes to the end: a lane's weight is asked of another one)
            const int p = k + quarter;
            const float w = __shfl(theirs, p);  // past the last: 0
            float y[D / 16];
            load_row<PSC_F32, D / 16>(q.part_acc + (at + (int64_t)(p0 + min(p, last - 1)) * q.unit_rows) * D + run * (D / 16), y);
#pragma unroll
            for (int j = 0; j < D / 16; ++j) x[j] = __builtin_fmaf(y[j], w, x[j]);
        }
    }
#pragma unroll
    for (int j = 0; j < D / 16; ++j) x[j] = column_sum(x[j]);
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    if (lane == 0) {
        if (q.lse) q.lse[row] = sum == 0.f ? kNegInf : log_sum(top, sum);
        if (q.stat) *(float2 *)(q.stat + row * 2) = make_float2(top == kNegInf ? 0.f : top, inv);
    }
#pragma unroll
    for (int j = 0; j < D / 16; ++j) x[j] *= inv;
    if (quarter == 0) store_row<DT, D / 16>((typename Element<DT>::type *)q.out + row * D + run * (D / 16), x);
}

// The weight that every token received, from the scores that the attention left: a thread to four slots.  For up to
// kScoreRows rows (query heads times rows of a sequence): the scores' 4 bytes to a row, written and read, are then less than
// the keys' bytes and what comes with expanding them (32 x 4k tokens, 4 rows: 31 us with the keys once more).  They are kept up to a
// size that a caller can spare (whole calls of 8 rows x 128, kept and not: 8 x 8 x 131k tokens, 0.27 GB of scores, 269 and 355 us;
// 16 x 8 x 262k, 1.1 GB, 1118 and 1426).
constexpr int kScoreRows = 8;
constexpr int64_t kMostScoreBytes = (int64_t)4 << 30;
template <int N>
__global__ __launch_bounds__(256) void kv_weights_of_scores_kernel(KvView c, KvQueries q, const float *given, float *received)
{
    const int b = (int)blockIdx.z / c.heads, head = (int)blockIdx.z % c.heads;
    const int64_t stride = (int64_t)c.width << c.page_shift, dense = (int64_t)blockIdx.z * stride;
    const int64_t first = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (first >= stride) return;
    const int slot = (int)first;
    const RowSet s = rows_of(c, q, b);
    const int m_all = s.rows * q.group;
    f32x4 total = {0.f, 0.f, 0.f, 0.f};
    if (given) total = *(const f32x4 *)(given + dense + slot);
    if (slot < s.n && m_all > 0) {
        const Blocks blocks = blocks_of(q, s.n, s.first_pos, s.first_pos + s.rows - 1);
        if (slot / 32 < blocks.sink_blocks || (slot / 32 >= blocks.main && slot / 32 < blocks.end)) {
            f32x4 x[N], sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int m = 0; m < N; ++m)
                x[m] = *(const f32x4 *)(q.scores + ((int64_t)blockIdx.z * q.scores_rows + min(m, m_all - 1)) * stride + slot);
#pragma unroll
            for (int m = 0; m < N; ++m) {
                const int mm = min(m, m_all - 1);
                const float2 st = *(const float2 *)(q.stat + ((int64_t)(s.first_row + mm / q.group) * q.q_heads + head * q.group + mm % q.group) * 2);
                const float inv = m < m_all ? st.y : 0.f, most = most_exponent(st.x);
#pragma unroll
                for (int j = 0; j < 4; ++j)  // (the larger of NaN and 0 is 0: rows that came out NaN add nothing)
                    sum[j] += fmaxf(exp2_fast(fminf(__builtin_fmaf(x[m][j], q.factor, -st.x), most)) * inv, 0.f);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) total[j] += slot + j < s.n ? sum[j] : 0.f;
        }
    }
    *(f32x4 *)(received + dense + slot) = total;
}

// The same with the scores once more, from the same products as in the attention itself, so that with the row's reference and
// sum each probability is the one that was used, before it was rounded.  kSplitRows: a workgroup has 16 kTiles tokens and each wave a quarter of the
// rows that can see one; otherwise a wave has 16 kTiles tokens and all rows.  The next 16 rows are on their way while 16 are worked on,
// their places found by adding, not dividing.  The shares are added in one order.  Rows that came out NaN add nothing.  16 exp2
// and some 90 other vector instructions for 16 rows x 64 tokens: up to 701 rows of 3 x 4 heads x 64 over 5003, 40 us (with 32
// tokens 52), in which a compute unit works 58 % of the time and issues vector instructions in 81 % of the cycles that it works.
template <int D, int DT, bool kSplitRows, int kTiles>
__global__ __launch_bounds__(256, D == 256 && DT == PSC_F32 ? 1 : 2) void kv_weights_kernel(KvView c, KvQueries q, const float *given, float *received)
{
    const int lane = lane_id(), i = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int b = (int)blockIdx.z / c.heads, head = (int)blockIdx.z % c.heads;
    const RowSet s = rows_of(c, q, b);
    const int64_t stride = (int64_t)c.width << c.page_shift, dense = (int64_t)blockIdx.z * stride;
    const int64_t block = kSplitRows ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * 4 + wave;
    if (block * 16 * kTiles >= stride) return;  // (with kSplitRows the whole workgroup)
    const int slot = (int)(block * 16 * kTiles), m_all = s.rows * q.group;

    float total[kTiles][4] = {};
    if (slot < s.n && m_all > 0) {
        int places[kTiles], pos[kTiles][4];
        bool there = !q.positions;
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
                pos[h][r] = q.positions && at < s.n ? q.positions[dense + at] : at;
            }
        }
        int64_t m_begin = 0, m_end = m_all;
        if (!q.positions) {
            if (q.causal) m_begin = max((int64_t)0, (int64_t)slot - s.first_pos) * q.group / 16 * 16;
            if (q.window > 0 && slot >= q.sinks)
                m_end = min(m_end, max((int64_t)0, (int64_t)slot + 16 * kTiles - 1 + q.window - s.first_pos) * q.group);
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
                const bool coarse = is_coarse(st.x), mine = there && !coarse && (!q.causal || pos_q >= slot + 16 * kTiles - 1) && (q.window <= 0 || (int64_t)pos_q - slot < q.window || slot + 16 * kTiles <= q.sinks);
                if (!__all(mine)) {
                    const RowMask mask = row_mask(q, pos_q);
#pragma unroll
                    for (int h = 0; h < kTiles; ++h)
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (!(places[h] >= 0 && slot + 16 * h + 4 * g + r < s.n && sees(q, mask, pos[h][r]))) x[h][r] = kNegInf;
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
    if (one && slot + in_block < stride) received[dense + slot + in_block] = (given ? given[dense + slot + in_block] : 0.f) + mine;
}

// ------------------------------------------------------------------------------------------- eviction
constexpr int kEvictThreads = 1024;

// Order of a token's claim to stay: the first and the most recent above all, then the weight; NaN below all.  A slot without a page
// holds no token: below the budget it stays as it is (it can take none), behind it it is never kept.
constexpr uint32_t kStays = 0xffffffffu, kNanClaim = 1u, kNoToken = 0u;
__device__ __forceinline__ uint32_t claim_of(const KvEvict &e, int seen, float weight, int pos)
{
    if (pos < e.sinks || (int64_t)pos >= (int64_t)seen - e.recent) return kStays;
    return weight == weight ? dist_key(weight) : kNanClaim;
}

// Selecting and listing.  The budget-th largest claim is found digit by digit (11, 11 and 10 bits) from counts in LDS;
// the slots below the budget that fall free and the kept ones behind it are then listed in order.  A workgroup takes
// kSegment slots, 16 to a thread; a wave's are consecutive, so that ballots give places in order.
// Memories of one segment: all of it in one kernel, claims in registers.  Longer ones are cut into segments, at the budget
// first, so that a segment has either free slots or kept ones to list, and go through
//   kv_count_kernel   counts of the first digit, per segment
//   kv_gather_kernel  the first digit of the wanted claim, and the claims that share it, in order (a workgroup per segment,
//                     each adding up all segments' counts)
//   kv_pick_kernel    the rest of the claim from these few, and what each segment keeps (a workgroup per kv head)
//   kv_list_kernel    the lists
// One workgroup per kv head for all of it took 231 us for 8 x 8 memories of up to 131072 tokens, five passes of which each
// waits for memory; the four
// kernels take 65 (whole call 123; when it was 121.6, with 8, 12, 24, 32 claims to a thread 127, 123, 131, 146): issue of the ballots and the
// counts' conflicts in LDS, then what each waits for at its start.
constexpr int kSegmentKeys = 16, kSegment = kEvictThreads * kSegmentKeys, kBins = 2048;

struct Segment {
    int begin, end;  // slots
    bool below;      // the budget
};
__device__ __forceinline__ Segment segment_of(const KvEvict &e, int n, int seg)
{
    Segment x;
    x.below = seg < e.segments_below;
    const int64_t from = x.below ? (int64_t)seg * kSegment : e.budget + (int64_t)(seg - e.segments_below) * kSegment;
    const int64_t to = x.below ? min((int64_t)e.budget, from + kSegment) : from + kSegment;
    x.begin = (int)min((int64_t)n, from);
    x.end = (int)min((int64_t)n, to);
    return x;
}

struct Memory {
    int b, n, seen;
    int64_t dense;
};
__device__ __forceinline__ Memory memory_of(const KvView &c, const KvEvict &e, int bh)
{
    Memory m;
    m.b = bh / c.heads;
    const int64_t stride = (int64_t)c.width << c.page_shift;
    m.n = (int)max((int64_t)0, min((int64_t)c.lengths[m.b], stride));
    m.seen = e.seen ? e.seen[m.b] : m.n;
    m.dense = (int64_t)bh * stride;
    return m;
}

// The claims of slots begin .. end, N to a thread: its j-th at begin + (wave * N + j) * 64 + lane; 0 past the end.  The wave's slots
// lie on 65 pages at most, which the lanes look up together.
template <int N>
__device__ __forceinline__ void load_claims(const KvView &c, const KvEvict &e, const Memory &m, int begin, int end, uint32_t (&x)[N])
{
    const int wave_begin = begin + ((int)threadIdx.x >> 6) * (64 * N), at = wave_begin + lane_id();
    const int32_t *table = c.table + (int64_t)m.b * c.width;
    const int first_page = wave_begin >> c.page_shift;
    const int page = table[min(first_page + lane_id(), c.width - 1)], last_page = table[min(first_page + 64, c.width - 1)];
    float w[N];
    int pos[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const int s = max(0, min(at + j * 64, end - 1));
        w[j] = e.weights[m.dense + s];
        pos[j] = e.positions ? e.positions[m.dense + s] : s;
    }
#pragma unroll
    for (int j = 0; j < N; ++j) x[j] = at + j * 64 < end ? claim_of(e, m.seen, w[j], pos[j]) : 0u;
    const uint64_t missing = ballot64((uint32_t)page >= (uint32_t)c.pages);
    const bool last_missing = (uint32_t)last_page >= (uint32_t)c.pages;
    if (missing != 0u || last_missing) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int s = at + j * 64, p = (s >> c.page_shift) - first_page;
            if (s < end && (p < 64 ? missing >> p & 1u : last_missing)) x[j] = s < e.budget ? kStays : kNoToken;
        }
    }
}

// Adds one to the digit's count.  Lanes that agree with the first one are counted at once: many weights are equal (0 above
// all), and a bank adds one after another.
__device__ __forceinline__ void count_digit(uint32_t *counts, uint32_t digit)
{
    const uint32_t first = (uint32_t)__builtin_amdgcn_readfirstlane((int)digit);
    const uint64_t same = ballot64(digit == first);
    if (digit != first) atomicAdd(&counts[digit], 1u);
    else if (prefix_count(same) == 0) atomicAdd(&counts[digit], (uint32_t)__popcll(same));
}

// With counts[kBins] in LDS: the bin of the wanted-th from the top (1-based), and which it is of that bin.
__device__ __forceinline__ void find_bin(const uint32_t *counts, uint32_t (&wave_sum)[16], uint32_t (&found)[2], uint32_t wanted)
{
    const int tid = (int)threadIdx.x, lane = lane_id(), wave = tid >> 6;
    const uint32_t hi = counts[kBins - 1 - 2 * tid], lo = counts[kBins - 2 - 2 * tid];
    uint32_t upto = hi + lo;
    for (int d = 1; d < 64; d *= 2) {
        const uint32_t y = (uint32_t)__shfl_up((int)upto, d);
        if (lane >= d) upto += y;
    }
    if (lane == 63) wave_sum[wave] = upto;
    __syncthreads();
    for (int w = 0; w < wave; ++w) upto += wave_sum[w];
    const uint32_t from = upto - hi - lo;
    if (from < wanted && wanted <= upto) {
        const bool first = wanted <= from + hi;
        found[0] = (uint32_t)(first ? kBins - 1 - 2 * tid : kBins - 2 - 2 * tid);
        found[1] = wanted - (first ? from : from + hi);
    }
    __syncthreads();
}

// Exclusive sum over the workgroup's waves of a number that all lanes of a wave hold; and the sum of all.
__device__ __forceinline__ uint32_t waves_before(uint32_t mine, uint32_t (&wave_sum)[16], uint32_t *all)
{
    const int wave = (int)threadIdx.x >> 6;
    __syncthreads();
    if (lane_id() == 0) wave_sum[wave] = mine;
    __syncthreads();
    uint32_t before = 0u, total = 0u;
    for (int w = 0; w < 16; ++w) {
        if (w < wave) before += wave_sum[w];
        total += wave_sum[w];
    }
    *all = total;
    return before;
}

// The lists of a segment: claims above `claim` are kept, and of those equal to it the first `ties`.  Free slots (those
// below the budget that are not kept) go to `holes`, kept ones behind it to `later`, in order.
template <int N>
__device__ __forceinline__ void list_segment(const KvEvict &e, const uint32_t (&x)[N], int begin, int end, uint32_t claim, uint32_t ties,
                                             int32_t *kept, int32_t *holes, int32_t *later, uint32_t (&wave_sum)[16], uint32_t *all_holes)
{
    const int at = begin + ((int)threadIdx.x >> 6) * (64 * N) + lane_id();
    uint32_t equal = 0u, all;
#pragma unroll
    for (int j = 0; j < N; ++j) equal += (uint32_t)__popcll(ballot64(at + j * 64 < end && x[j] == claim));
    uint32_t eq = waves_before(equal, wave_sum, &all);
    uint32_t stays = 0u, nh = 0u, nl = 0u;  // (bit j: the thread's j-th)
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const int s = at + j * 64;
        const bool same = s < end && x[j] == claim;
        const uint64_t sames = ballot64(same);
        const bool keep = s < end && (x[j] > claim || (same && eq + (uint32_t)prefix_count(sames) < ties));
        eq += (uint32_t)__popcll(sames);
        stays |= keep ? 1u << j : 0u;
        nh += (uint32_t)__popcll(ballot64(s < end && s < e.budget && !keep));
        nl += (uint32_t)__popcll(ballot64(keep && s >= e.budget));
    }
    nh = waves_before(nh, wave_sum, all_holes);
    nl = waves_before(nl, wave_sum, &all);
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const int s = at + j * 64;
        const bool keep = stays >> j & 1u, hole = s < end && s < e.budget && !keep, later_one = keep && s >= e.budget;
        const uint64_t hs = ballot64(hole), ls = ballot64(later_one);
        if (s < end && s < e.budget) kept[s] = keep ? s : -2;  // (a free slot: kv_move_kernel writes what it takes)
        if (hole) holes[nh + (uint32_t)prefix_count(hs)] = s;
        if (later_one) later[nl + (uint32_t)prefix_count(ls)] = s;
        nh += (uint32_t)__popcll(hs);
        nl += (uint32_t)__popcll(ls);
    }
}

// (N = 2 for up to 2048 slots: 6 x 4 memories of 1300 tokens 8 us, with N = 16 17.)
template <int N>
__global__ __launch_bounds__(kEvictThreads) void kv_select_kernel(KvView c, KvEvict e)
{
    const int bh = (int)blockIdx.x, tid = (int)threadIdx.x;
    const Memory m = memory_of(c, e, bh);
    int32_t *kept = e.kept + (int64_t)bh * e.budget;
    if (m.n <= e.budget) {
        for (int s = tid; s < e.budget; s += kEvictThreads) kept[s] = s < m.n ? s : -1;
        if (tid == 0) e.free_slots[bh] = 0u;
        return;
    }
    __shared__ uint32_t counts[kBins], wave_sum[16], found[2];
    uint32_t x[N];
    load_claims(c, e, m, 0, m.n, x);
    const int at = (tid >> 6) * (64 * N) + lane_id();
    uint32_t prefix = 0u, known = 0u, wanted = (uint32_t)e.budget;
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
        const uint32_t digits = pass == 2 ? 1023u : 2047u;
        counts[tid] = counts[tid + kEvictThreads] = 0u;
        __syncthreads();
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (at + j * 64 < m.n && (x[j] & known) == prefix) count_digit(counts, x[j] >> shift & digits);
        __syncthreads();
        find_bin(counts, wave_sum, found, wanted);
        prefix |= found[0] << shift;
        known |= digits << shift;
        wanted = found[1];
        __syncthreads();
    }
    uint32_t all_holes;
    list_segment(e, x, 0, m.n, prefix, wanted, kept, e.holes + (int64_t)bh * e.budget, e.later + (int64_t)bh * e.budget, wave_sum, &all_holes);
    if (tid == 0) e.free_slots[bh] = all_holes;
}

// (8 waves to a SIMD here and in the next, two workgroups to a compute unit: 8 x 8 memories of 131072 tokens cut to 8192 3 % faster)
__global__ __launch_bounds__(kEvictThreads, 8) void kv_count_kernel(KvView c, KvEvict e)
{
    const int bh = (int)blockIdx.y, tid = (int)threadIdx.x;
    const Memory m = memory_of(c, e, bh);
    if (m.n <= e.budget) return;
    const Segment seg = segment_of(e, m.n, (int)blockIdx.x);
    __shared__ uint32_t counts[kBins];
    counts[tid] = counts[tid + kEvictThreads] = 0u;
    __syncthreads();
    if (seg.begin < seg.end) {
        uint32_t x[kSegmentKeys];
        load_claims(c, e, m, seg.begin, seg.end, x);
        const int at = seg.begin + (tid >> 6) * (64 * kSegmentKeys) + lane_id();
#pragma unroll
        for (int j = 0; j < kSegmentKeys; ++j)
            if (at + j * 64 < seg.end) count_digit(counts, x[j] >> 21);
    }
    __syncthreads();
    uint32_t *to = e.counts + ((int64_t)bh * e.segments + blockIdx.x) * kBins;
    to[tid] = counts[tid];
    to[tid + kEvictThreads] = counts[tid + kEvictThreads];
}

__global__ __launch_bounds__(kEvictThreads, 8) void kv_gather_kernel(KvView c, KvEvict e)
{
    const int bh = (int)blockIdx.y, tid = (int)threadIdx.x, seg_no = (int)blockIdx.x;
    const Memory m = memory_of(c, e, bh);
    if (m.n <= e.budget) return;
    const Segment seg = segment_of(e, m.n, seg_no);
    __shared__ uint32_t counts[kBins], wave_sum[16], found[2], before_bin;
    uint32_t x[kSegmentKeys];  // (asked for first: they come while the counts are added up)
    if (seg.begin < seg.end) load_claims(c, e, m, seg.begin, seg.end, x);
    const uint32_t *from = e.counts + (int64_t)bh * e.segments * kBins;
    uint32_t a = 0u, b = 0u;
    for (int s0 = 0; s0 < e.segments; s0 += 8) {  // (eight at a time on their way)
        uint32_t y[8], z[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int64_t at = (int64_t)min(s0 + j, e.segments - 1) * kBins + tid;
            y[j] = from[at];
            z[j] = from[at + kEvictThreads];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            a += s0 + j < e.segments ? y[j] : 0u;
            b += s0 + j < e.segments ? z[j] : 0u;
        }
    }
    counts[tid] = a;
    counts[tid + kEvictThreads] = b;
    __syncthreads();
    find_bin(counts, wave_sum, found, (uint32_t)e.budget);
    const uint32_t bin = found[0];
    // of the segments before this one: claims of that bin; of this one: claims above it
    uint32_t above = 0u, all, before = 0u;
    for (int t = tid; t < kBins; t += kEvictThreads) above += (uint32_t)t > bin ? from[(int64_t)seg_no * kBins + t] : 0u;
    for (int s = tid; s < seg_no; s += kEvictThreads) before += from[(int64_t)s * kBins + bin];
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        above += (uint32_t)__shfl_xor((int)above, d);
        before += (uint32_t)__shfl_xor((int)before, d);
    }
    waves_before(before, wave_sum, &all);
    if (tid == 0) before_bin = all;
    waves_before(above, wave_sum, &all);
    KvSegment *info = e.info + (int64_t)bh * e.segments + seg_no;
    if (tid == 0) {
        info->above = all;
        info->first = before_bin;
        info->count = from[(int64_t)seg_no * kBins + bin];
        if (seg_no == 0) e.chosen[bh] = make_uint2(bin, found[1]);
    }
    if (seg.begin >= seg.end) return;  // (the whole workgroup)
    uint32_t mine = 0u;
    const int at = seg.begin + (tid >> 6) * (64 * kSegmentKeys) + lane_id();
#pragma unroll
    for (int j = 0; j < kSegmentKeys; ++j) mine += (uint32_t)__popcll(ballot64(at + j * 64 < seg.end && x[j] >> 21 == bin));
    uint32_t to = waves_before(mine, wave_sum, &all) + before_bin;
    uint32_t *gathered = e.gathered + m.dense;
#pragma unroll
    for (int j = 0; j < kSegmentKeys; ++j) {
        const bool in = at + j * 64 < seg.end && x[j] >> 21 == bin;
        const uint64_t ins = ballot64(in);
        if (in) gathered[to + (uint32_t)prefix_count(ins)] = x[j];
        to += (uint32_t)__popcll(ins);
    }
}

__global__ __launch_bounds__(kEvictThreads) void kv_pick_kernel(KvView c, KvEvict e)
{
    const int bh = (int)blockIdx.x, tid = (int)threadIdx.x, wave = tid >> 6, lane = lane_id();
    const Memory m = memory_of(c, e, bh);
    if (m.n <= e.budget) return;
    __shared__ uint32_t counts[kBins], wave_sum[16], found[2];
    KvSegment *info = e.info + (int64_t)bh * e.segments;
    const uint32_t *gathered = e.gathered + m.dense;
    const int n = (int)(info[e.segments - 1].first + info[e.segments - 1].count);
    uint32_t prefix = e.chosen[bh].x << 21, known = 2047u << 21, wanted = e.chosen[bh].y;
    for (int pass = 1; pass < 3; ++pass) {
        const int shift = pass == 1 ? 10 : 0;
        const uint32_t digits = pass == 2 ? 1023u : 2047u;
        counts[tid] = counts[tid + kEvictThreads] = 0u;
        __syncthreads();
        for (int s0 = 0; s0 < n; s0 += 8 * kEvictThreads) {
            uint32_t x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = gathered[min(n - 1, s0 + j * kEvictThreads + tid)];
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (s0 + j * kEvictThreads + tid < n && (x[j] & known) == prefix) count_digit(counts, x[j] >> shift & digits);
        }
        __syncthreads();
        find_bin(counts, wave_sum, found, wanted);
        prefix |= found[0] << shift;
        known |= digits << shift;
        wanted = found[1];
        __syncthreads();
    }
    // per segment the gathered claims above and equal to it (a wave to a segment)
    for (int s = wave; s < e.segments; s += 16) {
        const int begin = (int)info[s].first, end = begin + (int)info[s].count;
        uint32_t above = 0u, equal = 0u;
        for (int t = begin + lane; t - lane < end; t += 64) {
            const uint32_t x = t < end ? gathered[t] : 0u;
            above += (uint32_t)__popcll(ballot64(t < end && x > prefix));
            equal += (uint32_t)__popcll(ballot64(t < end && x == prefix));
        }
        if (lane == 0) {
            info[s].above += above;
            info[s].count = equal;
        }
    }
    __syncthreads();
    if (tid > 0) return;
    uint32_t holes = 0u, later = 0u, left = wanted;
    for (int s = 0; s < e.segments; ++s) {
        const Segment seg = segment_of(e, m.n, s);
        const uint32_t ties = min(left, info[s].count), stays = info[s].above + ties;
        left -= ties;
        info[s].ties = ties;
        info[s].first = seg.below ? holes : later;
        if (seg.below) holes += (uint32_t)(seg.end - seg.begin) - stays;
        else later += stays;
    }
    e.chosen[bh].x = prefix;
    e.free_slots[bh] = holes;
}

__global__ __launch_bounds__(kEvictThreads) void kv_list_kernel(KvView c, KvEvict e)
{
    const int bh = (int)blockIdx.y, tid = (int)threadIdx.x;
    const Memory m = memory_of(c, e, bh);
    int32_t *kept = e.kept + (int64_t)bh * e.budget;
    if (m.n <= e.budget) {
        for (int64_t s = (int64_t)blockIdx.x * kEvictThreads + tid; s < e.budget; s += (int64_t)gridDim.x * kEvictThreads) kept[s] = s < m.n ? (int)s : -1;
        if (blockIdx.x == 0 && tid == 0) e.free_slots[bh] = 0u;
        return;
    }
    const Segment seg = segment_of(e, m.n, (int)blockIdx.x);
    if (seg.begin >= seg.end) return;
    __shared__ uint32_t wave_sum[16];
    const KvSegment info = e.info[(int64_t)bh * e.segments + blockIdx.x];
    uint32_t x[kSegmentKeys], all;
    load_claims(c, e, m, seg.begin, seg.end, x);
    const int64_t first = (int64_t)bh * e.budget + info.first;
    const uint32_t claim = e.chosen[bh].x;
    if (info.ties != 0u && info.ties != info.count) {
        list_segment(e, x, seg.begin, seg.end, claim, info.ties, kept, e.holes + first, e.later + first, wave_sum, &all);
        return;
    }
    // none or all of the equal ones: a comparison decides, and the slots lie on one side of the budget
    const int at = seg.begin + (tid >> 6) * (64 * kSegmentKeys) + lane_id();
    const auto stays = [&](int j) { return x[j] > claim || (info.ties != 0u && x[j] == claim); };
    uint32_t mine = 0u;
#pragma unroll
    for (int j = 0; j < kSegmentKeys; ++j) mine += (uint32_t)__popcll(ballot64(at + j * 64 < seg.end && stays(j) != seg.below));
    uint32_t to = waves_before(mine, wave_sum, &all);
    int32_t *list = (seg.below ? e.holes : e.later) + first;
#pragma unroll
    for (int j = 0; j < kSegmentKeys; ++j) {
        const bool in = at + j * 64 < seg.end, keep = stays(j), listed = in && keep != seg.below;
        const uint64_t those = ballot64(listed);
        if (listed) list[to + (uint32_t)prefix_count(those)] = at + j * 64;
        if (in && seg.below) kept[at + j * 64] = keep ? at + j * 64 : -2;
        to += (uint32_t)__popcll(those);
    }
}

// D / 32 lanes to a slot below the budget that stays as it is (its position and weight), and to a free one and the token that
// it takes: position, weight, codes.  Sources lie at and behind the budget, targets below it: no order is needed.  Bound by
// the sectors of memory that scattered rows of D / 2 and D / 32 bytes touch (504 thousand tokens of 136 bytes in 45 us); two or
// four tokens to a lane, to have more on the way: 47 and 60.
template <int D>
__global__ __launch_bounds__(256) void kv_move_kernel(KvView c, KvEvict e)
{
    constexpr int L = D / 32;  // 16 bytes of the key's codes to a lane, then of the value's
    const int64_t item = ((int64_t)blockIdx.x * 256 + threadIdx.x) / L;
    const int part = (int)threadIdx.x % L;
    if (item >= (int64_t)c.batch * c.heads * e.budget) return;
    const int bh = (int)(item / e.budget), i = (int)(item % e.budget), b = bh / c.heads, head = bh % c.heads;
    const int64_t stride = (int64_t)c.width << c.page_shift, dense = bh * stride, out = bh * e.out_stride;
    int from = -1, to = 0;
    if ((uint32_t)i < e.free_slots[bh]) {
        from = e.later[item];
        to = e.holes[item];
    }
    if (part == 0) {
        const int same = e.kept[item];  // i: stays; -1: past the length; otherwise free
        if (same == i || same == -1) {
            if (e.positions_out) e.positions_out[out + i] = same < 0 ? -1 : e.positions ? e.positions[dense + i] : i;
            e.weights_out[out + i] = same < 0 ? 0.f : e.weights[dense + i];
        }
        if (from >= 0) {
            if (e.positions_out) e.positions_out[out + to] = e.positions ? e.positions[dense + from] : from;
            e.weights_out[out + to] = e.weights[dense + from];
            e.kept[(int64_t)bh * e.budget + to] = from;  // whoever reads it before or after: not its own number, not -1
        }
        if (i == 0 && head == 0)  // the one thread that reads this length: it may be the same array
            e.lengths_out[b] = (int32_t)max((int64_t)0, min(min((int64_t)c.lengths[b], stride), (int64_t)e.budget));
    }
    if (from < 0) return;
    const int p0 = page_of(c, b, from), p1 = page_of(c, b, to);
    if (p0 < 0 || p1 < 0) return;
    const int in_page = (1 << c.page_shift) - 1;
    const int64_t src = (((int64_t)p0 * c.heads + head) << c.page_shift) + (from & in_page);
    const int64_t dst = (((int64_t)p1 * c.heads + head) << c.page_shift) + (to & in_page);
    const u32x4 k = *(const u32x4 *)(c.k_codes + src * (D / 2) + part * 16), v = *(const u32x4 *)(c.v_codes + src * (D / 2) + part * 16);
    const uint8_t ks = c.k_scales[src * L + part], vs = c.v_scales[src * L + part];
    *(u32x4 *)(c.k_codes + dst * (D / 2) + part * 16) = k;
    *(u32x4 *)(c.v_codes + dst * (D / 2) + part * 16) = v;
    c.k_scales[dst * L + part] = ks;
    c.v_scales[dst * L + part] = vs;
}

template <int DT, int D>
int run_append(const KvView &c, const KvRows &r, hipStream_t s)
{
    const int64_t blocks = ((int64_t)r.nrows * c.heads * (D / 8) + 255) / 256;
    kv_append_kernel<DT, D><<<(uint32_t)blocks, 256, 0, s>>>(c, r);
    PSC_HIP_TRY(hipGetLastError());
    return PSC_OK;
}
template <int DT, int D>
int run_read(const KvView &c, const KvRows &r, void *k, void *v, hipStream_t s)
{
    const int64_t blocks = ((int64_t)r.nrows * c.heads * (D / 8) + 255) / 256;
    kv_read_kernel<DT, D><<<(uint32_t)blocks, 256, 0, s>>>(c, r, k, v);
    PSC_HIP_TRY(hipGetLastError());
    return PSC_OK;
}

// Blocks of a part at least, and blocks of a memory up to which a unit stays whole (128 rows over 1500 tokens, 47 blocks:
// 28 us in parts, 20 whole; one row over 16000 tokens: 23.5 us with parts of 8 blocks or more, 21.0 with 16, 21.6 with 24).
constexpr int64_t kLeastBlocks = 16, kFewBlocks = 64;

// Rows of a wave, in sixteens, at most.
template <int DT, int D>
constexpr int most_row_tiles()
{
    return DT == PSC_F32 || D == 256 ? 1 : 2;
}

// Sixteens of tokens of a workgroup that shares out rows for the weights: as many as leave room for two waves' registers.
constexpr int split_tiles(int dim) { return dim == 256 ? 2 : 4; }

template <int DT, int D>
int run_attention(const KvView &c, const KvQueries &q, const KvPlan &p, const float *given, float *received, hipStream_t s)
{
    constexpr int kMost = most_row_tiles<DT, D>();
    if (q.nrows > 0) {
        const uint32_t groups = (uint32_t)(c.batch * c.heads);
        const auto launch = [&](auto rt, auto pos) {
            if (p.workgroups) kv_attention_kernel<D, DT, rt.value, pos.value, true><<<(uint32_t)p.most_parts, 256, 0, s>>>(c, q);
            else kv_attention_kernel<D, DT, rt.value, pos.value, false><<<dim3((uint32_t)p.row_groups, 1, groups), 256, 0, s>>>(c, q);
        };
        const auto launch_rows = [&](auto pos) {
            if (p.row_tiles == 1) launch(std::integral_constant<int, 1>(), pos);
            else launch(std::integral_constant<int, kMost>(), pos);
        };
        if (q.positions) launch_rows(std::true_type());
        else launch_rows(std::false_type());
        PSC_HIP_TRY(hipGetLastError());
        if (p.workgroups) {
            kv_join_kernel<D, DT><<<(uint32_t)(((int64_t)q.nrows * q.q_heads + 3) / 4), 256, 0, s>>>(c, q);
            PSC_HIP_TRY(hipGetLastError());
        }
    }
    if (received) {
        const dim3 grid((uint32_t)p.weights_groups, 1, (uint32_t)(c.batch * c.heads));
        if (p.scores_rows > 0) {
            if (p.scores_rows == 1) kv_weights_of_scores_kernel<1><<<grid, 256, 0, s>>>(c, q, given, received);
            else if (p.scores_rows <= 4) kv_weights_of_scores_kernel<4><<<grid, 256, 0, s>>>(c, q, given, received);
            else kv_weights_of_scores_kernel<kScoreRows><<<grid, 256, 0, s>>>(c, q, given, received);
        } else if (p.split_rows) {
            kv_weights_kernel<D, DT, true, split_tiles(D)><<<grid, 256, 0, s>>>(c, q, given, received);
        } else {
            kv_weights_kernel<D, DT, false, 2><<<grid, 256, 0, s>>>(c, q, given, received);
        }
        PSC_HIP_TRY(hipGetLastError());
    }
    return PSC_OK;
}

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

}  // namespace

int launch_kv_append(const KvView &c, int dtype, const KvRows &r, hipStream_t s)
{
    return PSC_KV_DISPATCH(run_append, dtype, c.dim, c, r, s);
}

int launch_kv_read(const KvView &c, int dtype, const KvRows &r, void *k_out, void *v_out, hipStream_t s)
{
    return PSC_KV_DISPATCH(run_read, dtype, c.dim, c, r, k_out, v_out, s);
}

KvPlan plan_kv_attention(const KvView &c, int dtype, int group, int64_t nrows, int max_rows, int window, int sinks, bool ordered, bool weights)
{
    KvPlan p;
    const int64_t m = (int64_t)max_rows * group, rows = nrows * group * c.heads, slots = (int64_t)c.width << c.page_shift;
    p.row_tiles = m <= 16 || dtype == PSC_F32 || c.dim == 256 ? 1 : 2;
    p.row_groups = (m + 16 * p.row_tiles - 1) / (16 * p.row_tiles);
    // blocks of 32 tokens that a group of rows can see at most
    int64_t blocks = (slots + 31) / 32;
    if (ordered && window > 0) blocks = std::min(blocks, ((int64_t)window + 16 * p.row_tiles / group + 1) / 32 + 2 + ((int64_t)sinks + 31) / 32);
    const int64_t units = p.row_groups * c.batch * c.heads;
    // workgroups to a compute unit that attention_waves leaves registers for (of 64 coordinates with 32 rows or float32 the
    // compiler makes kernels small enough for three; two are counted)
    const int waves = dtype == PSC_F32 ? (c.dim == 256 ? 1 : 2) : c.dim == 256 || p.row_tiles == 2 ? 2 : c.dim == 64 ? 4 : 3;
    // As many units as that, or memories of a few blocks to a wave: parts and their join would cost more than they save.
    if (units > 0 && units < 256 * waves && blocks > kFewBlocks && units * blocks < (int64_t)1 << 31)
        p.workgroups = 256 * waves;
    if (p.workgroups) {
        // at most one part more to a unit than `wanted` of Parts, which is half of the workgroups or more
        p.most_parts = std::min(p.workgroups + units, units * ((blocks + kLeastBlocks - 1) / kLeastBlocks));
        p.part_stat_bytes = (size_t)(p.most_parts * 16 * p.row_tiles * 8 + 255) / 256 * 256;
        p.part_acc_bytes = (size_t)(p.most_parts * 16 * p.row_tiles * c.dim * 4 + 255) / 256 * 256;
    }
    p.least_blocks = kLeastBlocks;
    const int64_t scores_bytes = (int64_t)c.batch * c.heads * m * slots * 4;
    const bool keep_scores = weights && nrows > 0 && m <= kScoreRows && scores_bytes <= kMostScoreBytes;
    p.split_rows = m > 64;
    const int64_t tokens = keep_scores ? 1024 : p.split_rows ? 16 * split_tiles(c.dim) : 128;
    p.weights_groups = weights ? (slots + tokens - 1) / tokens : 0;
    p.stat_bytes = weights ? (size_t)(rows * 8 + 255) / 256 * 256 : 0;
    if (keep_scores) {
        p.scores_rows = (int)m;
        p.scores_bytes = (size_t)(scores_bytes + 255) / 256 * 256;
    }
    return p;
}

int launch_kv_attention(const KvView &c, int dtype, const KvQueries &q, const KvPlan &p, const float *given, float *received, hipStream_t s)
{
    return PSC_KV_DISPATCH(run_attention, dtype, c.dim, c, q, p, given, received, s);
}

KvEvictPlan plan_kv_evict(const KvView &c, int budget)
{
    KvEvictPlan p;
    const int64_t slots = (int64_t)c.width << c.page_shift, bh = (int64_t)c.batch * c.heads;
    const auto up = [](size_t bytes) { return (bytes + 255) / 256 * 256; };
    p.segments = 1;
    if (slots > kSegment) {
        p.segments_below = (std::min<int64_t>(budget, slots) + kSegment - 1) / kSegment;
        p.segments = p.segments_below + (std::max<int64_t>(0, slots - budget) + kSegment - 1) / kSegment;
        p.counts_bytes = up((size_t)(bh * p.segments * kBins * 4));
        p.info_bytes = up((size_t)(bh * p.segments * sizeof(KvSegment)));
        p.gathered_bytes = up((size_t)(bh * slots * 4));
    }
    p.list_bytes = up((size_t)(bh * budget * 4));
    p.head_bytes = up((size_t)(bh * 12));
    return p;
}

int launch_kv_evict(const KvView &c, KvEvict e, const KvEvictPlan &p, char *ws, hipStream_t s)
{
    const uint32_t bh = (uint32_t)(c.batch * c.heads);
    e.chosen = (uint2 *)ws;
    e.free_slots = (uint32_t *)(e.chosen + bh);
    ws += p.head_bytes;
    e.holes = (int32_t *)ws;
    e.later = (int32_t *)(ws + p.list_bytes);
    ws += 2 * p.list_bytes;
    e.segments = (int)p.segments;
    e.segments_below = (int)p.segments_below;
    if (p.counts_bytes == 0) {
        if ((int64_t)c.width << c.page_shift <= 2 * kEvictThreads) kv_select_kernel<2><<<bh, kEvictThreads, 0, s>>>(c, e);
        else kv_select_kernel<kSegmentKeys><<<bh, kEvictThreads, 0, s>>>(c, e);
    } else {
        e.info = (KvSegment *)ws;
        e.counts = (uint32_t *)(ws + p.info_bytes);
        e.gathered = (uint32_t *)(ws + p.info_bytes + p.counts_bytes);
        const dim3 grid((uint32_t)p.segments, bh);
        kv_count_kernel<<<grid, kEvictThreads, 0, s>>>(c, e);
        PSC_HIP_TRY(hipGetLastError());
        kv_gather_kernel<<<grid, kEvictThreads, 0, s>>>(c, e);
        PSC_HIP_TRY(hipGetLastError());
        kv_pick_kernel<<<bh, kEvictThreads, 0, s>>>(c, e);
        PSC_HIP_TRY(hipGetLastError());
        kv_list_kernel<<<grid, kEvictThreads, 0, s>>>(c, e);
    }
    PSC_HIP_TRY(hipGetLastError());
    const int64_t lanes = (int64_t)bh * e.budget * (c.dim / 32);
    const uint32_t blocks = (uint32_t)((lanes + 255) / 256);
    if (c.dim == 64) kv_move_kernel<64><<<blocks, 256, 0, s>>>(c, e);
    else if (c.dim == 128) kv_move_kernel<128><<<blocks, 256, 0, s>>>(c, e);
    else kv_move_kernel<256><<<blocks, 256, 0, s>>>(c, e);
    PSC_HIP_TRY(hipGetLastError());
    return PSC_OK;
}

}  // namespace psc
