// Rotary positions: pairs (a, b) of a head's first `dims` coordinates turned by an angle that grows with the row's position,
//   a' = f (a cos t - b sin t)   b' = f (b cos t + a sin t)   t = position * frequency of the pair
// alone (the transposed, which is the gradient, turns by -t), and for keys on their way into the memory in 4 bits.
//
// Angles.  A frequency is held as the share of a turn that a position adds, in 64 bits: position * frequency modulo 2^64 is then
// the angle without its whole turns, exactly, in one integer product, however far the position.  What is left of a
// quarter turn after the nearest quarters are taken off goes into Taylor's series in 64 bits (|t| <= pi/4: sine to t^15, off by
// 5e-17, cosine to t^16, off by 2e-18).  64-bit operations issue at the rate of single 32-bit ones here, and a thread uses its sines and
// cosines for several heads.
//
// Bound by HBM: 16384 rows of 32 heads x 128 bfloat16 in 54 us, 5.0 TB/s (67 with rows, not heads, beside each other in a wave); 27 thousand rows
// of 32 query heads and 8 kv heads x 128 float16 into the memory in 121 us, 5.0 TB/s (when it took 133, 159 without the loads ahead).  Dimensions
// or places that the wide kernel does not take: two-byte accesses, 24 of 96 coordinates of 16384 rows x 32 heads bfloat16 in 80 us, 2.5 TB/s.
#include "kv_device.h"

namespace psc {
namespace {

__device__ __forceinline__ void sincos_of_turns(uint64_t turns, double *sine, double *cosine)
{
    const uint64_t quarters = ((turns >> 61) + 1) >> 1;
    const double t = (double)(int64_t)(turns - (quarters << 62)) * (0x1.921fb54442d18p+2 * 0x1p-64), tt = t * t;
    double s = -1.0 / 1307674368000.0, c = 1.0 / 20922789888000.0;
    s = __builtin_fma(s, tt, 1.0 / 6227020800.0);
    s = __builtin_fma(s, tt, -1.0 / 39916800.0);
    s = __builtin_fma(s, tt, 1.0 / 362880.0);
    s = __builtin_fma(s, tt, -1.0 / 5040.0);
    s = __builtin_fma(s, tt, 1.0 / 120.0);
    s = __builtin_fma(s, tt, -1.0 / 6.0);
    s = __builtin_fma(s * tt, t, t);
    c = __builtin_fma(c, tt, -1.0 / 87178291200.0);
    c = __builtin_fma(c, tt, 1.0 / 479001600.0);
    c = __builtin_fma(c, tt, -1.0 / 3628800.0);
    c = __builtin_fma(c, tt, 1.0 / 40320.0);
    c = __builtin_fma(c, tt, -1.0 / 720.0);
    c = __builtin_fma(c, tt, 1.0 / 24.0);
    c = __builtin_fma(c, tt, -0.5);
    c = __builtin_fma(c, tt, 1.0);
    const double s0 = quarters & 1 ? c : s, c0 = quarters & 1 ? s : c;
    *sine = quarters & 2 ? -s0 : s0;
    *cosine = (quarters + 1) & 2 ? -c0 : c0;
}

// Sine and cosine of a pair times the factor.
__device__ __forceinline__ void turn_of(const Rotary &t, int pair, int64_t position, double *sine, double *cosine)
{
    sincos_of_turns((uint64_t)position * t.turns[pair], sine, cosine);
    *sine *= t.factor;
    *cosine *= t.factor;
}

// What is copied -- coordinates behind the turned ones, rows that nobody has -- keeps its bits: turned by nothing, an infinity or a NaN would
// make its partner NaN, and -0 could become 0.
template <int DT>
struct RawRow {  // 8 coordinates as they lie in memory
    static constexpr int kWords = DT == PSC_F32 ? 8 : 4;
    u32x4 w[kWords / 4];  // (arrays of words that are copied as bytes go to LDS)
    __device__ __forceinline__ void load(const void *p)
    {
#pragma unroll
        for (int i = 0; i < kWords / 4; ++i) w[i] = ((const u32x4 *)p)[i];
    }
    __device__ __forceinline__ void store(void *p) const
    {
#pragma unroll
        for (int i = 0; i < kWords / 4; ++i) ((u32x4 *)p)[i] = w[i];
    }
    __device__ __forceinline__ void get(float (&x)[8]) const
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (DT == PSC_F32) x[i] = __uint_as_float(w[i / 4][i % 4]);
            else x[i] = Element<DT>::load((uint16_t)(i & 1 ? w[0][i / 2] >> 16 : w[0][i / 2]));
        }
    }
    // x, or what was given: of all coordinates.
    __device__ __forceinline__ void choose(bool given, const float (&x)[8])
    {
#pragma unroll
        for (int i = 0; i < kWords; ++i) {
            uint32_t made;
            if constexpr (DT == PSC_F32) made = __float_as_uint(x[i]);
            else made = (uint32_t)Element<DT>::store(x[2 * i]) | (uint32_t)Element<DT>::store(x[2 * i + 1]) << 16;
            w[i / 4][i % 4] = given ? w[i / 4][i % 4] : made;
        }
    }
};

// ------------------------------------------------------------------------------------------- rows on their own
// A thread takes 8 pairs (or 16 coordinates that are copied) of a row, in every `slots`-th head: threads beside it take
// the row's other pairs, then the heads beside it, so that a wave reads and writes in one piece.
template <int DT, bool kInterleaved>
__global__ __launch_bounds__(256) void rotary_kernel(Rotary t, RotaryRows r)
{
    typedef typename Element<DT>::type T;
    const int turned = t.dims / 16, chunks = turned + (r.head_dim - t.dims + 15) / 16;
    const int64_t item = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int chunk = (int)(item % chunks);
    const int64_t rest = item / chunks;
    const int from = (int)(rest % r.slots), row = (int)(rest / r.slots);
    if (row >= r.nrows) return;
    const T *x = (const T *)r.x + row * r.row_stride;
    T *y = (T *)r.out + row * r.out_row_stride;
    int64_t position = 0;
    bool copied = chunk >= turned;
    const int at0 = copied ? t.dims + (chunk - turned) * 16 : kInterleaved ? chunk * 16 : chunk * 8, at1 = copied || kInterleaved ? at0 + 8 : at0 + t.dims / 2;
    if (!copied) position = r.position_of(row, &copied);
    if (copied) {
        const bool second = at1 < r.head_dim;
        for (int h = from; h < r.heads; h += r.slots) {
            RawRow<DT> a, b;
            a.load(x + h * r.head_stride + at0);
            b.load(x + h * r.head_stride + (second ? at1 : at0));
            a.store(y + h * r.out_head_stride + at0);
            if (second) b.store(y + h * r.out_head_stride + at1);
        }
        return;
    }
    float s[8], c[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        double sine, cosine;
        turn_of(t, chunk * 8 + i, position, &sine, &cosine);
        s[i] = r.transposed ? -(float)sine : (float)sine;
        c[i] = (float)cosine;
    }
#pragma unroll 4
    for (int h = from; h < r.heads; h += r.slots) {
        float u[8], v[8], p[8], q[8];
        load_row<DT, 8>(x + h * r.head_stride + at0, u);
        load_row<DT, 8>(x + h * r.head_stride + at1, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (kInterleaved) {
                const float a = i < 4 ? u[2 * i] : v[2 * i - 8], b = i < 4 ? u[2 * i + 1] : v[2 * i - 7];
                (i < 4 ? p[2 * i] : q[2 * i - 8]) = a * c[i] - b * s[i];
                (i < 4 ? p[2 * i + 1] : q[2 * i - 7]) = b * c[i] + a * s[i];
            } else {
                p[i] = u[i] * c[i] - v[i] * s[i];
                q[i] = v[i] * c[i] + u[i] * s[i];
            }
        }
        store_row<DT, 8>(y + h * r.out_head_stride + at0, p);
        store_row<DT, 8>(y + h * r.out_head_stride + at1, q);
    }
}

// Any number of dimensions, strides and alignment: a thread takes a pair, or a coordinate that is copied.
template <int DT>
__global__ __launch_bounds__(256) void rotary_single_kernel(Rotary t, RotaryRows r)
{
    typedef typename Element<DT>::type T;
    const int half = t.dims / 2, places = half + r.head_dim - t.dims;
    const int64_t item = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int place = (int)(item % places);
    const int64_t rest = item / places;
    const int from = (int)(rest % r.slots), row = (int)(rest / r.slots);
    if (row >= r.nrows) return;
    const T *x = (const T *)r.x + row * r.row_stride;
    T *y = (T *)r.out + row * r.out_row_stride;
    if (place >= half) {
        const int at = half + place;
        for (int h = from; h < r.heads; h += r.slots) y[h * r.out_head_stride + at] = x[h * r.head_stride + at];
        return;
    }
    const int at0 = t.interleaved ? 2 * place : place, at1 = t.interleaved ? at0 + 1 : at0 + half;
    bool nobodys;
    const int64_t position = r.position_of(row, &nobodys);
    if (nobodys) {
        for (int h = from; h < r.heads; h += r.slots) {
            const T a = x[h * r.head_stride + at0], b = x[h * r.head_stride + at1];
            y[h * r.out_head_stride + at0] = a;
            y[h * r.out_head_stride + at1] = b;
        }
        return;
    }
    double sine, cosine;
    turn_of(t, place, position, &sine, &cosine);
    const float s = r.transposed ? -(float)sine : (float)sine, c = (float)cosine;
#pragma unroll 4
    for (int h = from; h < r.heads; h += r.slots) {
        const float a = Element<DT>::load(x[h * r.head_stride + at0]), b = Element<DT>::load(x[h * r.head_stride + at1]);
        y[h * r.out_head_stride + at0] = Element<DT>::store(a * c - b * s);
        y[h * r.out_head_stride + at1] = Element<DT>::store(b * c + a * s);
    }
}

// ------------------------------------------------------------------------------------------- into the memory
// D / 8 lanes to a row, 8 coordinates to a lane.  First the keys, which are turned, rounded and written with their values: lanes beside each
// other have rows that follow each other, whose codes lie side by side, in a group of the kv heads.  Then the queries, in every `slots`-th
// head: lanes beside each other have heads beside each other.  A key's products are made in 64 bits and rounded to 32, then to 4: a
// coordinate next to a border between two codes comes out on the same side as in any other exact computation.
//
// The way from load to load -- offsets, first, lengths, table -- is long beside the work of a lane, so the first head's coordinates are asked
// for before it, and the next head's before a head is worked on.
template <int DT, int D, bool kInterleaved>
__global__ __launch_bounds__(256) void kv_append_rotary_kernel(KvView c, KvRows r, Rotary t, RotaryQueries q)
{
    constexpr int L = D / 8;
    typedef typename Element<DT>::type T;
    const int64_t item = ((int64_t)blockIdx.x * 256 + threadIdx.x) / L;
    const int part = (int)(threadIdx.x % L);
    const bool keys = item < q.key_items;
    const int64_t query = item - q.key_items;
    const int row = (int)(keys ? item % r.nrows : q.slots ? query / q.slots : r.nrows), from = (int)(keys ? item / r.nrows * q.key_group : q.slots ? query % q.slots : 0);
    if (row >= r.nrows) return;
    // the lane's pairs; of pairs half of `dims` apart it has one side, and reads the other side too
    constexpr int kPairs = kInterleaved ? 4 : 8;
    const int at = part * 8, half = t.dims / 2;
    const bool turned = at < t.dims, second = !kInterleaved && at >= half;
    const int other = kInterleaved || !turned ? at : second ? at - half : at + half;

    const T *k = (const T *)r.k + row * r.k_stride, *v = (const T *)r.v + row * r.v_stride, *from_q = (const T *)q.q + row * q.row_stride;
    const int to = keys ? min(from + q.key_group, c.heads) : q.heads;
    RawRow<DT> mine, side, value;
    const auto load = [&](int h) {
        const T *p = keys ? k + h * r.k_head_stride : from_q + h * q.head_stride;
        mine.load(p + at);
        if (!kInterleaved) side.load(p + other);
        if (keys) value.load(v + h * r.v_head_stride + at);
    };
    if (from < to) load(from);

    const RowPlace p = place_of(c, r, row);
    const bool nobodys = p.place < 0 || (r.offsets && row >= r.offsets[c.batch]);
    const int64_t position = (int64_t)(r.first ? r.first[p.b] : c.lengths[p.b]) + p.place;
    double s[kPairs], co[kPairs];
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
        s[i] = 0.0;
        co[i] = 1.0;
    }
    if (turned) {
#pragma unroll
        for (int i = 0; i < kPairs; ++i) {
            turn_of(t, kInterleaved ? part * 4 + i : second ? other + i : at + i, position, &s[i], &co[i]);
            if (!kInterleaved && !second) s[i] = -s[i];  // (then x cos + other sin on both sides)
        }
    }
    if (keys) {
        for (int h = from; h < to; ++h) {
            float x[2][8], o[8];
            mine.get(x[0]);
            value.get(x[1]);
            side.get(o);
            if (h + 1 < to) load(h + 1);
            // (coordinates behind the turned ones keep their bits: a product with 1 would make a signalling NaN a quiet one)
            if constexpr (kInterleaved) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const double a = x[0][2 * i], b = x[0][2 * i + 1];
                    const float u = (float)__builtin_fma(a, co[i], -(b * s[i])), w = (float)__builtin_fma(b, co[i], a * s[i]);
                    x[0][2 * i] = turned ? u : x[0][2 * i];
                    x[0][2 * i + 1] = turned ? w : x[0][2 * i + 1];
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float u = (float)__builtin_fma((double)x[0][i], co[i], (double)o[i] * s[i]);
                    x[0][i] = turned ? u : x[0][i];
                }
            }
            write_token<D>(c, r, p, h, part, x);
        }
        return;
    }
    const bool copied = !turned || nobodys;
    float sf[kPairs], cf[kPairs];
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
        sf[i] = (float)s[i];
        cf[i] = (float)co[i];
    }
#pragma unroll 2
    for (int h = from; h < to; h += q.slots) {
        float x[8], o[8];
        RawRow<DT> out = mine;
        mine.get(x);
        side.get(o);
        if (h + q.slots < to) load(h + q.slots);
        if constexpr (kInterleaved) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float a = x[2 * i], b = x[2 * i + 1];
                x[2 * i] = a * cf[i] - b * sf[i];
                x[2 * i + 1] = b * cf[i] + a * sf[i];
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = x[i] * cf[i] + o[i] * sf[i];
        }
        out.choose(copied, x);
        out.store((T *)q.out + ((int64_t)row * q.heads + h) * D + at);
    }
}

// Threads to a row's place: a thread takes so many heads that enough threads are left to fill the card, 8 at most.
constexpr int64_t kThreads = (int64_t)256 * 2048;
int group_of(int64_t threads_of_a_head, int heads)
{
    int group = 1;
    while (group < 8 && group < heads && threads_of_a_head * heads / (2 * group) >= kThreads) group *= 2;
    return group;
}
int slots_of(int64_t threads_of_a_head, int heads)
{
    const int group = group_of(threads_of_a_head, heads);
    int slots = 1;  // (a power of two: so many heads lie beside each other in a wave)
    while (slots * group < heads) slots *= 2;
    return slots;
}

template <int DT>
int run_rotary(const Rotary &t, RotaryRows r, bool wide, hipStream_t s)
{
    const int64_t places = wide ? t.dims / 16 + (r.head_dim - t.dims + 15) / 16 : t.dims / 2 + r.head_dim - t.dims;
    r.slots = slots_of(places * r.nrows, r.heads);
    const int64_t blocks = (places * r.nrows * r.slots + 255) / 256;
    if (!wide) rotary_single_kernel<DT><<<(uint32_t)blocks, 256, 0, s>>>(t, r);
    else if (t.interleaved) rotary_kernel<DT, true><<<(uint32_t)blocks, 256, 0, s>>>(t, r);
    else rotary_kernel<DT, false><<<(uint32_t)blocks, 256, 0, s>>>(t, r);
    PSC_HIP_TRY(hipGetLastError());
    return PSC_OK;
}

template <int DT, int D>
int run_append_rotary(const KvView &c, const KvRows &r, const Rotary &t, RotaryQueries q, hipStream_t s)
{
    const int64_t threads = (int64_t)r.nrows * (D / 8);
    q.key_group = group_of(threads, c.heads);
    q.key_items = (int64_t)r.nrows * ((c.heads + q.key_group - 1) / q.key_group);
    q.slots = q.heads ? slots_of(threads, q.heads) : 0;
    const int64_t blocks = ((q.key_items + (int64_t)r.nrows * q.slots) * (D / 8) + 255) / 256;
    if (t.interleaved) kv_append_rotary_kernel<DT, D, true><<<(uint32_t)blocks, 256, 0, s>>>(c, r, t, q);
    else kv_append_rotary_kernel<DT, D, false><<<(uint32_t)blocks, 256, 0, s>>>(c, r, t, q);
    PSC_HIP_TRY(hipGetLastError());
    return PSC_OK;
}

}  // namespace

int launch_rotary(const Rotary &t, int dtype, const RotaryRows &r, bool wide, hipStream_t s)
{
    return dtype == PSC_BF16 ? run_rotary<PSC_BF16>(t, r, wide, s) : dtype == PSC_F16 ? run_rotary<PSC_F16>(t, r, wide, s) : run_rotary<PSC_F32>(t, r, wide, s);
}

int launch_kv_append_rotary(const KvView &c, int dtype, const KvRows &r, const Rotary &t, const RotaryQueries &q, hipStream_t s)
{
    return PSC_KV_DISPATCH(run_append_rotary, dtype, c.dim, c, r, t, q, s);
}

}  // namespace psc
