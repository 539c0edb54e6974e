// Norms before and after a block, with the block's gate and the residual scale, and their gradients:
//   u = rms(y) * after * act(gate)      rms(t) = t / sqrt(mean t^2 + eps)
//   h = residual_scale x + block_scale u      z = rms(h) * before
// A row lies in the registers of `lanes` lanes, 8 consecutive coordinates (or twice 8) to each: 8 to 64 lanes of a wave for narrow rows,
// a workgroup for wide ones.  Each input is read once and each output written once; everything between is 32-bit floats.
// Bound by HBM: 16384 x 4096 bfloat16 with a gate, forward 139 us, backward 226 to 235 (4.6 to 4.8 TB/s).  A few rows: the start and the way through
// the instructions (6 rows 4.5 and 9.5 us).  Rows wider than 8192 have 1024 lanes and so 128 registers each, which do not do for the backward pass:
// 316 to 492 bytes of a lane lie in scratch (forward 68 to 140), and weights are read again for every row.  4096 x 12288 and x 16384, forward
// 126 and 143 us (4.0 and 4.7 TB/s), backward 591 and 649 (1.4 and 1.7), where 4096 x 8192 takes 74 and 136.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "common.h"
#include "entry.h"

namespace psc {
namespace {

template <int DT>
struct Stored;
template <>
struct Stored<PSC_BF16> {
    typedef uint16_t type;
    static __device__ float load(type x) { return __uint_as_float((uint32_t)x << 16); }
    static __device__ type store(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }
};
template <>
struct Stored<PSC_F16> {
    typedef uint16_t type;
    static __device__ float load(type x) { return (float)__builtin_bit_cast(_Float16, x); }
    static __device__ type store(float x) { return __builtin_bit_cast(uint16_t, (_Float16)x); }
};
template <>
struct Stored<PSC_F32> {
    typedef float type;
    static __device__ float load(type x) { return x; }
    static __device__ type store(float x) { return x; }
};

// 8 coordinates as they lie in memory; `n` of them are there: 8 or none, and fewer at the end of a row whose width is no multiple of 8
// (`tail`).  Rows of odd widths begin anywhere: global loads of 16 bytes need no alignment.
template <int DT>
struct Eight {  // (words, two coordinates to each: as 16-bit elements the compiler gives each a register of its own)
    uint32_t w[4];
    __device__ float operator[](int i) const
    {
        if constexpr (DT == PSC_BF16) return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
        else return Stored<DT>::load((uint16_t)(i & 1 ? w[i / 2] >> 16 : w[i / 2]));
    }
    __device__ void set(const float (&x)[8])
    {
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = (uint32_t)Stored<DT>::store(x[2 * k]) | (uint32_t)Stored<DT>::store(x[2 * k + 1]) << 16;
    }
    // The first n < 8 of them, by fours, twos and one.
    __device__ void load_first(const uint16_t *q, int n)
    {
        uint32_t two = 0u, one = 0u;
        if (n & 4) __builtin_memcpy(w, q, 8);
        if (n & 2) __builtin_memcpy(&two, q + (n & 4), 4);
        if (n & 1) one = q[n - 1];
        w[0] = (n & 6) == 2 ? two : n == 1 ? one : w[0];
        w[2] = (n & 6) == 6 ? two : n == 5 ? one : w[2];
        w[1] = n == 3 ? one : w[1];
        w[3] = n == 7 ? one : w[3];
    }
    __device__ void store_first(uint16_t *q, int n) const
    {
        const uint32_t two = n & 4 ? w[2] : w[0], one = n == 1 ? w[0] : n == 3 ? w[1] : n == 5 ? w[2] : w[3];
        if (n & 4) __builtin_memcpy(q, w, 8);
        if (n & 2) __builtin_memcpy(q + (n & 4), &two, 4);
        if (n & 1) q[n - 1] = (uint16_t)one;
    }
};
template <>
struct Eight<PSC_F32> {
    float w[8];
    __device__ float operator[](int i) const { return w[i]; }
    __device__ void set(const float (&x)[8])
    {
#pragma unroll
        for (int k = 0; k < 8; ++k) w[k] = x[k];
    }
    __device__ void load_first(const float *q, int n)
    {
        float two[2] = {}, one = 0.f;
        if (n & 4) __builtin_memcpy(w, q, 16);
        if (n & 2) __builtin_memcpy(two, q + (n & 4), 8);
        if (n & 1) one = q[n - 1];
        w[0] = (n & 6) == 2 ? two[0] : n == 1 ? one : w[0];
        w[1] = (n & 6) == 2 ? two[1] : w[1];
        w[2] = n == 3 ? one : w[2];
        w[4] = (n & 6) == 6 ? two[0] : n == 5 ? one : w[4];
        w[5] = (n & 6) == 6 ? two[1] : w[5];
        w[6] = n == 7 ? one : w[6];
    }
    __device__ void store_first(float *q, int n) const
    {
        const float two[2] = {n & 4 ? w[4] : w[0], n & 4 ? w[5] : w[1]}, one = n == 1 ? w[0] : n == 3 ? w[2] : n == 5 ? w[4] : w[6];
        if (n & 4) __builtin_memcpy(q, w, 16);
        if (n & 2) __builtin_memcpy(q + (n & 4), two, 8);
        if (n & 1) q[n - 1] = one;
    }
};
template <int DT>
__device__ __forceinline__ void load_eight(const void *p, int64_t at, int n, bool tail, Eight<DT> &x)
{
    const typename Stored<DT>::type *q = (const typename Stored<DT>::type *)p + at;
#pragma unroll
    for (auto &w : x.w) w = 0;
    if (n >= 8) __builtin_memcpy(x.w, q, sizeof x.w);
    else if (tail && n > 0) x.load_first(q, n);
}
template <int DT>
__device__ __forceinline__ void store_eight(void *p, int64_t at, int n, bool tail, const Eight<DT> &x)
{
    typename Stored<DT>::type *q = (typename Stored<DT>::type *)p + at;
    if (n >= 8) __builtin_memcpy(q, x.w, sizeof x.w);
    else if (tail && n > 0) x.store_first(q, n);
}
template <int DT>
__device__ __forceinline__ void load_weights(const ResidualNorm &p, const void *w, int at, int n, bool tail, float (&x)[8])
{
    if (p.weight_f32) {
        Eight<PSC_F32> t;
        load_eight<PSC_F32>(w, at, n, tail, t);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = t[i];
    } else {
        Eight<DT> t;
        load_eight<DT>(w, at, n, tail, t);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = t[i];
    }
}

// Sum over a row's lanes (8 to 64 of a wave, or whole waves), the same in all of them: neighbours, mirrored halves, then rows of 16
// swapped, without LDS inside a wave.  `turn` says which half of the LDS array the waves meet in: one barrier a sum.
template <int kControl>
__device__ __forceinline__ float add_moved(float x) { return x + __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), kControl, 0xf, 0xf, false)); }
struct RowSum {
    float (*shared)[16];  // [2][16]
    int lanes, turn;
    __device__ float operator()(float x)
    {
        typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
        x = add_moved<0xb1>(x);   // quads: 1 0 3 2
        x = add_moved<0x4e>(x);   // 2 3 0 1
        x = add_moved<0x141>(x);  // halves of a row of 16, mirrored
        if (lanes > 8) x = add_moved<0x140>(x);  // the row mirrored
        if (lanes > 16) {
            const u32x2 y = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false));
            x = __uint_as_float(y.x) + __uint_as_float(y.y);
        }
        if (lanes > 32) {
            const u32x2 y = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false));
            x = __uint_as_float(y.x) + __uint_as_float(y.y);
        }
        if (lanes <= 64) return x;
        const int waves = lanes / 64;
        if (lane_id() == 0) shared[turn][threadIdx.x >> 6] = x;
        __syncthreads();
        x = 0.f;
        for (int w = 0; w < waves; ++w) x += shared[turn][w];
        turn ^= 1;
        return x;
    }
};

// 1 / (1 + e^-g).  What rounding -g log2 e to 32 bits leaves goes back in, so that the power is off by some 2^-23 wherever it counts.
__device__ __forceinline__ float sigmoid(float g)
{
    const float t = g * -1.44269504f, rest = __builtin_fmaf(g, -1.44269504f, -t) + g * 1.925963e-8f * -1.f;
    const float e = __builtin_amdgcn_exp2f(t);
    const float p = fabsf(t) < 126.f ? __builtin_fmaf(e, rest * 0.693147181f, e) : e;  // (infinite and zero powers stay)
    return __builtin_amdgcn_rcpf(1.f + p);
}

// From m = sigmoid(-|g|).
__device__ __forceinline__ float sigmoid_of(float g, float m) { return g >= 0.f ? 1.f - m : m; }
__device__ __forceinline__ float sigmoid_slope(float m) { return m * (1.f - m); }
__device__ __forceinline__ float silu_slope(float g, float m) { return __builtin_fmaf(g, sigmoid_slope(m), sigmoid_of(g, m)); }

// Places of a lane's coordinates in its row.
struct Columns {
    int lane, lanes, width;
    bool tail;
    __device__ int at(int v) const { return (v * lanes + lane) * 8; }
    // Coordinates of vector v of NV: all but the last vector are whole in every lane (half the lanes would not do for the row).
    template <int NV>
    __device__ int count(int v) const { return v < NV - 1 ? 8 : max(0, min(8, width - at(v))); }
};

// The weights of both norms: a workgroup's rows share them in LDS (in registers they would cost a third of the waves: at the step that took 156
// us forward, 195), where a lane's eight lie in two planes, 16 bytes beside the next lane's.  The widest rows' do not fit and are read again for every row.
template <int TB, int NV, bool kLds>
struct NormWeights {
    float4 *lds;
    __device__ void fill(const ResidualNorm &p, const Columns &col)
    {
        if constexpr (kLds) {
            if ((int)threadIdx.x < col.lanes) {
#pragma unroll
                for (int which = 0; which < 2; ++which) {
                    const void *w = which ? p.before : p.after;
                    if (!w) continue;
#pragma unroll
                    for (int v = 0; v < NV; ++v) {
                        float x[8];
                        load_weights<TB>(p, w, col.at(v), col.template count<NV>(v), col.tail, x);
#pragma unroll
                        for (int half = 0; half < 2; ++half)
                            lds[((which * NV + v) * 2 + half) * col.lanes + col.lane] = make_float4(x[4 * half], x[4 * half + 1], x[4 * half + 2], x[4 * half + 3]);
                    }
                }
            }
            __syncthreads();
        }
    }
    __device__ void get(const ResidualNorm &p, const Columns &col, int which, float (&x)[NV][8]) const
    {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            if constexpr (kLds) {
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const float4 t = lds[((which * NV + v) * 2 + half) * col.lanes + col.lane];
                    x[v][4 * half] = t.x;
                    x[v][4 * half + 1] = t.y;
                    x[v][4 * half + 2] = t.z;
                    x[v][4 * half + 3] = t.w;
                }
            } else {
                load_weights<TB>(p, which ? p.before : p.after, col.at(v), col.template count<NV>(v), col.tail, x[v]);
            }
        }
    }
};
template <int NV>
constexpr size_t weights_lds(int lanes) { return (size_t)lanes * NV * 64; }

#define PSC_EACH                        \
    _Pragma("unroll") for (int v = 0; v < NV; ++v) _Pragma("unroll") for (int i = 0; i < 8; ++i)

// Multiplies by the gate g's factor and by its derivative, from m = sigmoid(-|g|), the smaller of sigmoid(g) and 1 - sigmoid(g) (which a plain
// gate does not ask for): the larger, 1 - m, and the slope m (1 - m) keep their bits, where 1 - sigmoid(g) of an open gate would
// lose them (all of them from g = 17 on).  One of three loops, not a choice for every coordinate (which took 271 us backward instead of 226).
struct Gate {
    bool plain, silu;
    __device__ explicit Gate(int activation) : plain(activation == PSC_GATE_PLAIN), silu(activation == PSC_GATE_SILU) {}
    template <int TB, int NV>
    __device__ __forceinline__ void smaller(const Eight<TB> (&g)[NV], float (&m)[NV][8]) const
    {
        if (!plain) PSC_EACH m[v][i] = sigmoid(-fabsf(g[v][i]));
    }
    template <int TB, int NV>
    __device__ __forceinline__ void factors(const Eight<TB> (&g)[NV], float (&f)[NV][8]) const
    {
        if (plain) {
            PSC_EACH f[v][i] = g[v][i];
            return;
        }
        PSC_EACH f[v][i] = sigmoid(g[v][i]);
        if (silu) PSC_EACH f[v][i] *= g[v][i];
    }
    template <int TB, int NV>
    __device__ __forceinline__ void open(float (&x)[NV][8], const Eight<TB> (&g)[NV], const float (&m)[NV][8]) const
    {
        if (plain) PSC_EACH x[v][i] *= g[v][i];
        else if (silu) PSC_EACH x[v][i] *= g[v][i] * sigmoid_of(g[v][i], m[v][i]);
        else PSC_EACH x[v][i] *= sigmoid_of(g[v][i], m[v][i]);
    }
    template <int TB, int NV>
    __device__ __forceinline__ void slope(float (&x)[NV][8], const Eight<TB> (&g)[NV], const float (&m)[NV][8]) const
    {
        if (plain) return;
        if (silu) PSC_EACH x[v][i] *= silu_slope(g[v][i], m[v][i]);
        else PSC_EACH x[v][i] *= sigmoid_slope(m[v][i]);
    }
};

// What a lane holds of a row as it lies in memory.
template <int TS, int TB, int NV, bool kBack, bool kGate>
struct RowData {
    Eight<TB> y[NV], g[kGate ? NV : 1], dz[kBack ? NV : 1];
    Eight<TS> x[NV], dh[kBack ? NV : 1];
    float2 stat;
    __device__ __forceinline__ void load(const ResidualNorm &p, const NormGradients *d, const Columns &col, int64_t row, int64_t gate_row)
    {
        if constexpr (kBack) stat = *(const float2 *)(d->stat + row * 2);
        if (p.y)
#pragma unroll
            for (int v = 0; v < NV; ++v) load_eight<TB>(p.y, row * p.y_stride + col.at(v), col.template count<NV>(v), col.tail, y[v]);
        if (kGate && p.gate)
#pragma unroll
            for (int v = 0; v < NV; ++v) load_eight<TB>(p.gate, gate_row * p.gate_stride + col.at(v), col.template count<NV>(v), col.tail, g[kGate ? v : 0]);
        if (p.x)
#pragma unroll
            for (int v = 0; v < NV; ++v) load_eight<TS>(p.x, row * p.x_stride + col.at(v), col.template count<NV>(v), col.tail, x[v]);
        if constexpr (kBack) {
            if (d->dz)
#pragma unroll
                for (int v = 0; v < NV; ++v) load_eight<TB>(d->dz, row * p.width + col.at(v), col.template count<NV>(v), col.tail, dz[v]);
            if (d->dh)
#pragma unroll
                for (int v = 0; v < NV; ++v) load_eight<TS>(d->dh, row * p.width + col.at(v), col.template count<NV>(v), col.tail, dh[v]);
        }
    }
};

template <int DT, int NV>
__device__ __forceinline__ void store_vectors(void *to, int64_t row, const Columns &col, const float (&x)[NV][8])
{
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        Eight<DT> t;
        t.set(x[v]);
        store_eight<DT>(to, row * col.width + col.at(v), col.template count<NV>(v), col.tail, t);
    }
}

// The next row is on its way while one is worked on.
template <int TS, int TB, int NV, int kThreads>
__global__ __launch_bounds__(kThreads) void residual_norm_kernel(ResidualNorm p, void *h_out, void *z_out, float *stat)
{
    __shared__ float shared[2][16];
    extern __shared__ float4 dynamic[];
    constexpr bool kLds = kThreads <= 512;
    const int lanes = p.lanes, rows_at_once = lanes > 64 ? 1 : (int)blockDim.x / lanes, step = (int)gridDim.x * rows_at_once;
    const Columns col{(int)threadIdx.x % lanes, lanes, p.width, p.width % 8 != 0};
    RowSum sum{shared, lanes, 0};
    NormWeights<TB, NV, kLds> weights{dynamic};
    int row = (int)blockIdx.x * rows_at_once + (int)threadIdx.x / lanes;
    const Gate gate(p.activation);
    RowData<TS, TB, NV, false, true> now, next;
    if (row < p.rows) now.load(p, nullptr, col, row, p.gate ? row / p.gate_each : 0);
    weights.fill(p, col);
    const float each = 1.f / (float)p.width;
    while (row < p.rows) {
        const int after = row <= p.rows - step ? row + step : p.rows;  // (p.rows: none)
        if (after < p.rows) next.load(p, nullptr, col, after, p.gate ? after / p.gate_each : 0);
        float root_y = 1.f, root_h = 1.f, h[NV][8];
        if (p.y) {
            PSC_EACH h[v][i] = now.y[v][i];
            if (p.after) {
                float s = 0.f, w[NV][8];
                PSC_EACH s = __builtin_fmaf(h[v][i], h[v][i], s);
                weights.get(p, col, 0, w);
                root_y = 1.f / sqrtf(sum(s) * each + p.eps);
                PSC_EACH h[v][i] = h[v][i] * root_y * w[v][i];
            }
            if (p.gate) {
                float f[NV][8];
                gate.factors(now.g, f);
                PSC_EACH h[v][i] *= f[v][i];
            }
            PSC_EACH h[v][i] *= p.block_scale;
            if (p.x) PSC_EACH h[v][i] = __builtin_fmaf(p.residual_scale, now.x[v][i], h[v][i]);
        } else {
            PSC_EACH h[v][i] = p.residual_scale * now.x[v][i];
        }
        if (h_out) store_vectors<TS>(h_out, row, col, h);
        if (p.before) {
            float s = 0.f, w[NV][8];
            PSC_EACH s = __builtin_fmaf(h[v][i], h[v][i], s);
            weights.get(p, col, 1, w);
            root_h = 1.f / sqrtf(sum(s) * each + p.eps);
            PSC_EACH h[v][i] = h[v][i] * root_h * w[v][i];
            if (z_out) store_vectors<TB>(z_out, row, col, h);
        }
        if (stat && col.lane == 0) *(float2 *)(stat + (int64_t)row * 2) = make_float2(root_y, root_h);
        now = next;
        row = after;
    }
}

// Sums over a workgroup's rows, a place of each lane's own in LDS (registers would leave room for half the waves: at the step that took 272 us
// backward, 570), in planes of 16 bytes to a lane.
template <int NV>
struct RowSums {
    float4 *lds;
    __device__ float4 &plane(int k) const { return lds[k * (int)blockDim.x + (int)threadIdx.x]; }
    __device__ void set(const float (&x)[NV][8]) const
    {
#pragma unroll
        for (int k = 0; k < 2 * NV; ++k) plane(k) = make_float4(x[k / 2][k % 2 * 4], x[k / 2][k % 2 * 4 + 1], x[k / 2][k % 2 * 4 + 2], x[k / 2][k % 2 * 4 + 3]);
    }
    __device__ void add(const float (&x)[NV][8]) const
    {
#pragma unroll
        for (int k = 0; k < 2 * NV; ++k) {
            float4 t = plane(k);
            t.x += x[k / 2][k % 2 * 4];
            t.y += x[k / 2][k % 2 * 4 + 1];
            t.z += x[k / 2][k % 2 * 4 + 2];
            t.w += x[k / 2][k % 2 * 4 + 3];
            plane(k) = t;
        }
    }
    // The sums over the rows that the workgroup has at once, in the first row's lanes.
    __device__ void joined(int lanes, int rows, float (&x)[NV][8]) const
    {
        if (rows > 1) __syncthreads();
        if ((int)threadIdx.x < lanes) {
#pragma unroll
            for (int k = 0; k < 2 * NV; ++k) {
                float4 t = plane(k);
                for (int r = 1; r < rows; ++r) {
                    const float4 u = lds[k * (int)blockDim.x + r * lanes + (int)threadIdx.x];
                    t.x += u.x;
                    t.y += u.y;
                    t.z += u.z;
                    t.w += u.w;
                }
                x[k / 2][k % 2 * 4] = t.x;
                x[k / 2][k % 2 * 4 + 1] = t.y;
                x[k / 2][k % 2 * 4 + 2] = t.z;
                x[k / 2][k % 2 * 4 + 3] = t.w;
            }
        }
        if (rows > 1) __syncthreads();
    }
};
template <int NV>
constexpr size_t sums_lds(int threads) { return (size_t)threads * NV * 32; }

// Gradients.  A workgroup takes rows in a row of one gate row (or all rows of several gate rows, one after another), so that the
// sums over rows -- for the weights, and for a gate that many rows share (kShared) -- stay with it until the end; they are then
// left as the workgroup's share and added up in order by residual_norm_sums_kernel.
template <int TS, int TB, int NV, int kThreads, bool kShared>
__global__ __launch_bounds__(kThreads, 2) void residual_norm_backward_kernel(ResidualNorm p, NormGradients d)
{
    __shared__ float shared[2][16];
    extern __shared__ float4 dynamic[];
    constexpr bool kLds = kThreads <= 512, kAhead = kThreads <= 512 && TB != PSC_F32;  // (what comes next of float32 rows would not fit the registers)
    const int lanes = p.lanes, rows_at_once = lanes > 64 ? 1 : (int)blockDim.x / lanes, mine = (int)threadIdx.x / lanes;
    const Columns col{(int)threadIdx.x % lanes, lanes, p.width, p.width % 8 != 0};
    RowSum sum{shared, lanes, 0};
    NormWeights<TB, NV, kLds> weights{dynamic};
    float4 *behind = dynamic + (kLds ? weights_lds<NV>(lanes) / 16 : 0);
    const RowSums<NV> after_sums{behind}, before_sums{behind + sums_lds<NV>(blockDim.x) / 16}, gate_sums{behind + 2 * sums_lds<NV>(blockDim.x) / 16};
    const Gate act(p.activation);
    float dg[kShared ? NV : 1][8] = {};  // (which leaves room for the weights beside the others)
    {
        const float zero[NV][8] = {};
        after_sums.set(zero);
        before_sums.set(zero);
    }
    const float each = 1.f / (float)p.width;
    const int span = kShared ? p.gate_each : p.rows, gates = kShared ? p.rows / p.gate_each : 1;  // rows of a gate row; gate rows
    const int gate_begin = d.split > 1 ? (int)blockIdx.x / d.split : (int)blockIdx.x * d.gates_of_group;
    const int gate_end = d.split > 1 ? gate_begin + 1 : min(gates, gate_begin + d.gates_of_group);
    const int part = d.split > 1 ? (int)blockIdx.x % d.split : 0;
    weights.fill(p, col);
    for (int gate = gate_begin; gate < gate_end; ++gate) {
        const int begin = gate * span + (int)((int64_t)span * part / d.split), end = gate * span + (int)((int64_t)span * (part + 1) / d.split);
        // (a workgroup's lanes to the end together: they meet at barriers; past the last row: the last one again, which does not count)
        RowData<TS, TB, NV, true, !kShared> now, next;
        const auto load = [&](int row0, RowData<TS, TB, NV, true, !kShared> &to) {
            const int row = min(row0 + mine, end - 1);
            to.load(p, &d, col, row, kShared ? gate : row);
        };
        if (kAhead && begin < end) load(begin, now);
        float of_gate[NV][8];  // its factors, where all of these rows share it; else what `smaller` gives of a row's
        const auto load_gate = [&](Eight<TB> (&g)[NV]) {
#pragma unroll
            for (int v = 0; v < NV; ++v) load_eight<TB>(p.gate, (int64_t)gate * p.gate_stride + col.at(v), col.template count<NV>(v), col.tail, g[v]);
        };
        if constexpr (kShared) {
            Eight<TB> g[NV];
            load_gate(g);
            act.factors(g, of_gate);
        }
        for (int row0 = begin; row0 < end; row0 += rows_at_once) {
            const int64_t row = min(row0 + mine, end - 1);
            const bool there = row0 + mine < end;
            if constexpr (kAhead) load(min(row0 + rows_at_once, end - 1), next);
            else load(row0, now);
            const float root_y = now.stat.x, root_h = now.stat.y;
            float grad[NV][8];  // of h, then of u and what lies before it
            Eight<TB> g[kShared ? 1 : NV];
            if constexpr (!kShared) {
                if (p.gate) {
#pragma unroll
                    for (int v = 0; v < NV; ++v) g[v] = now.g[v];
                    act.smaller(g, of_gate);
                }
            }
            const auto open = [&](float (&x)[NV][8]) __attribute__((always_inline)) {
                if constexpr (kShared) PSC_EACH x[v][i] *= of_gate[v][i];
                else act.open(x, g, of_gate);
            };
            if (d.dz) {
                float normed[NV][8], w[NV][8], s = 0.f;
                if (p.y) {
                    PSC_EACH normed[v][i] = now.y[v][i];
                    if (p.after) {
                        weights.get(p, col, 0, w);
                        PSC_EACH normed[v][i] = normed[v][i] * root_y * w[v][i];
                    }
                    if (p.gate) open(normed);
                    PSC_EACH normed[v][i] *= p.block_scale;
                    if (p.x) PSC_EACH normed[v][i] = __builtin_fmaf(p.residual_scale, now.x[v][i], normed[v][i]);
                } else {
                    PSC_EACH normed[v][i] = p.residual_scale * now.x[v][i];
                }
                weights.get(p, col, 1, w);
                float t[NV][8];
                PSC_EACH
                {
                    normed[v][i] *= root_h;
                    t[v][i] = now.dz[v][i] * normed[v][i];
                    s = __builtin_fmaf(t[v][i], w[v][i], s);
                }
                if (there && d.before_parts) before_sums.add(t);
                s = sum(s) * each;
                PSC_EACH grad[v][i] = root_h * __builtin_fmaf(-normed[v][i], s, now.dz[v][i] * w[v][i]);
                if (d.dh) PSC_EACH grad[v][i] += now.dh[v][i];
            } else {
                if (d.dh) PSC_EACH grad[v][i] = now.dh[v][i];
                else PSC_EACH grad[v][i] = 0.f;
            }
            if (d.dx && there) {
                float t[NV][8];
                PSC_EACH t[v][i] = p.residual_scale * grad[v][i];
                store_vectors<TS>(d.dx, row, col, t);
            }
            if (p.y) {
                PSC_EACH grad[v][i] *= p.block_scale;
                float w[NV][8];
                if (p.after) weights.get(p, col, 0, w);
                if (p.gate) {
                    float t[NV][8];  // what the gate was multiplied by
                    PSC_EACH t[v][i] = now.y[v][i];
                    if (p.after) PSC_EACH t[v][i] = t[v][i] * root_y * w[v][i];
                    PSC_EACH t[v][i] *= grad[v][i];
                    if constexpr (kShared) {  // (a selection: 0 times an infinity would be NaN)
                        PSC_EACH dg[v][i] += there ? t[v][i] : 0.f;
                    } else if (d.dgate && there) {
                        act.slope(t, g, of_gate);
                        store_vectors<TB>(d.dgate, row, col, t);
                    }
                    open(grad);
                }
                if (p.after) {
                    float s = 0.f, t[NV][8];
                    PSC_EACH
                    {
                        t[v][i] = grad[v][i] * (now.y[v][i] * root_y);
                        s = __builtin_fmaf(t[v][i], w[v][i], s);
                    }
                    if (there && d.after_parts) after_sums.add(t);
                    s = sum(s) * each;
                    PSC_EACH grad[v][i] = root_y * __builtin_fmaf(-(now.y[v][i] * root_y), s, grad[v][i] * w[v][i]);
                }
                if (d.dy && there) store_vectors<TB>(d.dy, row, col, grad);
            }
            if constexpr (kAhead) now = next;
        }
        if constexpr (kShared) {
            if (d.dgate) {
                if (rows_at_once > 1) {
                    gate_sums.set(dg);
                    gate_sums.joined(lanes, rows_at_once, dg);
                }
                if (mine == 0) {
                    if (d.split > 1) {
                        store_vectors<PSC_F32>(d.gate_parts, (int64_t)blockIdx.x, col, dg);
                    } else {
                        Eight<TB> g[NV];
                        load_gate(g);
                        act.smaller(g, of_gate);
                        act.slope(dg, g, of_gate);
                        store_vectors<TB>(d.dgate, gate, col, dg);
                    }
                }
            }
            PSC_EACH dg[v][i] = 0.f;
        }
    }
    float sums[NV][8];
    if (d.after_parts) {
        after_sums.joined(lanes, rows_at_once, sums);
        if (mine == 0) store_vectors<PSC_F32>(d.after_parts, (int64_t)blockIdx.x, col, sums);
    }
    if (d.before_parts) {
        before_sums.joined(lanes, rows_at_once, sums);
        if (mine == 0) store_vectors<PSC_F32>(d.before_parts, (int64_t)blockIdx.x, col, sums);
    }
}

// Adds up the workgroups' shares: 16 columns to a workgroup, 16 threads to a column with every 16th share each, joined in order.  z = 0: the
// weights after, 1: those before, 2 and on: gate rows.
template <int TB>
__global__ __launch_bounds__(256) void residual_norm_sums_kernel(ResidualNorm p, NormGradients d)
{
    const int which = (int)blockIdx.y, column = (int)blockIdx.x * 16 + ((int)threadIdx.x & 15), lane = (int)threadIdx.x >> 4;
    const float *parts = which == 0 ? d.after_parts : which == 1 ? d.before_parts : d.gate_parts;
    if (!parts) return;
    const int64_t first = which < 2 ? 0 : (int64_t)(which - 2) * d.split, count = which < 2 ? d.groups : d.split;
    float x = 0.f;
    if (column < p.width) {
        float t[4] = {};
        int64_t i = lane;
        for (; i + 48 < count; i += 64)
#pragma unroll
            for (int j = 0; j < 4; ++j) t[j] += parts[(first + i + 16 * j) * p.width + column];
        for (; i < count; i += 16) t[0] += parts[(first + i) * p.width + column];
        x = (t[0] + t[1]) + (t[2] + t[3]);
    }
    __shared__ float sums[16][17];
    sums[lane][threadIdx.x & 15] = x;
    __syncthreads();
    if (lane > 0 || column >= p.width) return;
    for (int l = 1; l < 16; ++l) x += sums[l][threadIdx.x & 15];
    if (which < 2) {
        void *to = which == 0 ? d.dafter : d.dbefore;
        if (p.weight_f32) ((float *)to)[column] = x;
        else ((typename Stored<TB>::type *)to)[column] = Stored<TB>::store(x);
    } else {
        const float g = Stored<TB>::load(((const typename Stored<TB>::type *)p.gate)[(int64_t)(which - 2) * p.gate_stride + column]);
        if (p.activation != PSC_GATE_PLAIN) {
            const float m = sigmoid(-fabsf(g));
            x *= p.activation == PSC_GATE_SILU ? silu_slope(g, m) : sigmoid_slope(m);
        }
        ((typename Stored<TB>::type *)d.dgate)[(int64_t)(which - 2) * p.width + column] = Stored<TB>::store(x);
    }
}

// A row of up to 512 coordinates has 8 to 64 lanes with a vector of 8 each, a longer one lanes with two: a wave up to 1024.
int vectors_of(int width) { return width > 512 ? 2 : 1; }
int lanes_of(int width)
{
    const int vectors = (width + 7) / 8, per = vectors_of(width);
    int lanes = 8;
    while (lanes * per < vectors) lanes *= 2;
    return lanes;
}

// A workgroup is one wide row's lanes, or 256 lanes with several narrow rows.
int threads_of(int lanes) { return lanes > 64 ? lanes : 256; }

// Threads of the forward pass at most, of the backward pass at least where there are rows for them.
constexpr int kForwardThreads = 256 * 1024, kBackwardThreads = 256 * 512;

template <int TS, int TB>
int run_forward(const ResidualNorm &p, void *h, void *z, float *stat, hipStream_t s)
{
    const int threads = threads_of(p.lanes), rows = threads / p.lanes;
    const uint32_t groups = (uint32_t)std::min<int64_t>((p.rows + rows - 1) / rows, kForwardThreads / threads);
    const auto launch = [&](auto nv, auto most) {
        residual_norm_kernel<TS, TB, nv.value, most.value><<<groups, threads, most.value <= 512 ? weights_lds<nv.value>(p.lanes) : 0, s>>>(p, h, z, stat);
    };
    if (vectors_of(p.width) == 1) launch(std::integral_constant<int, 1>(), std::integral_constant<int, 256>());
    else if (threads <= 256) launch(std::integral_constant<int, 2>(), std::integral_constant<int, 256>());
    else if (threads <= 512) launch(std::integral_constant<int, 2>(), std::integral_constant<int, 512>());
    else launch(std::integral_constant<int, 2>(), std::integral_constant<int, 1024>());
    PSC_HIP_TRY(hipGetLastError());
    return PSC_OK;
}

template <int TS, int TB>
int run_backward(const ResidualNorm &p, const NormGradients &d, hipStream_t s)
{
    const int threads = threads_of(p.lanes);
    const auto launch = [&](auto nv, auto most) {
        const bool shared = p.gate && p.gate_each > 1;
        const size_t lds = (most.value <= 512 ? weights_lds<nv.value>(p.lanes) : 0) + (shared && p.lanes < threads ? 3 : 2) * sums_lds<nv.value>(threads);
        if (shared) residual_norm_backward_kernel<TS, TB, nv.value, most.value, true><<<(uint32_t)d.groups, threads, lds, s>>>(p, d);
        else residual_norm_backward_kernel<TS, TB, nv.value, most.value, false><<<(uint32_t)d.groups, threads, lds, s>>>(p, d);
    };
    if (vectors_of(p.width) == 1) launch(std::integral_constant<int, 1>(), std::integral_constant<int, 256>());
    else if (threads <= 256) launch(std::integral_constant<int, 2>(), std::integral_constant<int, 256>());
    else if (threads <= 512) launch(std::integral_constant<int, 2>(), std::integral_constant<int, 512>());
    else launch(std::integral_constant<int, 2>(), std::integral_constant<int, 1024>());
    PSC_HIP_TRY(hipGetLastError());
    if (d.after_parts || d.before_parts || d.gate_parts) {
        const uint32_t gates = d.gate_parts ? (uint32_t)(p.rows / p.gate_each) : 0;
        residual_norm_sums_kernel<TB><<<dim3((uint32_t)((p.width + 15) / 16), 2 + gates), 256, 0, s>>>(p, d);
        PSC_HIP_TRY(hipGetLastError());
    }
    return PSC_OK;
}

}  // namespace

NormPlan plan_residual_norm(int rows, int width, int gate_each)
{
    NormPlan p;
    p.lanes = lanes_of(width);
    const int threads = threads_of(p.lanes), at_once = threads / p.lanes;
    const int64_t wanted = std::max(256, kBackwardThreads / threads);
    const bool shared = gate_each > 1;
    const int64_t span = shared ? gate_each : rows, gates = shared ? rows / gate_each : 1;
    if (gates >= wanted) {
        p.gates_of_group = (int)((gates + wanted - 1) / wanted);
        p.groups = (int)((gates + p.gates_of_group - 1) / p.gates_of_group);
    } else {
        p.split = (int)std::max<int64_t>(1, std::min((wanted + gates - 1) / gates, (span + at_once - 1) / at_once));
        p.groups = (int)(gates * p.split);
    }
    return p;
}

#define PSC_NORM_DISPATCH(fn, stream, block, ...)                                                                                             \
    (stream == block ? (block == PSC_BF16  ? fn<PSC_BF16, PSC_BF16>(__VA_ARGS__)                                                              \
                        : block == PSC_F16 ? fn<PSC_F16, PSC_F16>(__VA_ARGS__)                                                                \
                                           : fn<PSC_F32, PSC_F32>(__VA_ARGS__))                                                               \
                     : (block == PSC_BF16 ? fn<PSC_F32, PSC_BF16>(__VA_ARGS__) : fn<PSC_F32, PSC_F16>(__VA_ARGS__)))

int launch_residual_norm(const ResidualNorm &p, int stream_dtype, int block_dtype, void *h, void *z, float *stat, hipStream_t s)
{
    return PSC_NORM_DISPATCH(run_forward, stream_dtype, block_dtype, p, h, z, stat, s);
}

int launch_residual_norm_backward(const ResidualNorm &p, int stream_dtype, int block_dtype, const NormGradients &d, hipStream_t s)
{
    return PSC_NORM_DISPATCH(run_backward, stream_dtype, block_dtype, p, d, s);
}

}  // namespace psc
