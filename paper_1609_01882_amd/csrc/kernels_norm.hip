// Norms before and after a block, with the block's gate and the residual scale, and their gradients:
//   u = rms(y) * after * act(gate)      rms(t) = t / sqrt(mean t^2 + eps)
//   h = residual_scale x + block_scale u      z = rms(h) * before
// A row lies in the registers of `lanes` lanes, 8 consecutive coordinates (or twice 8) to each: 8 to 64 lanes of a wave for narrow rows,
// a workgroup for wide ones.  Each input is read once and each output written once; everything between is 32-bit floats.
#include <algorithm>
#include <cmath>

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

// 8 coordinates as they lie in memory; `n` of them are there (8, or fewer at a row's end).  Rows of odd widths begin anywhere: global loads
// of 16 bytes need no alignment.
template <int DT>
struct Eight {
    typename Stored<DT>::type t[8];
    __device__ float operator[](int i) const { return Stored<DT>::load(t[i]); }
    __device__ void set(int i, float x) { t[i] = Stored<DT>::store(x); }
};
template <int DT>
__device__ __forceinline__ void load_eight(const void *p, int64_t at, int n, Eight<DT> &x)
{
    const typename Stored<DT>::type *q = (const typename Stored<DT>::type *)p + at;
    if (n >= 8) __builtin_memcpy(x.t, q, sizeof x.t);
    else
#pragma unroll
        for (int i = 0; i < 8; ++i) x.t[i] = i < n ? q[i] : Stored<DT>::store(0.f);
}
template <int DT>
__device__ __forceinline__ void store_eight(void *p, int64_t at, int n, const Eight<DT> &x)
{
    typename Stored<DT>::type *q = (typename Stored<DT>::type *)p + at;
    if (n >= 8) __builtin_memcpy(q, x.t, sizeof x.t);
    else
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) q[i] = x.t[i];
}
template <int DT>
__device__ __forceinline__ void load_weights(const ResidualNorm &p, const void *w, int at, int n, float (&x)[8])
{
    if (p.weight_f32) {
        Eight<PSC_F32> t;
        load_eight<PSC_F32>(w, at, n, t);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = t[i];
    } else {
        Eight<DT> t;
        load_eight<DT>(w, at, n, t);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = t[i];
    }
}

// Sum over a row's lanes, the same in all of them.  `turn` says which half of the LDS array is used: one barrier a sum.
struct RowSum {
    float (*shared)[16];  // [2][16]
    int lanes, turn;
    __device__ float operator()(float x)
    {
        for (int d = 1; d < min(lanes, 64); d *= 2) x += __shfl_xor(x, d);
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

__device__ __forceinline__ float sigmoid(float g) { return 1.f / (1.f + expf(-g)); }
// The gate's factor, and its derivative.
__device__ __forceinline__ float act(int activation, float g) { return activation == PSC_GATE_PLAIN ? g : activation == PSC_GATE_SIGMOID ? sigmoid(g) : g * sigmoid(g); }
__device__ __forceinline__ float slope(int activation, float g)
{
    if (activation == PSC_GATE_PLAIN) return 1.f;
    const float s = sigmoid(g);
    return activation == PSC_GATE_SIGMOID ? s * (1.f - s) : s * (1.f + g * (1.f - s));
}

// Places of a lane's coordinates in its row.
struct Columns {
    int lane, lanes, width;
    __device__ int at(int v) const { return (v * lanes + lane) * 8; }
    __device__ int count(int v) const { return max(0, min(8, width - at(v))); }
};

template <int TS, int TB, int NV>
__global__ __launch_bounds__(1024) void residual_norm_kernel(ResidualNorm p, void *h_out, void *z_out, float *stat)
{
    __shared__ float shared[2][16];
    const int lanes = p.lanes, rows_at_once = lanes > 64 ? 1 : (int)blockDim.x / lanes;
    const Columns col{(int)threadIdx.x % lanes, lanes, p.width};
    RowSum sum{shared, lanes, 0};
    float wa[NV][8], wb[NV][8];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        if (p.after) load_weights<TB>(p, p.after, col.at(v), col.count(v), wa[v]);
        if (p.before) load_weights<TB>(p, p.before, col.at(v), col.count(v), wb[v]);
    }
    const float each = 1.f / (float)p.width;
    for (int64_t row = (int64_t)blockIdx.x * rows_at_once + threadIdx.x / lanes; row < p.rows; row += (int64_t)gridDim.x * rows_at_once) {
        Eight<TS> x[NV];
        Eight<TB> y[NV], g[NV];
        const int64_t gate_row = p.gate ? row / p.gate_each : 0;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            if (p.x) load_eight<TS>(p.x, row * p.x_stride + col.at(v), col.count(v), x[v]);
            if (p.y) load_eight<TB>(p.y, row * p.y_stride + col.at(v), col.count(v), y[v]);
            if (p.gate) load_eight<TB>(p.gate, gate_row * p.gate_stride + col.at(v), col.count(v), g[v]);
        }
        float root_y = 1.f, root_h = 1.f;
        if (p.after) {
            float s = 0.f;
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int i = 0; i < 8; ++i) s += y[v][i] * y[v][i];
            root_y = 1.f / sqrtf(sum(s) * each + p.eps);
        }
        float h[NV][8], s = 0.f;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float u = 0.f;
                if (p.y) {
                    u = y[v][i];
                    if (p.after) u = u * root_y * wa[v][i];
                    if (p.gate) u *= act(p.activation, g[v][i]);
                    u *= p.block_scale;
                }
                h[v][i] = p.x ? p.residual_scale * x[v][i] + u : u;
                s += h[v][i] * h[v][i];
            }
            if (h_out) {
                Eight<TS> t;
#pragma unroll
                for (int i = 0; i < 8; ++i) t.set(i, h[v][i]);
                store_eight<TS>(h_out, row * p.width + col.at(v), col.count(v), t);
            }
        }
        if (p.before) {
            root_h = 1.f / sqrtf(sum(s) * each + p.eps);
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                Eight<TB> t;
#pragma unroll
                for (int i = 0; i < 8; ++i) t.set(i, h[v][i] * root_h * wb[v][i]);
                if (z_out) store_eight<TB>(z_out, row * p.width + col.at(v), col.count(v), t);
            }
        }
        if (stat && col.lane == 0) *(float2 *)(stat + row * 2) = make_float2(root_y, root_h);
    }
}

// Gradients.  A workgroup takes rows in a row of one gate row (or all rows of several gate rows, one after another), so that the
// sums over rows -- for the weights, and for a gate that many rows share -- stay in registers until the end; they are then
// left as the workgroup's share and added up in order by residual_norm_sums_kernel.
template <int TS, int TB, int NV>
__global__ __launch_bounds__(1024) void residual_norm_backward_kernel(ResidualNorm p, NormGradients d)
{
    __shared__ float shared[2][16];
    extern __shared__ float joined[];
    const int lanes = p.lanes, rows_at_once = lanes > 64 ? 1 : (int)blockDim.x / lanes, mine = (int)threadIdx.x / lanes;
    const Columns col{(int)threadIdx.x % lanes, lanes, p.width};
    RowSum sum{shared, lanes, 0};
    float wa[NV][8], wb[NV][8], da[NV][8] = {}, db[NV][8] = {}, dg[NV][8] = {};
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        if (p.after) load_weights<TB>(p, p.after, col.at(v), col.count(v), wa[v]);
        if (p.before) load_weights<TB>(p, p.before, col.at(v), col.count(v), wb[v]);
    }
    const float each = 1.f / (float)p.width;
    // the sum of an accumulator over the workgroup's rows, in the first row's lanes
    const auto join = [&](float (&x)[NV][8]) {
        if (rows_at_once == 1) return;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int i = 0; i < 8; ++i) joined[(v * 8 + i) * (int)blockDim.x + (int)threadIdx.x] = x[v][i];
        __syncthreads();
        if (mine == 0) {
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    for (int r = 1; r < rows_at_once; ++r) x[v][i] += joined[(v * 8 + i) * (int)blockDim.x + r * lanes + col.lane];
        }
        __syncthreads();
    };
    const bool shared_gate = p.gate && p.gate_each > 1;
    const int span = shared_gate ? p.gate_each : p.rows, gates = shared_gate ? p.rows / p.gate_each : 1;  // rows of a gate row; gate rows
    const int gate_begin = d.split > 1 ? (int)blockIdx.x / d.split : (int)blockIdx.x * d.gates_of_group;
    const int gate_end = d.split > 1 ? gate_begin + 1 : min(gates, gate_begin + d.gates_of_group);
    const int part = d.split > 1 ? (int)blockIdx.x % d.split : 0;
    for (int gate = gate_begin; gate < gate_end; ++gate) {
        const int begin = gate * span + (int)((int64_t)span * part / d.split), end = gate * span + (int)((int64_t)span * (part + 1) / d.split);
        for (int row0 = begin; row0 < end; row0 += rows_at_once) {  // (a workgroup's lanes to the end together: they meet at barriers)
            const int64_t row = min(row0 + mine, end - 1);
            const bool there = row0 + mine < end;
            Eight<TS> x[NV], dh[NV];
            Eight<TB> y[NV], g[NV], dz[NV];
            const int64_t gate_row = !p.gate ? 0 : shared_gate ? gate : row;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                if (p.x) load_eight<TS>(p.x, row * p.x_stride + col.at(v), col.count(v), x[v]);
                if (p.y) load_eight<TB>(p.y, row * p.y_stride + col.at(v), col.count(v), y[v]);
                if (p.gate) load_eight<TB>(p.gate, gate_row * p.gate_stride + col.at(v), col.count(v), g[v]);
                if (d.dh) load_eight<TS>(d.dh, row * p.width + col.at(v), col.count(v), dh[v]);
                if (d.dz) load_eight<TB>(d.dz, row * p.width + col.at(v), col.count(v), dz[v]);
            }
            const float2 st = *(const float2 *)(d.stat + row * 2);
            const float root_y = st.x, root_h = st.y;
            float grad[NV][8];  // of h, then of u and what lies before it
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int i = 0; i < 8; ++i) grad[v][i] = d.dh ? dh[v][i] : 0.f;
            if (d.dz) {
                float normed[NV][8], t[NV][8], s = 0.f;
#pragma unroll
                for (int v = 0; v < NV; ++v)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        float u = 0.f;
                        if (p.y) {
                            u = y[v][i];
                            if (p.after) u = u * root_y * wa[v][i];
                            if (p.gate) u *= act(p.activation, g[v][i]);
                            u *= p.block_scale;
                        }
                        normed[v][i] = (p.x ? p.residual_scale * x[v][i] + u : u) * root_h;
                        const float dzi = dz[v][i];
                        if (there) db[v][i] += dzi * normed[v][i];
                        t[v][i] = dzi * wb[v][i];
                        s += normed[v][i] * t[v][i];
                    }
                s = sum(s) * each;
#pragma unroll
                for (int v = 0; v < NV; ++v)
#pragma unroll
                    for (int i = 0; i < 8; ++i) grad[v][i] += root_h * (t[v][i] - normed[v][i] * s);
            }
            if (d.dx && there) {
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    Eight<TS> t;
#pragma unroll
                    for (int i = 0; i < 8; ++i) t.set(i, p.residual_scale * grad[v][i]);
                    store_eight<TS>(d.dx, row * p.width + col.at(v), col.count(v), t);
                }
            }
            if (!p.y) continue;
            float normed[NV][8], s = 0.f;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                Eight<TB> of_gate;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    normed[v][i] = p.after ? y[v][i] * root_y : y[v][i];
                    float du = p.block_scale * grad[v][i];
                    if (p.gate) {
                        const float share = p.after ? normed[v][i] * wa[v][i] : normed[v][i], by_gate = du * share;
                        if (shared_gate) {
                            if (there) dg[v][i] += by_gate;
                        } else {
                            of_gate.set(i, by_gate * slope(p.activation, g[v][i]));
                        }
                        du *= act(p.activation, g[v][i]);
                    }
                    if (p.after) {
                        if (there) da[v][i] += du * normed[v][i];
                        du *= wa[v][i];
                        s += normed[v][i] * du;
                    }
                    grad[v][i] = du;
                }
                if (p.gate && !shared_gate && d.dgate && there) store_eight<TB>(d.dgate, row * p.width + col.at(v), col.count(v), of_gate);
            }
            if (p.after) {
                s = sum(s) * each;
#pragma unroll
                for (int v = 0; v < NV; ++v)
#pragma unroll
                    for (int i = 0; i < 8; ++i) grad[v][i] = root_y * (grad[v][i] - normed[v][i] * s);
            }
            if (d.dy && there) {
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    Eight<TB> t;
#pragma unroll
                    for (int i = 0; i < 8; ++i) t.set(i, grad[v][i]);
                    store_eight<TB>(d.dy, row * p.width + col.at(v), col.count(v), t);
                }
            }
        }
        if (shared_gate && d.dgate) {
            join(dg);
            if (mine == 0) {
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    const int n = col.count(v);
                    if (d.split > 1) {
                        Eight<PSC_F32> t;
#pragma unroll
                        for (int i = 0; i < 8; ++i) t.t[i] = dg[v][i];
                        store_eight<PSC_F32>(d.gate_parts, (int64_t)blockIdx.x * p.width + col.at(v), n, t);
                    } else {
                        Eight<TB> g, t;
                        load_eight<TB>(p.gate, gate * p.gate_stride + col.at(v), n, g);
#pragma unroll
                        for (int i = 0; i < 8; ++i) t.set(i, dg[v][i] * slope(p.activation, g[i]));
                        store_eight<TB>(d.dgate, (int64_t)gate * p.width + col.at(v), n, t);
                    }
                }
            }
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int i = 0; i < 8; ++i) dg[v][i] = 0.f;
        }
    }
    const auto leave = [&](float (&x)[NV][8], float *parts) {
        if (!parts) return;
        join(x);
        if (mine > 0) return;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            Eight<PSC_F32> t;
#pragma unroll
            for (int i = 0; i < 8; ++i) t.t[i] = x[v][i];
            store_eight<PSC_F32>(parts, (int64_t)blockIdx.x * p.width + col.at(v), col.count(v), t);
        }
    };
    leave(da, d.after_parts);
    leave(db, d.before_parts);
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
        const typename Stored<TB>::type g = ((const typename Stored<TB>::type *)p.gate)[(int64_t)(which - 2) * p.gate_stride + column];
        ((typename Stored<TB>::type *)d.dgate)[(int64_t)(which - 2) * p.width + column] = Stored<TB>::store(x * slope(p.activation, Stored<TB>::load(g)));
    }
}

// Vectors of 8 coordinates to a lane.
int vectors_of(int width) { return width > 8 * 1024 ? 2 : 1; }
int lanes_of(int width)
{
    const int vectors = (width + 7) / 8, per = vectors_of(width);
    int lanes = 8;
    while (lanes * per < vectors) lanes *= 2;
    return lanes;
}

// A workgroup is one wide row's lanes, or 256 lanes with several narrow rows.
int threads_of(int lanes) { return lanes > 64 ? lanes : 256; }

template <int TS, int TB>
int run_forward(const ResidualNorm &p, void *h, void *z, float *stat, hipStream_t s)
{
    const int threads = threads_of(p.lanes), rows = threads / p.lanes;
    const int64_t groups = std::min<int64_t>((p.rows + rows - 1) / rows, 256 * (2048 / threads));
    if (vectors_of(p.width) == 1) residual_norm_kernel<TS, TB, 1><<<(uint32_t)groups, threads, 0, s>>>(p, h, z, stat);
    else residual_norm_kernel<TS, TB, 2><<<(uint32_t)groups, threads, 0, s>>>(p, h, z, stat);
    PSC_HIP_TRY(hipGetLastError());
    return PSC_OK;
}

template <int TS, int TB>
int run_backward(const ResidualNorm &p, const NormGradients &d, hipStream_t s)
{
    const int threads = threads_of(p.lanes), nv = vectors_of(p.width);
    const size_t lds = p.lanes < threads ? (size_t)threads * nv * 8 * 4 : 0;
    if (nv == 1) residual_norm_backward_kernel<TS, TB, 1><<<(uint32_t)d.groups, threads, lds, s>>>(p, d);
    else residual_norm_backward_kernel<TS, TB, 2><<<(uint32_t)d.groups, threads, lds, s>>>(p, d);
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
    const int64_t wanted = 256 * std::max(1, 1024 / threads);
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
