// C ABI of what a layer needs around its attention memory: rotary positions and norms around a block.  See include/psc.h for the contract.
#include "api_checks.h"

namespace psc {
namespace {

// 2^256 / (2 pi), most significant 64 bits first.
constexpr uint64_t kTurnsOfARadian[4] = {0x28be60db9391054aull, 0x7f09d5f47d4d3770ull, 0x36d8a5664f10e410ull, 0x7f9458eaf7aef158ull};

// radians / (2 pi) modulo 1 in units of 2^-64, to the nearest: the 53-bit mantissa times 256 bits of 1 / (2 pi).
uint64_t turns_of(double radians)
{
    if (radians == 0.0) return 0;
    int e;
    const double m = std::frexp(std::fabs(radians), &e);      // radians = m 2^e, 1/2 <= m < 1
    const uint64_t mantissa = (uint64_t)std::ldexp(m, 53);    // = mantissa 2^(e - 53)
    uint64_t product[5] = {};                                  // least significant first; 2^(e - 53 - 256) to a unit
    unsigned __int128 carry = 0;
    for (int i = 0; i < 4; ++i) {
        carry += (unsigned __int128)mantissa * kTurnsOfARadian[3 - i];
        product[i] = (uint64_t)carry;
        carry >>= 64;
    }
    product[4] = (uint64_t)carry;
    const int shift = 53 + 256 - 64 - e;                       // bits below the unit of the result
    const auto bits_from = [&](int at) -> uint64_t {           // 64 bits from bit `at` on
        if (at >= 320) return 0;
        const int word = at / 64, bit = at % 64;
        const uint64_t lo = product[word] >> bit, hi = bit && word + 1 < 5 ? product[word + 1] << (64 - bit) : 0;
        return lo | hi;
    };
    const uint64_t t = bits_from(shift) + (bits_from(shift - 1) & 1);
    return radians < 0 ? 0 - t : t;
}

int check_norm(const psc_residual_norm *n, ResidualNorm *p)
{
    PSC_REQUIRE(n != nullptr, "null residual_norm");
    PSC_REQUIRE(n->rows >= 0 && n->rows < 1 << 30, "%d rows: under 2^30", n->rows);
    PSC_REQUIRE(n->width >= 1 && n->width <= PSC_MAX_NORM_WIDTH, "width must be 1 to %d, got %d", PSC_MAX_NORM_WIDTH, n->width);
    PSC_TRY(check_dtype(n->stream_dtype));
    PSC_TRY(check_dtype(n->block_dtype));
    PSC_REQUIRE(n->stream_dtype == n->block_dtype || n->stream_dtype == PSC_F32, "the stream must be float32 or of the block's type");
    PSC_REQUIRE(n->weight_dtype == PSC_F32 || n->weight_dtype == n->block_dtype, "weights must be float32 or of the block's type");
    PSC_REQUIRE(n->rows == 0 || n->x_dev || n->y_dev, "null x and y");
    PSC_REQUIRE(n->y_dev || (!n->gate_dev && !n->after_dev), "a gate or a norm after the block without y");
    PSC_REQUIRE(n->activation == PSC_GATE_PLAIN || n->activation == PSC_GATE_SIGMOID || n->activation == PSC_GATE_SILU,
                "activation must be PSC_GATE_PLAIN, PSC_GATE_SIGMOID or PSC_GATE_SILU, got %d", n->activation);
    PSC_REQUIRE(std::isfinite(n->residual_scale) && std::isfinite(n->block_scale), "scales must be finite");
    PSC_REQUIRE(n->eps >= 0.f && std::isfinite(n->eps), "eps must be finite and not negative");
    const uintptr_t stream = n->stream_dtype == PSC_F32 ? 4 : 2, block = n->block_dtype == PSC_F32 ? 4 : 2, weight = n->weight_dtype == PSC_F32 ? 4 : 2;
    PSC_REQUIRE(aligned(n->x_dev, stream) && aligned(n->y_dev, block) && aligned(n->gate_dev, block) && aligned(n->after_dev, weight) && aligned(n->before_dev, weight),
                "misaligned x, y, gate or weights");
    PSC_REQUIRE(std::llabs(n->x_stride) < (1ll << 40) && std::llabs(n->y_stride) < (1ll << 40) && std::llabs(n->gate_stride) < (1ll << 40), "stride too large");
    if (n->gate_dev && n->rows > 0)
        PSC_REQUIRE(n->gate_rows >= 1 && n->rows % n->gate_rows == 0, "%d rows are no multiple of %d gate rows", n->rows, n->gate_rows);
    p->x = n->x_dev;
    p->y = n->y_dev;
    p->gate = n->gate_dev;
    p->after = n->after_dev;
    p->before = n->before_dev;
    p->x_stride = n->x_stride;
    p->y_stride = n->y_stride;
    p->gate_stride = n->gate_stride;
    p->rows = n->rows;
    p->width = n->width;
    p->gate_each = n->gate_dev && n->rows > 0 ? n->rows / n->gate_rows : 1;
    p->activation = n->activation;
    p->weight_f32 = n->weight_dtype == PSC_F32;
    p->residual_scale = n->residual_scale;
    p->block_scale = n->block_scale;
    p->eps = n->eps;
    p->lanes = plan_residual_norm(n->rows, n->width, p->gate_each).lanes;
    return PSC_OK;
}

size_t parts_bytes(const NormPlan &plan, int width) { return ((size_t)plan.groups * width * 4 + 255) / 256 * 256; }

}  // namespace
}  // namespace psc

using namespace psc;

extern "C" {

int psc_rotary_turns(const double *radians, int n, uint64_t *turns)
{
    PSC_REQUIRE(n >= 0 && (n == 0 || (radians && turns)), "null radians or turns");
    for (int i = 0; i < n; ++i) PSC_REQUIRE(std::isfinite(radians[i]) && std::fabs(radians[i]) <= 1024.0, "frequencies must lie between -1024 and 1024 radians");
    for (int i = 0; i < n; ++i) turns[i] = turns_of(radians[i]);
    return PSC_OK;
}

int psc_rotary_rows(const psc_rotary *rotary, int transposed, int dtype, const void *x_dev, int64_t row_stride,
                    int64_t head_stride, int nrows, int heads, int head_dim, const int32_t *positions_dev, int batch,
                    const int32_t *offsets_dev, const int32_t *first_dev, void *out_dev, int64_t out_row_stride,
                    int64_t out_head_stride, psc_stream stream)
{
    PSC_TRY(check_dtype(dtype));
    PSC_REQUIRE(head_dim >= 2 && head_dim <= 65536 && heads >= 1 && heads <= 65536, "%d heads of %d: 1 to 65536 of 2 to 65536", heads, head_dim);
    Rotary t{};
    PSC_TRY(check_rotary(rotary, head_dim, &t));
    PSC_REQUIRE(nrows >= 0, "%d rows", nrows);
    PSC_REQUIRE(!positions_dev || (!offsets_dev && !first_dev), "positions of rows and of sequences");
    PSC_REQUIRE(positions_dev || batch >= 1, "%d sequences", batch);
    PSC_REQUIRE(positions_dev || offsets_dev || nrows % batch == 0, "%d rows are no multiple of %d sequences, and there are no offsets", nrows, batch);
    PSC_REQUIRE(aligned(positions_dev, 4) && aligned(offsets_dev, 4) && aligned(first_dev, 4), "misaligned positions, offsets or first");
    if (nrows == 0) return PSC_OK;
    const uintptr_t size = dtype == PSC_F32 ? 4 : 2;
    PSC_REQUIRE(x_dev && out_dev && aligned(x_dev, size) && aligned(out_dev, size), "null or misaligned x or out");
    for (int64_t s : {row_stride, head_stride, out_row_stride, out_head_stride}) PSC_REQUIRE(std::llabs(s) < (1ll << 40), "stride too large");
    PSC_REQUIRE(out_dev != x_dev || ((row_stride == out_row_stride || nrows == 1) && (head_stride == out_head_stride || heads == 1)), "in place, strides must be the same");
    const auto sixteens = [&](const void *p, int64_t row, int64_t head) {
        return aligned(p) && (nrows == 1 || row * (int64_t)size % 16 == 0) && (heads == 1 || head * (int64_t)size % 16 == 0);
    };
    const bool wide = t.dims % 16 == 0 && head_dim % 8 == 0 && sixteens(x_dev, row_stride, head_stride) && sixteens(out_dev, out_row_stride, out_head_stride);
    PSC_REQUIRE((int64_t)nrows * 2 * heads * (wide ? t.dims / 16 + (head_dim - t.dims + 15) / 16 : head_dim - t.dims / 2) <= kMostWorkgroups * 256,
                "%d rows of %d heads of %d are too many for a launch", nrows, heads, head_dim);
    RotaryRows r{};
    r.x = x_dev;
    r.out = out_dev;
    r.row_stride = row_stride;
    r.head_stride = head_stride;
    r.out_row_stride = out_row_stride;
    r.out_head_stride = out_head_stride;
    r.nrows = nrows;
    r.heads = heads;
    r.head_dim = head_dim;
    r.batch = batch;
    r.each = positions_dev ? 0 : nrows / batch;
    r.positions = positions_dev;
    r.offsets = offsets_dev;
    r.first = first_dev;
    r.transposed = transposed != 0;
    return launch_rotary(t, dtype, r, wide, (hipStream_t)stream);
}

int psc_residual_norm_forward(const psc_residual_norm *norm, void *h_dev, void *z_dev, float *stat_dev, psc_stream stream)
{
    ResidualNorm p{};
    PSC_TRY(check_norm(norm, &p));
    PSC_REQUIRE(!z_dev || p.before, "z without the weights before");
    PSC_REQUIRE(aligned(h_dev, norm->stream_dtype == PSC_F32 ? 4 : 2) && aligned(z_dev, norm->block_dtype == PSC_F32 ? 4 : 2) && aligned(stat_dev, 8), "misaligned h, z or stat");
    if (p.rows == 0) return PSC_OK;
    return launch_residual_norm(p, norm->stream_dtype, norm->block_dtype, h_dev, z_dev, stat_dev, (hipStream_t)stream);
}

size_t psc_residual_norm_workspace_bytes(const psc_residual_norm *norm)
{
    ResidualNorm p{};
    if (check_norm(norm, &p) != PSC_OK || p.rows == 0) return 0;
    const NormPlan plan = plan_residual_norm(p.rows, p.width, p.gate_each);
    return 3 * parts_bytes(plan, p.width);
}

int psc_residual_norm_backward(const psc_residual_norm *norm, const float *stat_dev, const void *dh_dev, const void *dz_dev,
                               void *dx_dev, void *dy_dev, void *dgate_dev, void *dafter_dev, void *dbefore_dev,
                               void *workspace_dev, size_t workspace_bytes, psc_stream stream)
{
    ResidualNorm p{};
    PSC_TRY(check_norm(norm, &p));
    PSC_REQUIRE(!dz_dev || p.before, "dz without the weights before");
    PSC_REQUIRE((!dx_dev || p.x) && (!dy_dev || p.y) && (!dgate_dev || p.gate) && (!dafter_dev || p.after) && (!dbefore_dev || p.before),
                "a gradient of what is not there");
    const uintptr_t stream_size = norm->stream_dtype == PSC_F32 ? 4 : 2, block = norm->block_dtype == PSC_F32 ? 4 : 2, weight = p.weight_f32 ? 4 : 2;
    PSC_REQUIRE(aligned(dh_dev, stream_size) && aligned(dx_dev, stream_size) && aligned(dz_dev, block) && aligned(dy_dev, block) && aligned(dgate_dev, block) &&
                    aligned(dafter_dev, weight) && aligned(dbefore_dev, weight),
                "misaligned gradient");
    PSC_REQUIRE(p.rows > 0, "gradients of no rows");
    PSC_REQUIRE(stat_dev && aligned(stat_dev, 8), "null or misaligned stat");
    const NormPlan plan = plan_residual_norm(p.rows, p.width, p.gate_each);
    const size_t each = parts_bytes(plan, p.width);
    PSC_REQUIRE(workspace_bytes >= 3 * each && workspace_dev && aligned(workspace_dev), "workspace too small or misaligned: %zu bytes, %zu needed", workspace_bytes, 3 * each);
    NormGradients d{};
    d.stat = stat_dev;
    d.dh = dh_dev;
    d.dz = dz_dev;
    d.dx = dx_dev;
    d.dy = dy_dev;
    d.dgate = dgate_dev;
    d.dafter = dafter_dev;
    d.dbefore = dbefore_dev;
    d.groups = plan.groups;
    d.split = plan.split;
    d.gates_of_group = plan.gates_of_group;
    char *ws = (char *)workspace_dev;
    d.after_parts = dafter_dev ? (float *)ws : nullptr;
    d.before_parts = dbefore_dev ? (float *)(ws + each) : nullptr;
    d.gate_parts = dgate_dev && p.gate_each > 1 && plan.split > 1 ? (float *)(ws + 2 * each) : nullptr;
    return launch_residual_norm_backward(p, norm->stream_dtype, norm->block_dtype, d, (hipStream_t)stream);
}

}  // extern "C"
