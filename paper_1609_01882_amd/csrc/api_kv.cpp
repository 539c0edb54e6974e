// C ABI of the attention memory in 4 bits: argument checking and dispatch.  See include/psc.h for the contract.
#include <algorithm>
#include <cmath>
#include <cstdlib>

#include "common.h"

namespace psc {
namespace {

constexpr int64_t kMostSlots = (int64_t)1 << 30, kMostGroups = 65535;
constexpr int64_t kMostWorkgroups = ((int64_t)1 << 24) - 1;  // of 256 lanes: a dimension of a grid has under 2^32 lanes

bool aligned(const void *p, uintptr_t to = 16) { return (uintptr_t)p % to == 0; }

// The cache's own fields; what a call does not touch may be null (tables and lengths are always needed).
int check_cache(const psc_kv_cache *c, KvView *v)
{
    PSC_REQUIRE(c != nullptr, "null cache");
    PSC_REQUIRE(c->head_dim == 64 || c->head_dim == 128 || c->head_dim == 256, "head_dim must be 64, 128 or 256, got %d", c->head_dim);
    PSC_REQUIRE(c->page == 16 || c->page == 32 || c->page == 64 || c->page == 128 || c->page == 256,
                "page must be 16, 32, 64, 128 or 256, got %d", c->page);
    PSC_REQUIRE(c->kv_heads >= 1 && c->batch >= 1 && (int64_t)c->kv_heads * c->batch <= kMostGroups,
                "%d sequences of %d kv heads: at least 1 of each, at most %d together", c->batch, c->kv_heads, (int)kMostGroups);
    PSC_REQUIRE(c->pages >= 1 && c->pages <= 0x7fffffff, "%lld pages: 1 to 2^31 - 1", (long long)c->pages);
    PSC_REQUIRE(c->table_width >= 1 && (int64_t)c->table_width * c->page < kMostSlots, "table of %d pages of %d slots: 1 page to under 2^30 slots",
                c->table_width, c->page);
    PSC_REQUIRE((__int128)c->pages * c->kv_heads * c->page < (__int128)1 << 35, "%lld pages of %d heads and %d slots: under 2^35 together",
                (long long)c->pages, c->kv_heads, c->page);
    v->pages = c->pages;
    v->heads = c->kv_heads;
    v->dim = c->head_dim;
    v->page_shift = __builtin_ctz((unsigned)c->page);
    v->batch = c->batch;
    v->width = c->table_width;
    return PSC_OK;
}

int check_buffers(const psc_kv_cache *c, KvView *v)
{
    const int rc = check_cache(c, v);
    if (rc != PSC_OK) return rc;
    PSC_REQUIRE(c->k_codes_dev && c->k_scales_dev && c->v_codes_dev && c->v_scales_dev && c->table_dev && c->lengths_dev, "null cache buffer");
    PSC_REQUIRE(aligned(c->k_codes_dev) && aligned(c->k_scales_dev) && aligned(c->v_codes_dev) && aligned(c->v_scales_dev),
                "cache buffers must be 16-byte aligned");
    PSC_REQUIRE(aligned(c->table_dev, 4) && aligned(c->lengths_dev, 4), "misaligned table or lengths");
    v->k_codes = c->k_codes_dev;
    v->k_scales = c->k_scales_dev;
    v->v_codes = c->v_codes_dev;
    v->v_scales = c->v_scales_dev;
    v->table = c->table_dev;
    v->lengths = c->lengths_dev;
    return PSC_OK;
}

int check_dtype(int dtype)
{
    PSC_REQUIRE(dtype == PSC_BF16 || dtype == PSC_F16 || dtype == PSC_F32, "dtype must be PSC_BF16, PSC_F16 or PSC_F32, got %d", dtype);
    return PSC_OK;
}

int check_rows(const KvView &v, int nrows, const int32_t *offsets)
{
    PSC_REQUIRE(nrows >= 0, "%d rows", nrows);
    PSC_REQUIRE(offsets || nrows % v.batch == 0, "%d rows are no multiple of %d sequences, and there are no offsets", nrows, v.batch);
    PSC_REQUIRE(aligned(offsets, 4), "misaligned offsets");
    return PSC_OK;
}

// (A stride that leads to no second row or head may be anything.)
int check_strides(const char *what, const void *p, int dtype, int nrows, int64_t row, int heads, int64_t head)
{
    const int64_t unit = dtype == PSC_F32 ? 4 : 8;  // elements in 16 bytes
    row = nrows > 1 ? row : 0;
    head = heads > 1 ? head : 0;
    PSC_REQUIRE(p != nullptr, "null %s", what);
    PSC_REQUIRE(aligned(p) && row % unit == 0 && head % unit == 0, "%s: rows and heads must start at multiples of 16 bytes", what);
    PSC_REQUIRE(std::llabs(row) < (1ll << 40) && std::llabs(head) < (1ll << 40), "%s: stride too large", what);
    return PSC_OK;
}

int check_attention(const KvView &v, int dtype, int nrows, int max_rows, int q_heads, int window, int sinks)
{
    const int rc = check_dtype(dtype);
    if (rc != PSC_OK) return rc;
    PSC_REQUIRE(nrows >= 0 && max_rows >= 0, "%d rows, at most %d of a sequence", nrows, max_rows);
    PSC_REQUIRE(q_heads >= 1 && q_heads <= 65536 && q_heads % v.heads == 0, "%d query heads are no multiple of %d kv heads", q_heads, v.heads);
    PSC_REQUIRE((int64_t)nrows * q_heads < kMostSlots, "%d rows of %d heads: under 2^30 together", nrows, q_heads);
    PSC_REQUIRE(window >= 0 && sinks >= 0, "window (%d) and sinks (%d) must not be negative", window, sinks);
    return PSC_OK;
}

}  // namespace
}  // namespace psc

using namespace psc;

#define PSC_TRY(expr)                  \
    do {                               \
        const int rc_ = (expr);        \
        if (rc_ != PSC_OK) return rc_; \
    } while (0)

extern "C" {

int psc_kv_append(const psc_kv_cache *cache, int dtype, const void *k_dev, int64_t k_row_stride, int64_t k_head_stride,
                  const void *v_dev, int64_t v_row_stride, int64_t v_head_stride, int nrows, const int32_t *offsets_dev,
                  const int32_t *first_dev, int32_t *positions_dev, float *weights_dev, psc_stream stream)
{
    KvView v{};
    PSC_TRY(check_buffers(cache, &v));
    PSC_TRY(check_dtype(dtype));
    PSC_TRY(check_rows(v, nrows, offsets_dev));
    if (nrows == 0) return PSC_OK;
    PSC_TRY(check_strides("k", k_dev, dtype, nrows, k_row_stride, v.heads, k_head_stride));
    PSC_TRY(check_strides("v", v_dev, dtype, nrows, v_row_stride, v.heads, v_head_stride));
    PSC_REQUIRE(aligned(first_dev, 4) && aligned(positions_dev) && aligned(weights_dev), "misaligned first, positions or weights");
    PSC_REQUIRE((int64_t)nrows * v.heads * (v.dim / 8) <= kMostWorkgroups * 256, "%d rows of %d heads of %d are too many for a launch", nrows, v.heads, v.dim);
    const KvRows r{k_dev, v_dev, k_row_stride, k_head_stride, v_row_stride, v_head_stride, nrows, nrows / v.batch, offsets_dev, first_dev,
                   positions_dev, weights_dev};
    return launch_kv_append(v, dtype, r, (hipStream_t)stream);
}

int psc_kv_read(const psc_kv_cache *cache, int dtype, int nrows, const int32_t *offsets_dev, void *k_dev, void *v_dev,
                psc_stream stream)
{
    KvView v{};
    PSC_TRY(check_buffers(cache, &v));
    PSC_TRY(check_dtype(dtype));
    PSC_TRY(check_rows(v, nrows, offsets_dev));
    if (nrows == 0) return PSC_OK;
    PSC_TRY(check_strides("k", k_dev, dtype, 0, 0, 0, 0));
    PSC_TRY(check_strides("v", v_dev, dtype, 0, 0, 0, 0));
    PSC_REQUIRE((int64_t)nrows * v.heads * (v.dim / 8) <= kMostWorkgroups * 256, "%d rows of %d heads of %d are too many for a launch", nrows, v.heads, v.dim);
    KvRows r{};
    r.nrows = nrows;
    r.each = nrows / v.batch;
    r.offsets = offsets_dev;
    return launch_kv_read(v, dtype, r, k_dev, v_dev, (hipStream_t)stream);
}

size_t psc_kv_attention_workspace_bytes(const psc_kv_cache *cache, int dtype, int nrows, int max_rows, int q_heads,
                                        int window, int sinks, int has_positions, int has_weights)
{
    KvView v{};
    if (check_cache(cache, &v) != PSC_OK || check_attention(v, dtype, nrows, max_rows, q_heads, window, sinks) != PSC_OK) return 0;
    if (nrows == 0) return 0;
    // with offsets the call plans for max_rows, without for nrows / batch; neither plan contains the other
    const auto bytes = [&](int most) {
        return plan_kv_attention(v, dtype, q_heads / v.heads, nrows, most, window, sinks, !has_positions, has_weights != 0).bytes();
    };
    return std::max(bytes(max_rows), bytes((int)(((int64_t)nrows + v.batch - 1) / v.batch)));
}

int psc_kv_attention(const psc_kv_cache *cache, int dtype, const void *q_dev, int64_t q_row_stride,
                     int64_t q_head_stride, int nrows, int max_rows, int q_heads, const int32_t *offsets_dev,
                     const int32_t *first_dev, const int32_t *positions_dev, float scale, int causal, int window,
                     int sinks, void *out_dev, float *lse_dev, const float *weights_in_dev, float *weights_out_dev,
                     void *workspace_dev, size_t workspace_bytes, psc_stream stream)
{
    KvView v{};
    PSC_TRY(check_buffers(cache, &v));
    PSC_TRY(check_attention(v, dtype, nrows, max_rows, q_heads, window, sinks));
    PSC_TRY(check_rows(v, nrows, offsets_dev));
    PSC_REQUIRE(scale > 0.f && std::isfinite(scale), "scale must be positive and finite");
    PSC_REQUIRE(window == 0 || causal, "a window needs causal attention");
    PSC_REQUIRE(weights_out_dev || !weights_in_dev, "weights_in without weights_out");
    PSC_REQUIRE(aligned(first_dev, 4) && aligned(positions_dev) && aligned(weights_in_dev) && aligned(weights_out_dev) && aligned(lse_dev, 4),
                "misaligned first, positions, weights or lse");
    if (!offsets_dev || nrows == 0) max_rows = nrows / v.batch;
    PSC_REQUIRE(nrows == 0 || max_rows >= 1, "max_rows must be at least 1");
    PSC_REQUIRE((int64_t)max_rows * v.batch >= nrows, "%d rows are more than max_rows (%d) of each of %d sequences", nrows, max_rows, v.batch);
    if (nrows > 0) {
        PSC_TRY(check_strides("q", q_dev, dtype, nrows, q_row_stride, q_heads, q_head_stride));
        PSC_TRY(check_strides("out", out_dev, dtype, 0, 0, 0, 0));
    } else if (!weights_out_dev) {
        return PSC_OK;
    }
    const int group = q_heads / v.heads;
    const KvPlan p = plan_kv_attention(v, dtype, group, nrows, max_rows, window, sinks, !positions_dev, weights_out_dev != nullptr);
    PSC_REQUIRE(p.row_groups <= kMostWorkgroups, "%d rows of a sequence are too many for a launch", max_rows);
    PSC_REQUIRE(p.weights_groups <= kMostWorkgroups, "%lld slots are too many for the weights of %d rows", (long long)v.width << v.page_shift, max_rows);
    PSC_REQUIRE(workspace_bytes >= p.bytes() && (p.bytes() == 0 || workspace_dev), "workspace too small: %zu bytes, %zu needed", workspace_bytes, p.bytes());
    PSC_REQUIRE(aligned(workspace_dev), "workspace must be 16-byte aligned");
    KvQueries q{};
    q.q = q_dev;
    q.row_stride = q_row_stride;
    q.head_stride = q_head_stride;
    q.nrows = nrows;
    q.each = nrows / v.batch;
    q.max_rows = max_rows;
    q.q_heads = q_heads;
    q.group = group;
    q.offsets = offsets_dev;
    q.first = first_dev;
    q.positions = positions_dev;
    q.factor = (float)((double)scale * 1.4426950408889634);
    q.causal = causal != 0;
    q.window = window;
    q.sinks = sinks;
    q.out = out_dev;
    q.lse = lse_dev;
    q.unit_rows = 16 * p.row_tiles;
    q.workgroups = (uint32_t)p.workgroups;
    q.least_blocks = (uint32_t)p.least_blocks;
    char *ws = (char *)workspace_dev;
    q.part_stat = (float *)ws;
    q.part_acc = (float *)(ws + p.part_stat_bytes);
    q.stat = p.stat_bytes ? (float *)(ws + p.part_stat_bytes + p.part_acc_bytes) : nullptr;
    q.scores = p.scores_bytes ? (float *)(ws + p.part_stat_bytes + p.part_acc_bytes + p.stat_bytes) : nullptr;
    q.scores_rows = p.scores_rows;
    return launch_kv_attention(v, dtype, q, p, weights_in_dev, weights_out_dev, (hipStream_t)stream);
}

size_t psc_kv_evict_workspace_bytes(const psc_kv_cache *cache, int budget)
{
    KvView v{};
    if (check_cache(cache, &v) != PSC_OK || budget < 1 || budget >= kMostSlots) return 0;
    return plan_kv_evict(v, budget).bytes();
}

int psc_kv_evict(const psc_kv_cache *cache, const float *weights_dev, const int32_t *positions_dev,
                 const int32_t *seen_dev, int budget, int sinks, int recent, int32_t *kept_dev,
                 int32_t *lengths_out_dev, int32_t *positions_out_dev, float *weights_out_dev, int64_t out_stride,
                 void *workspace_dev, size_t workspace_bytes, psc_stream stream)
{
    KvView v{};
    PSC_TRY(check_buffers(cache, &v));
    PSC_REQUIRE(budget >= 1 && budget < kMostSlots, "budget must be 1 to under 2^30, got %d", budget);
    PSC_REQUIRE(sinks >= 0 && recent >= 0 && (int64_t)sinks + recent <= budget, "sinks (%d) and recent (%d) must not be negative, nor more than the budget (%d) together",
                sinks, recent, budget);
    PSC_REQUIRE(weights_dev && kept_dev && lengths_out_dev && weights_out_dev, "null weights, kept, lengths_out or weights_out");
    PSC_REQUIRE(out_stride >= budget, "out_stride (%lld) is less than the budget (%d)", (long long)out_stride, budget);
    const int64_t slots = (int64_t)v.width << v.page_shift;
    PSC_REQUIRE((weights_out_dev != weights_dev && (!positions_dev || positions_out_dev != positions_dev)) || out_stride == slots,
                "in place, out_stride must be the %lld slots of a sequence", (long long)slots);
    PSC_REQUIRE(aligned(weights_dev, 4) && aligned(positions_dev, 4) && aligned(seen_dev, 4) && aligned(kept_dev, 4) && aligned(lengths_out_dev, 4) &&
                    aligned(positions_out_dev, 4) && aligned(weights_out_dev, 4),
                "misaligned array");
    const KvEvictPlan p = plan_kv_evict(v, budget);
    const size_t need = p.bytes();
    PSC_REQUIRE((int64_t)v.batch * v.heads * budget * (v.dim / 32) <= kMostWorkgroups * 256, "budget %d of %d x %d memories is too large for a launch", budget,
                v.batch, v.heads);
    PSC_REQUIRE(workspace_dev && workspace_bytes >= need && aligned(workspace_dev), "workspace too small or misaligned: %zu bytes, %zu needed", workspace_bytes, need);
    KvEvict e{};
    e.weights = weights_dev;
    e.positions = positions_dev;
    e.seen = seen_dev;
    e.budget = budget;
    e.sinks = sinks;
    e.recent = recent;
    e.out_stride = out_stride;
    e.kept = kept_dev;
    e.lengths_out = lengths_out_dev;
    e.positions_out = positions_out_dev;
    e.weights_out = weights_out_dev;
    return launch_kv_evict(v, e, p, (char *)workspace_dev, (hipStream_t)stream);
}

}  // extern "C"
