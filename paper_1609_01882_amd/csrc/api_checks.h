// Checks that the calls around the attention memory share.
#pragma once

#include <cmath>
#include <cstdlib>

#include "common.h"

#define PSC_TRY(expr)                  \
    do {                               \
        const int rc_ = (expr);        \
        if (rc_ != PSC_OK) return rc_; \
    } while (0)

namespace psc {

constexpr int64_t kMostWorkgroups = ((int64_t)1 << 24) - 1;  // of 256 lanes: a dimension of a grid has under 2^32 lanes

inline bool aligned(const void *p, uintptr_t to = 16) { return (uintptr_t)p % to == 0; }

inline int check_dtype(int dtype)
{
    PSC_REQUIRE(dtype == PSC_BF16 || dtype == PSC_F16 || dtype == PSC_F32, "dtype must be PSC_BF16, PSC_F16 or PSC_F32, got %d", dtype);
    return PSC_OK;
}

// (A stride that leads to no second row or head may be anything.)
inline int check_strides(const char *what, const void *p, int dtype, int nrows, int64_t row, int heads, int64_t head)
{
    const int64_t unit = dtype == PSC_F32 ? 4 : 8;  // elements in 16 bytes
    row = nrows > 1 ? row : 0;
    head = heads > 1 ? head : 0;
    PSC_REQUIRE(p != nullptr, "null %s", what);
    PSC_REQUIRE(aligned(p) && row % unit == 0 && head % unit == 0, "%s: rows and heads must start at multiples of 16 bytes", what);
    PSC_REQUIRE(std::llabs(row) < (1ll << 40) && std::llabs(head) < (1ll << 40), "%s: stride too large", what);
    return PSC_OK;
}

inline int check_rotary(const psc_rotary *r, int head_dim, Rotary *t)
{
    PSC_REQUIRE(r != nullptr, "null rotary");
    PSC_REQUIRE(r->dims >= 2 && r->dims % 2 == 0 && r->dims <= head_dim, "dims must be even, 2 to the head's %d, got %d", head_dim, r->dims);
    PSC_REQUIRE(r->turns_dev != nullptr && aligned(r->turns_dev, 8), "null or misaligned turns");
    PSC_REQUIRE(std::isfinite(r->factor), "factor must be finite");
    t->turns = r->turns_dev;
    t->dims = r->dims;
    t->interleaved = r->interleaved != 0;
    t->factor = r->factor;
    return PSC_OK;
}

}  // namespace psc
