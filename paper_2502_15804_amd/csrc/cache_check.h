// What every entry point over a growing cache asks of its arguments, on the host.
#pragma once
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "cache_rows.h"
#include "fairkv.h"

namespace fairkv {

inline bool aligned(const void *p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
constexpr int64_t kMaxGroups = UINT32_MAX / 256;      // a grid's threads are counted in 32 bits
inline int launched() { return hipGetLastError() == hipSuccess ? FAIRKV_OK : FAIRKV_EHIP; }

inline int check_cache(const fairkv_cache *c)
{
    if (!c || !c->k || !c->v || !c->cap || (c->off == nullptr) == (c->pages == nullptr)) return FAIRKV_EINVAL;
    if (c->B < 1 || c->Hkv < 1 || c->D < 1 || c->n_rows < 0 || !aligned(c->k, 16) || !aligned(c->v, 16)) return FAIRKV_EINVAL;
    if (static_cast<int64_t>(c->B) * c->Hkv > INT32_MAX / 2) return FAIRKV_EINVAL;
    if (c->expected_rows < 0) return FAIRKV_EINVAL;
    if (c->pages && (c->max_pages < 1 || c->page_rows < 16 || (c->page_rows & (c->page_rows - 1)) != 0 || c->page_rows > (1 << 30))) return FAIRKV_EINVAL;
    if (c->off && (c->max_pages != 0 || c->page_rows != 0)) return FAIRKV_EINVAL;
    if (c->dtype != FAIRKV_BF16 && c->dtype != FAIRKV_F32 && c->dtype != FAIRKV_E4M3) return FAIRKV_EUNSUPPORTED;
    if (c->D != 64 && c->D != 128) return FAIRKV_EUNSUPPORTED;
    if (c->dtype != FAIRKV_E4M3) return c->n_scales == 0 ? FAIRKV_OK : FAIRKV_EINVAL;
    if (c->n_scales > FAIRKV_CACHE_SCALES) return FAIRKV_EUNSUPPORTED;
    if (c->n_scales != 1 && c->n_scales != c->Hkv) return FAIRKV_EINVAL;
    auto usable = [](float scale) { return std::isfinite(scale) && scale != 0.f && std::isfinite(1.f / scale); };      // smaller ones have few bits of their own left
    for (int32_t h = 0; h < c->n_scales; ++h)
        if (!usable(c->k_scale[h]) || !usable(c->v_scale[h])) return FAIRKV_EINVAL;
    return FAIRKV_OK;
}

inline RowMap row_map(const fairkv_cache *c)
{
    int shift = 0;
    while (c->pages && (1 << shift) < c->page_rows) ++shift;
    return RowMap{c->off, c->pages, c->n_rows, c->max_pages, shift};
}

}  // namespace fairkv
