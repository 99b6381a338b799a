// Host checks that the entry points of a serving step share, in whichever source they stand.
#pragma once

#include <stdint.h>

#include <cmath>

#include "../../include/qgemm.h"
#include "api_util.hpp"

namespace {

using qg::aligned16;
using qg::check_launch;
using qg::fail;
using qg::ok;

inline bool aligned(const void* p, unsigned n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

inline int page_log2(int page) {
  int n = 0;
  while ((1 << n) < page) ++n;
  return n;
}

inline bool good_page(int page) { return page >= 16 && page <= 1024 && (page & (page - 1)) == 0; }

inline int check_cache(int Hkv, int D, int pages, int page) {
  if (Hkv < 1) return fail(QGEMM_EINVAL, "Hkv must be >= 1 (got %d)", Hkv);
  if (D != 64 && D != 128) return fail(QGEMM_EUNSUPPORTED, "head dimension must be 64 or 128 (got %d)", D);
  if (!good_page(page)) return fail(QGEMM_EINVAL, "page must be a power of two in [16, 1024] (got %d)", page);
  if (pages < 1) return fail(QGEMM_EINVAL, "pages must be >= 1 (got %d)", pages);
  if ((long)Hkv * page * (D + D / 16) > 0x7fffffffL) return fail(QGEMM_EUNSUPPORTED, "a page of all heads spans 2 GiB or more");
  if ((long)pages * page > 0x7fffffffL) return fail(QGEMM_EUNSUPPORTED, "the cache has 2^31 or more slots");
  return QGEMM_OK;
}

inline int check_scale(float scale, float* sl2) {
  if (!(scale > 0.0f) || !std::isfinite(scale)) return fail(QGEMM_EINVAL, "scale must be finite and > 0");
  *sl2 = (float)((double)scale * 1.4426950408889634);   // exp(x) = exp2(x log2 e)
  return QGEMM_OK;
}

inline int check_heads(int H, int Hkv) {
  if (H < 1 || Hkv < 1 || H % Hkv != 0)
    return fail(QGEMM_EINVAL, "H and Hkv must be >= 1 with H a multiple of Hkv (got %d, %d)", H, Hkv);
  return QGEMM_OK;
}

// Rows of `row` elements each, `stride` elements apart, read or written 16 bytes at a time.
inline int check_rows(const char* name, const void* p, int64_t stride, int64_t row, int elem_bytes) {
  if (!aligned16(p)) return fail(QGEMM_EALIGN, "%s must be 16-byte aligned", name);
  if (stride < row) return fail(QGEMM_EINVAL, "%s: rows of %lld elements overlap at stride %lld", name, (long long)row, (long long)stride);
  if (stride * elem_bytes % 16 != 0) return fail(QGEMM_EALIGN, "%s: the row stride must be a multiple of 16 bytes", name);
  return QGEMM_OK;
}

// A plan's tables: none that is written may share memory with another, as workgroups write while others still read.
struct PlanTable {
  const char* name;
  const int32_t* at;
  int64_t n;
};

inline int check_apart(const PlanTable* written, int n_written, const PlanTable* read, int n_read) {
  auto overlap = [](const PlanTable& a, const PlanTable& b) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a.at), y = reinterpret_cast<uintptr_t>(b.at);
    return a.n > 0 && b.n > 0 && x < y + 4 * (uintptr_t)b.n && y < x + 4 * (uintptr_t)a.n;
  };
  for (int i = 0; i < n_written; ++i) {
    for (int j = 0; j < i; ++j)
      if (overlap(written[i], written[j])) return fail(QGEMM_EINVAL, "%s and %s overlap", written[j].name, written[i].name);
    for (int j = 0; j < n_read; ++j)
      if (overlap(written[i], read[j])) return fail(QGEMM_EINVAL, "%s, which is written, overlaps %s", written[i].name, read[j].name);
  }
  return QGEMM_OK;
}

}  // namespace
