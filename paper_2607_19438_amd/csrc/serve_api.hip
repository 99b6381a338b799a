// C entry points of a serving step around the projections: the plan of a ragged batch, rotary positions, the
// paged 4-bit cache with the attention that reads it, and attention over packed prompts (declarations and
// contracts in include/qgemm.h). A source of its own, and so a code object of its own.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "../../include/qgemm.h"
#include "api_util.hpp"
#include "attn_kernels.hpp"
#include "attn_kv4.hpp"
#include "serve_kernels.hpp"
#include "tile_rules.hpp"

namespace {

using qg::aligned16;
using qg::check_launch;
using qg::fail;
using qg::ok;

bool aligned(const void* p, unsigned n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

int page_log2(int page) {
  int n = 0;
  while ((1 << n) < page) ++n;
  return n;
}

bool good_page(int page) { return page >= 16 && page <= 1024 && (page & (page - 1)) == 0; }

int check_cache(int Hkv, int D, int pages, int page) {
  if (Hkv < 1) return fail(QGEMM_EINVAL, "Hkv must be >= 1 (got %d)", Hkv);
  if (D != 64 && D != 128) return fail(QGEMM_EUNSUPPORTED, "head dimension must be 64 or 128 (got %d)", D);
  if (!good_page(page)) return fail(QGEMM_EINVAL, "page must be a power of two in [16, 1024] (got %d)", page);
  if (pages < 1) return fail(QGEMM_EINVAL, "pages must be >= 1 (got %d)", pages);
  if ((long)Hkv * page * (D + D / 16) > 0x7fffffffL) return fail(QGEMM_EUNSUPPORTED, "a page of all heads spans 2 GiB or more");
  if ((long)pages * page > 0x7fffffffL) return fail(QGEMM_EUNSUPPORTED, "the cache has 2^31 or more slots");
  return QGEMM_OK;
}

int check_scale(float scale, float* sl2) {
  if (!(scale > 0.0f) || !std::isfinite(scale)) return fail(QGEMM_EINVAL, "scale must be finite and > 0");
  *sl2 = (float)((double)scale * 1.4426950408889634);   // exp(x) = exp2(x log2 e)
  return QGEMM_OK;
}

int check_heads(int H, int Hkv) {
  if (H < 1 || Hkv < 1 || H % Hkv != 0)
    return fail(QGEMM_EINVAL, "H and Hkv must be >= 1 with H a multiple of Hkv (got %d, %d)", H, Hkv);
  return QGEMM_OK;
}

// Rows of `row` elements each, `stride` elements apart, read or written 16 bytes at a time.
int check_rows(const char* name, const void* p, int64_t stride, int64_t row, int elem_bytes) {
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

int check_apart(const PlanTable* written, int n_written, const PlanTable* read, int n_read) {
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

// ---------------------------------------------------------------------------
// attention over the cache: how many workgroups, and how many rows in a tile
// ---------------------------------------------------------------------------

constexpr long kCUs = 256;

struct Kv4Plan {
  int nt;             // 16-row tiles that share a pass over the keys
  int gran_log2;      // of the keys of a granule, which are not split
  int groups;         // workgroups
  long part_floats;   // of one partial result
};

Kv4Plan kv4_plan(int T, int R, int H, int Hkv, int D, int W, int page) {
  const long G = H / Hkv;
  const long rows = ((long)T * G + R - 1) / R;          // of a request and head, on average
  Kv4Plan p{};
  // Two tiles share the unpacking of the keys and values where a request's rows need more than one; a wave of four
  // has the registers of a whole SIMD. (us, one tile, two, four: 2 chunks of 550 rows, 5000 keys, 32/8 heads of 128
  // 190, 159, 199; 6 requests of 8 to 32 rows and 32/4 heads 43.2, 41.5, 49.3; 16 of 6 rows and 32/8 heads 38.3,
  // 33.7; 9 of 3 to 9 rows, 32/8 heads of 64 17.5, 17.2.)
  // Wide tiles unpack a key once for 128 rows, but each part of one is eight times a small tile's: taken where requests
  // fill them and there are almost as many as workgroups, so that few are split. (us, pairs of tiles and wide, 32/8 heads
  // of 128: chunks of 550 rows over 5000 keys 150, 131; 200 to 1500 over 12000 586, 436; a first chunk of 1000 45.8,
  // 31.1; 4 of 60 to 300 rows 86.1, 86.0; 12 of 64 to 128 rows 52.6, 59.1; one of 256 over 4000 45.6, 48.2.)
  const bool wide = rows >= 512 && (long)T * G / (16 * qg::kKv4Wide) * Hkv >= 208;
  p.nt = rows <= 16 ? 1 : wide ? qg::kKv4Wide : 2;
  const long tiles = ((long)T * G) / (16 * p.nt) + R;   // at least their number, requests of no tokens aside
  const long most_keys = (long)W * page;
  // As many workgroups as the CUs hold at once, or fewer if there are not so many granules. Of the pairs of 64-wide tiles
  // a CU holds three, which leaves each a third less of the work and more parts to join: taken from 24 granules of the
  // longest table each. (us with two, three, by those granules and requests x tokens: 32/8 heads, 7 24 x 5-16 20.9, 22.4;
  // 12 20 x 5-9 21.7, 22.8; 17 64 x 5-12 31.5, 32.2; 25 40 x 5-9 31.1, 30.3; 29 2 x 550 64.4, 61.8; 41 24 x 5-16 45.6,
  // 43.3; 58 2 x 550 105.5, 96.6; 80 100 x 5-30 83.9, 77.5.)
  long per_cu = wide       ? qg::kKv4PerCU<128, qg::kKv4Wide>
                : D == 128 ? (p.nt == 2 ? qg::kKv4PerCU<128, 2> : qg::kKv4PerCU<128, 1>)
                           : (p.nt == 2 ? qg::kKv4PerCU<64, 2> : qg::kKv4PerCU<64, 1>);
  if (D == 64 && p.nt == 2 && tiles * Hkv * qg::ceil_div(most_keys, 1L << qg::kKv4GranuleLog2) < 24 * per_cu * kCUs) per_cu = 2;
  const long fill = kCUs * per_cu;
  // Short units are left whole: a granule as long as the longest, no second kernel, and no part to write. With more units
  // than workgroups some of those would take two, so only very short ones. Measured (us, split, whole; by units and
  // the longest request, lengths down to a thirtieth of it):
  //   8 units, D=128    300 9.5, 7.3   500 9.6, 8.5    1000 9.8, 12.1
  //   48                300 8.1, 6.5   500 9.0, 7.6    1000 10.1, 10.3 (12 requests 10.9, 10.2)  1500 10.4, 12.8
  //   256               300 12.4, 7.6  500 13.4, 8.8   1000 14.1, 12.3  1500 15.6, 16.3
  //   512, D=64         300 11.3, 7.4  500 12.4, 8.4   1000 13.8, 11.2  1500 14.8, 14.0  2000 16.4, 17.2
  //   800, D=128        300 14.6, 13.2 500 15.9, 16.3  1000 20.0, 24.8
  const long units = Hkv * std::max<long>(R, (long)T * G / (16 * p.nt));
  p.gran_log2 = qg::kKv4GranuleLog2;
  if (most_keys <= (units > fill ? 256 : units >= 48 ? 1024 : 512))
    while ((1L << p.gran_log2) < most_keys) ++p.gran_log2;
  const long grans = std::max<long>(1, qg::ceil_div(most_keys, 1L << p.gran_log2));
  const long most = std::min(tiles, fill) * std::min<long>(Hkv, fill) * std::min(grans, fill);
  p.groups = (int)std::min(fill, most);
  p.part_floats = 16L * p.nt * (D + 2);
  return p;
}

long kv4_workspace_bytes(const Kv4Plan& p) { return p.groups * ((long)sizeof(qg::Kv4Head) + 2 * p.part_floats * (long)sizeof(float)); }

int check_kv4(int T, int R, int H, int Hkv, int D, int W, int page) {
  int rc = check_heads(H, Hkv);
  if (rc != QGEMM_OK) return rc;
  if (T < 0 || R < 0 || W < 0) return fail(QGEMM_EINVAL, "T, R and W must be >= 0 (got %d, %d, %d)", T, R, W);
  if (D != 64 && D != 128) return fail(QGEMM_EUNSUPPORTED, "head dimension must be 64 or 128 (got %d)", D);
  if (!good_page(page)) return fail(QGEMM_EINVAL, "page must be a power of two in [16, 1024] (got %d)", page);
  if ((long)T * H * D > 0x7fffffffL) return fail(QGEMM_EUNSUPPORTED, "T*H*D must be below 2^31");
  if ((long)W * page > (1 << 30)) return fail(QGEMM_EUNSUPPORTED, "W*page must be at most 2^30");
  if (R > (1 << 20)) return fail(QGEMM_EUNSUPPORTED, "more than 2^20 requests");
  // the kernel counts (16-row tile, key/value head, 128 keys) of all requests in 32 bits
  const double grans = (double)std::max<long>(1, qg::ceil_div((long)W * page, 1L << qg::kKv4GranuleLog2)) + qg::kKv4Start;
  if ((double)((long)T * (H / Hkv) / 16 + R) * Hkv * grans >= 2147483648.0)
    return fail(QGEMM_EUNSUPPORTED, "T, R, Hkv and W*page are too large together");
  return QGEMM_OK;
}

template <int D, int NT>
int launch_kv4(const qg::Kv4Args& a, bool join, hipStream_t s) {
  hipLaunchKernelGGL((qg::kv4_attn_kernel<D, NT>), dim3((unsigned)a.nwg), dim3(qg::kKv4Threads), 0, s, a);
  int rc = check_launch("qgemm_attention_kv4");
  if (rc != QGEMM_OK || !join) return rc;
  hipLaunchKernelGGL((qg::kv4_join_kernel<D, NT>), dim3((unsigned)a.nwg, 16 * NT / qg::kKv4JoinRows),
                     dim3(64 * qg::kKv4JoinRows), 0, s, a);
  return check_launch("qgemm_attention_kv4 (join)");
}

template <int D>
int launch_kv4_nt(const qg::Kv4Args& a, int nt, bool join, hipStream_t s) {
  if (nt == 1) return launch_kv4<D, 1>(a, join, s);
  return nt == 2 ? launch_kv4<D, 2>(a, join, s) : launch_kv4<D, qg::kKv4Wide>(a, join, s);
}

}  // namespace

extern "C" {

int qgemm_kv_plan(const int32_t* kv_len, const int32_t* q_len, int32_t* block_table, const int32_t* free_pages,
                  int32_t* cu_q, int32_t* positions, int32_t* slots, int32_t* total_len, int32_t* used, int R, int W,
                  int F, int page, int T, hipStream_t stream) {
  if (R < 0 || W < 0 || F < 0 || T < 0)
    return fail(QGEMM_EINVAL, "R, W, F and T must be >= 0 (got %d, %d, %d, %d)", R, W, F, T);
  if (!good_page(page)) return fail(QGEMM_EINVAL, "page must be a power of two in [16, 1024] (got %d)", page);
  if (R > qg::kPlanMaxR) return fail(QGEMM_EUNSUPPORTED, "R = %d exceeds the supported %d requests", R, qg::kPlanMaxR);
  if ((R && (!kv_len || !q_len || !total_len || (W && !block_table))) || !cu_q || !used || (F && !free_pages) ||
      (T && (!positions || !slots)))
    return fail(QGEMM_EINVAL, "null pointer argument");
  for (const void* p : {(const void*)kv_len, (const void*)q_len, (const void*)block_table, (const void*)free_pages,
                        (const void*)cu_q, (const void*)positions, (const void*)slots, (const void*)total_len, (const void*)used})
    if (!aligned(p, 4)) return fail(QGEMM_EALIGN, "the tables must be 4-byte aligned");
  const PlanTable written[] = {{"block_table", block_table, (int64_t)R * W}, {"cu_q", cu_q, R + 1}, {"positions", positions, T},
                               {"slots", slots, T},                          {"total_len", total_len, R}, {"used", used, 1}};
  const PlanTable read[] = {{"kv_len", kv_len, R}, {"q_len", q_len, R}, {"free_pages", free_pages, F}};
  int rc = check_apart(written, 6, read, 3);
  if (rc != QGEMM_OK) return rc;
  (void)hipGetLastError();
  const qg::PlanArgs a{kv_len, q_len, block_table, free_pages, cu_q, positions, slots, total_len, used,
                       R,      W,     F,           page_log2(page), T};
  const unsigned groups = (unsigned)std::max<long>(1, qg::ceil_div(T, qg::kPlanTokens));
  hipLaunchKernelGGL(qg::kv_plan_kernel, dim3(groups), dim3(qg::kPlanThreads), (size_t)R * 3 * sizeof(int32_t), stream, a);
  rc = check_launch("qgemm_kv_plan");
  return rc == QGEMM_OK ? ok() : rc;
}

int qgemm_rope_frequencies(double* inv_freq, float* gain, int rot, double base, int scaling, double factor, double low,
                           double high, double length) {
  if (!inv_freq || !gain) return fail(QGEMM_EINVAL, "null pointer argument");
  if (rot < 2 || rot > 2 * qg::kRopeMaxPairs || rot % 2 != 0)
    return fail(QGEMM_EINVAL, "rot must be even and in [2, %d] (got %d)", 2 * qg::kRopeMaxPairs, rot);
  if (!(base > 1.0) || !std::isfinite(base)) return fail(QGEMM_EINVAL, "base must be finite and > 1");
  if (scaling < QGEMM_ROPE_PLAIN || scaling > QGEMM_ROPE_YARN) return fail(QGEMM_EINVAL, "unknown scaling %d", scaling);
  if (scaling != QGEMM_ROPE_PLAIN && (!(factor >= 1.0) || !std::isfinite(factor)))
    return fail(QGEMM_EINVAL, "factor must be finite and >= 1");
  if (scaling == QGEMM_ROPE_LLAMA3 || scaling == QGEMM_ROPE_YARN) {
    if (!(low > 0.0) || !(high > low) || !std::isfinite(high) || !(length > 0.0) || !std::isfinite(length))
      return fail(QGEMM_EINVAL, "0 < low < high and length > 0 must hold, all finite");
  }
  const double two_pi = 6.283185307179586;
  auto between = [](double x) { return std::min(1.0, std::max(0.0, x)); };
  double from = 0, to = 0;             // YaRN: pairs up to `from` keep their frequency, from `to` on all is divided
  if (scaling == QGEMM_ROPE_YARN) {
    auto pair_of = [&](double turns) { return rot * std::log(length / (turns * two_pi)) / (2.0 * std::log(base)); };
    from = std::max(std::floor(pair_of(high)), 0.0);
    to = std::min(std::ceil(pair_of(low)), rot - 1.0);
  }
  for (int i = 0; i < rot / 2; ++i) {
    const double f = std::pow(base, -2.0 * i / rot);
    double keep = 1.0;
    if (scaling == QGEMM_ROPE_LINEAR) keep = 0.0;
    if (scaling == QGEMM_ROPE_LLAMA3) keep = between((length * f / two_pi - low) / (high - low));
    if (scaling == QGEMM_ROPE_YARN) keep = 1.0 - between((i - from) / (to > from ? to - from : 0.001));
    inv_freq[i] = scaling == QGEMM_ROPE_PLAIN ? f : keep * f + (1.0 - keep) * f / factor;
  }
  *gain = scaling == QGEMM_ROPE_YARN ? (float)(0.1 * std::log(factor) + 1.0) : 1.0f;
  return ok();
}

int qgemm_rope(const void* x, int x_type, const int32_t* positions, const double* inv_freq, void* y, int T, int heads,
               int rot_heads, int D, int rot, int64_t x_stride, int64_t y_stride, int interleaved, float gain,
               hipStream_t stream) {
  if (x_type != QGEMM_F32 && x_type != QGEMM_BF16) return fail(QGEMM_EINVAL, "unknown type %d of x", x_type);
  if (T < 0) return fail(QGEMM_EINVAL, "T must be >= 0 (got %d)", T);
  if (heads < 1 || rot_heads < 0 || rot_heads > heads)
    return fail(QGEMM_EINVAL, "heads must be >= 1 and rot_heads in [0, heads] (got %d, %d)", heads, rot_heads);
  if (D < 2 || D % 2 != 0 || D > 4096) return fail(QGEMM_EINVAL, "D must be even and in [2, 4096] (got %d)", D);
  if (rot < 2 || rot % 2 != 0 || rot > D) return fail(QGEMM_EINVAL, "rot must be even and in [2, D] (got %d)", rot);
  if (rot > 2 * qg::kRopeMaxPairs) return fail(QGEMM_EUNSUPPORTED, "rot = %d exceeds the supported %d", rot, 2 * qg::kRopeMaxPairs);
  if (interleaved != 0 && interleaved != 1) return fail(QGEMM_EINVAL, "interleaved must be 0 or 1 (got %d)", interleaved);
  if (!std::isfinite(gain)) return fail(QGEMM_EINVAL, "gain must be finite");
  if ((long)heads * D > (1 << 24)) return fail(QGEMM_EUNSUPPORTED, "heads*D must be at most 2^24");
  const int64_t row = (int64_t)heads * D;
  if (x_stride < row || y_stride < row) return fail(QGEMM_EINVAL, "rows of %lld elements overlap", (long long)row);
  if (T == 0) return ok();
  if (!x || !positions || !inv_freq || !y) return fail(QGEMM_EINVAL, "null pointer argument");
  const int xb = x_type == QGEMM_F32 ? 4 : 2;
  if (!aligned(x, xb) || !aligned(y, 2) || !aligned(positions, 4) || !aligned(inv_freq, 8))
    return fail(QGEMM_EALIGN, "x, y, positions and inv_freq must be aligned to their elements");
  if (x == y && (x_type != QGEMM_BF16 || x_stride != y_stride))
    return fail(QGEMM_EINVAL, "only bf16 rows can be rotated in place, at one stride");
  const bool wide = D % 16 == 0 && rot % 16 == 0 && aligned16(x) && aligned16(y) && x_stride * xb % 16 == 0 && y_stride * 2 % 16 == 0;
  qg::RopeArgs a{x, positions, inv_freq, static_cast<uint16_t*>(y), T, heads, rot_heads, D, rot, (long)x_stride, (long)y_stride, gain, 1, 1};
  // One token to a workgroup, or as many (up to four) as give each thread 16 elements while 1024 workgroups remain; below
  // 1024 tokens up to 16 workgroups share a token's heads. (8192 rows of 40 x 128: 46.7 us with one token, 48.8 with two,
  // 50.2 with four; 3000 rows of 24 x 64: 6.1, 5.2, 5.2.)
  const long items = std::max<long>(1, row / 16);
  if (T >= 1024) a.tokens = (int)std::max<long>(1, std::min({4L, qg::kRopeThreads / items, (long)T / 1024}));
  else a.parts = (int)std::min<long>(std::min(heads, 16), std::max<long>(1, items / qg::kRopeThreads));
  const long groups = qg::ceil_div(T, a.tokens) * a.parts;
  if (!qg::grid_fits(groups, qg::kRopeThreads)) return fail(QGEMM_EUNSUPPORTED, "too many workgroups");
  (void)hipGetLastError();
  auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(qg::kRopeThreads), 0, stream, a); };
  auto by_form = [&](auto type) {
    using TX = decltype(type);
    if (interleaved) wide ? launch(qg::rope_kernel<TX, true, true>) : launch(qg::rope_kernel<TX, true, false>);
    else wide ? launch(qg::rope_kernel<TX, false, true>) : launch(qg::rope_kernel<TX, false, false>);
  };
  if (x_type == QGEMM_F32) by_form(float{});
  else by_form(uint16_t{});
  const int rc = check_launch("qgemm_rope");
  return rc == QGEMM_OK ? ok() : rc;
}

int qgemm_kv4_store(const void* k, const void* v, const int32_t* slots, void* cache, int T, int Hkv, int D,
                    int64_t k_stride, int64_t v_stride, int pages, int page, hipStream_t stream) {
  int rc = check_cache(Hkv, D, pages, page);
  if (rc != QGEMM_OK) return rc;
  if (T < 0) return fail(QGEMM_EINVAL, "T must be >= 0 (got %d)", T);
  if (T == 0) return ok();
  if (!k || !v || !slots || !cache) return fail(QGEMM_EINVAL, "null pointer argument");
  rc = check_rows("k", k, k_stride, (int64_t)Hkv * D, 2);
  if (rc == QGEMM_OK) rc = check_rows("v", v, v_stride, (int64_t)Hkv * D, 2);
  if (rc != QGEMM_OK) return rc;
  if (!aligned16(cache) || !aligned(slots, 4))
    return fail(QGEMM_EALIGN, "the cache must be 16-byte and slots 4-byte aligned");
  qg::CacheArgs a{};
  a.k = static_cast<const uint16_t*>(k);
  a.v = static_cast<const uint16_t*>(v);
  a.cache = static_cast<uint8_t*>(cache);
  a.slots = slots;
  a.ks = k_stride;
  a.vs = v_stride;
  a.Hkv = Hkv;
  a.nslots = pages * page;
  a.units_log2 = D == 128 ? 4 : 3;
  a.lay = {D, page_log2(page)};
  const long n = ((long)T * 2 * Hkv) << a.units_log2;
  const long groups = qg::ceil_div(n, qg::kCacheThreads);
  if (!qg::grid_fits(groups, qg::kCacheThreads)) return fail(QGEMM_EUNSUPPORTED, "too many workgroups");
  a.n = (unsigned)n;
  (void)hipGetLastError();
  hipLaunchKernelGGL(qg::kv4_store_kernel, dim3((unsigned)groups), dim3(qg::kCacheThreads), 0, stream, a);
  rc = check_launch("qgemm_kv4_store");
  return rc == QGEMM_OK ? ok() : rc;
}

int qgemm_kv4_load(const void* cache, const int32_t* slots, void* k, void* v, int T, int Hkv, int D, int pages,
                   int page, hipStream_t stream) {
  int rc = check_cache(Hkv, D, pages, page);
  if (rc != QGEMM_OK) return rc;
  if (T < 0) return fail(QGEMM_EINVAL, "T must be >= 0 (got %d)", T);
  if (T == 0) return ok();
  if (!k || !v || !slots || !cache) return fail(QGEMM_EINVAL, "null pointer argument");
  if (!aligned16(cache) || !aligned16(k) || !aligned16(v) || !aligned(slots, 4))
    return fail(QGEMM_EALIGN, "the cache, k and v must be 16-byte and slots 4-byte aligned");
  qg::CacheArgs a{};
  a.ko = static_cast<uint16_t*>(k);
  a.vo = static_cast<uint16_t*>(v);
  a.cache = const_cast<uint8_t*>(static_cast<const uint8_t*>(cache));
  a.slots = slots;
  a.Hkv = Hkv;
  a.nslots = pages * page;
  a.units_log2 = D == 128 ? 4 : 3;
  a.lay = {D, page_log2(page)};
  const long n = ((long)T * 2 * Hkv) << a.units_log2;
  const long groups = qg::ceil_div(n, qg::kCacheThreads);
  if (!qg::grid_fits(groups, qg::kCacheThreads)) return fail(QGEMM_EUNSUPPORTED, "too many workgroups");
  a.n = (unsigned)n;
  (void)hipGetLastError();
  hipLaunchKernelGGL(qg::kv4_load_kernel, dim3((unsigned)groups), dim3(qg::kCacheThreads), 0, stream, a);
  rc = check_launch("qgemm_kv4_load");
  return rc == QGEMM_OK ? ok() : rc;
}

int qgemm_attention_packed(const void* q, const void* k, const void* v, const int32_t* cu, void* o, int T, int R,
                           int H, int Hkv, int D, int64_t q_stride, int64_t k_stride, int64_t v_stride,
                           int64_t o_stride, float scale, hipStream_t stream) {
  if (T < 0 || R < 0) return fail(QGEMM_EINVAL, "T and R must be >= 0 (got %d, %d)", T, R);
  int rc = check_heads(H, Hkv);
  if (rc != QGEMM_OK) return rc;
  if (D != 64 && D != 128) return fail(QGEMM_EUNSUPPORTED, "head dimension must be 64 or 128 (got %d)", D);
  qg::AttnArgs a{};
  rc = check_scale(scale, &a.sl2);
  if (rc != QGEMM_OK) return rc;
  if ((long)T * H * D > 0x7fffffffL) return fail(QGEMM_EUNSUPPORTED, "T*H*D must be below 2^31");
  if (T == 0 || R == 0) return ok();
  if (!q || !k || !v || !cu || !o) return fail(QGEMM_EINVAL, "null pointer argument");
  rc = check_rows("q", q, q_stride, (int64_t)H * D, 2);
  if (rc == QGEMM_OK) rc = check_rows("k", k, k_stride, (int64_t)Hkv * D, 2);
  if (rc == QGEMM_OK) rc = check_rows("v", v, v_stride, (int64_t)Hkv * D, 2);
  if (rc == QGEMM_OK) rc = check_rows("o", o, o_stride, (int64_t)H * D, 2);
  if (rc != QGEMM_OK) return rc;
  if (!aligned(cu, 4)) return fail(QGEMM_EALIGN, "cu must be 4-byte aligned");
  // the kernel counts a tensor's bytes in 32 bits, and reads (as zeros) up to a key block past its end
  if (std::max({q_stride, k_stride, v_stride}) > (0x7ffffff0L - 1) / ((long)T + 128))
    return fail(QGEMM_EUNSUPPORTED, "q, k and v must each span less than 4 GiB");
  const bool split = qg::attn_packed_split(D == 64, T, R, H);
  const long groups = (long)H * qg::ceil_div(T, split ? qg::kAttnBQ<true> : qg::kAttnBQ<false>);
  if (!qg::grid_fits(groups, qg::kAttnThreads)) return fail(QGEMM_EUNSUPPORTED, "too many workgroups");
  a.q = static_cast<const uint16_t*>(q);
  a.k = static_cast<const uint16_t*>(k);
  a.v = static_cast<const uint16_t*>(v);
  a.o = static_cast<uint16_t*>(o);
  a.B = 1;
  a.S = T;
  a.H = H;
  a.Hkv = Hkv;
  a.cu = cu;
  a.R = R;
  a.qs = q_stride;
  a.ks = k_stride;
  a.vs = v_stride;
  a.os = o_stride;
  (void)hipGetLastError();
  auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(qg::kAttnThreads), 0, stream, a); };
  if (D == 128) split ? launch(qg::attn_packed_kernel<128, true>) : launch(qg::attn_packed_kernel<128, false>);
  else split ? launch(qg::attn_packed_kernel<64, true>) : launch(qg::attn_packed_kernel<64, false>);
  rc = check_launch("qgemm_attention_packed");
  return rc == QGEMM_OK ? ok() : rc;
}

int qgemm_attention_kv4_workspace(int T, int R, int H, int Hkv, int D, int W, int page, int64_t* bytes) {
  if (!bytes) return fail(QGEMM_EINVAL, "null pointer argument");
  const int rc = check_kv4(T, R, H, Hkv, D, W, page);
  if (rc != QGEMM_OK) return rc;
  *bytes = T == 0 || R == 0 ? 0 : kv4_workspace_bytes(kv4_plan(T, R, H, Hkv, D, W, page));
  return ok();
}

int qgemm_attention_kv4(const void* q, const void* cache, const int32_t* block_table, const int32_t* kv_len,
                        const int32_t* cu_q, void* o, void* workspace, int64_t workspace_bytes, int T, int R, int H,
                        int Hkv, int D, int W, int pages, int page, int64_t q_stride, float scale, hipStream_t stream) {
  int rc = check_kv4(T, R, H, Hkv, D, W, page);
  if (rc != QGEMM_OK) return rc;
  rc = check_cache(Hkv, D, pages, page);
  if (rc != QGEMM_OK) return rc;
  qg::Kv4Args a{};
  rc = check_scale(scale, &a.sl2);
  if (rc != QGEMM_OK) return rc;
  if (!cu_q && T != R) return fail(QGEMM_EINVAL, "without cu_q every request has one token: T = %d, R = %d", T, R);
  if (T == 0 || R == 0) return ok();
  if (!q || !cache || (W && !block_table) || !kv_len || !o || !workspace) return fail(QGEMM_EINVAL, "null pointer argument");
  rc = check_rows("q", q, q_stride, (int64_t)H * D, 2);
  if (rc != QGEMM_OK) return rc;
  if (!aligned16(cache) || !aligned16(o) || !aligned16(workspace))
    return fail(QGEMM_EALIGN, "the cache, o and the workspace must be 16-byte aligned");
  if (!aligned(block_table, 4) || !aligned(kv_len, 4) || !aligned(cu_q, 4))
    return fail(QGEMM_EALIGN, "the tables must be 4-byte aligned");
  const Kv4Plan plan = kv4_plan(T, R, H, Hkv, D, W, page);
  if (workspace_bytes < kv4_workspace_bytes(plan))
    return fail(QGEMM_EINVAL, "a workspace of %lld bytes is needed (got %lld)", (long long)kv4_workspace_bytes(plan),
                (long long)workspace_bytes);
  a.q = static_cast<const uint16_t*>(q);
  a.cache = static_cast<const uint8_t*>(cache);
  a.table = block_table;
  a.kv_len = kv_len;
  a.cu = cu_q;
  a.o = static_cast<uint16_t*>(o);
  a.head = static_cast<qg::Kv4Head*>(workspace);
  a.part = reinterpret_cast<float*>(a.head + plan.groups);
  a.T = T;
  a.R = R;
  a.H = H;
  a.Hkv = Hkv;
  a.W = W;
  a.pages = pages;
  a.page_log2 = page_log2(page);
  a.nwg = plan.groups;
  a.gran_log2 = plan.gran_log2;
  a.qs = q_stride;
  const bool join = (long)W * page > (1L << plan.gran_log2);      // else every unit is one granule
  (void)hipGetLastError();
  rc = D == 128 ? launch_kv4_nt<128>(a, plan.nt, join, stream) : launch_kv4_nt<64>(a, plan.nt, join, stream);
  return rc == QGEMM_OK ? ok() : rc;
}

}  // extern "C"
