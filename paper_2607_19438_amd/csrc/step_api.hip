// C entry points of serving steps with many continuations of a prompt and many tenants: attention over a cache whose
// first keys requests share, the selection of a beam search with the tables and pages that follow it, and low-rank
// adapters beside a projection (declarations and contracts in include/qgemm.h). A source of its own, and so a code
// object of its own.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "../../include/qgemm.h"
#include "adapter_kernels.hpp"
#include "api_checks.hpp"
#include "attn_shared.hpp"
#include "beam_kernels.hpp"
#include "tile_rules.hpp"

namespace {

constexpr long kCUs = 256;

long round16(long n) { return (n + 15) & -16L; }

// ---------------------------------------------------------------------------
// attention over shared keys
// ---------------------------------------------------------------------------

struct SharedPlan {
  int np, nt;         // 16-row tiles of a unit over shared keys, and of one behind them
  int cost;           // of a granule over shared keys, in sixteenths of one behind them
  int groups;         // workgroups
  long part_floats;
  long at_rows, at_part, at_whole, at_ml, bytes;       // of the workspace
};

SharedPlan shared_plan(int T, int R, int Gn, int H, int Hkv, int D, int W, int page) {
  const long G = H / Hkv;
  const long rows = qg::ceil_div((long)T * G, R), group_rows = qg::ceil_div((long)T * G, std::max(Gn, 1));
  SharedPlan p{};
  // Units over shared keys take pairs of 16-row tiles, and wide ones only for many rows: each part of a wide tile is 64 KiB,
  // and a few tiles over long keys are cut into many parts. (us, pairs and wide: 64 requests behind 7919 keys, 32/8 heads of 128
  // 34.3, 34.0; the same with D = 64 25.7, 27.0; 24 x 8 beams, 32/4 heads of 64 25.5, 29.3; 128 requests, 32/4 heads of 128 36.4,
  // 39.0; 192 with 32/8 63.9, 58.8; 64 of 5 tokens 69.4, 59.4.)
  const bool wide = group_rows >= 256 && (long)T * G / (16 * qg::kKv4Wide) * Hkv >= 40;
  p.nt = rows <= 16 ? 1 : rows >= 512 ? qg::kKv4Wide : 2;
  p.np = p.nt == qg::kKv4Wide || wide ? qg::kKv4Wide : group_rows <= 16 && p.nt == 1 ? 1 : 2;
  // What a granule over shared keys takes longer: measured for pairs against single tiles with 16, 20, 24, 28: 24 x 8 beams 26.7,
  // 25.8, 25.5, 25.8; 64 requests 36.6, 34.9, 34.6, 34.3; for wide against single ones with 24, 32, 48: 192 requests 62.6, 64.4,
  // 58.8; wide against pairs: 64 of 5 tokens 61.9, 59.4, 62.2.
  p.cost = p.np == p.nt ? 16 : p.np == 2 ? 24 : p.nt == 1 ? 48 : 32;
  const int most = std::max(p.np, p.nt);
  const long per_cu = most == qg::kKv4Wide ? 2 : (D == 128 ? 3 : 4) - (most - 1);
  const long fill = kCUs * per_cu;
  const long grans = std::max<long>(1, qg::ceil_div((long)W * page, 1L << qg::kKv4GranuleLog2));
  const double work = (double)Hkv * (((double)T * G / (16 * p.np) + Gn) + ((double)T * G / (16 * p.nt) + R)) * (double)grans;
  p.groups = (int)std::max(2.0, std::min((double)fill, work));
  p.part_floats = 16L * most * (D + 2);
  p.at_rows = round16(sizeof(qg::SharedCut));
  p.at_part = p.at_rows + round16((long)R * sizeof(qg::SharedRow));
  p.at_whole = p.at_part + p.groups * 2L * p.part_floats * (long)sizeof(float);
  p.at_ml = p.at_whole + 2L * T * H * D * (long)sizeof(float);
  p.bytes = round16(p.at_ml + 2L * T * H * 2 * (long)sizeof(float));
  return p;
}

int check_shared(int T, int R, int Gn, int H, int Hkv, int D, int W, int page) {
  int rc = check_heads(H, Hkv);
  if (rc != QGEMM_OK) return rc;
  if (T < 0 || R < 0 || Gn < 0 || W < 0) return fail(QGEMM_EINVAL, "T, R, G and W must be >= 0 (got %d, %d, %d, %d)", T, R, Gn, W);
  if (D != 64 && D != 128) return fail(QGEMM_EUNSUPPORTED, "head dimension must be 64 or 128 (got %d)", D);
  if (!good_page(page)) return fail(QGEMM_EINVAL, "page must be a power of two in [16, 1024] (got %d)", page);
  if ((long)T * H * D > 0x7fffffffL) return fail(QGEMM_EUNSUPPORTED, "T*H*D must be below 2^31");
  if ((long)W * page > (1 << 30)) return fail(QGEMM_EUNSUPPORTED, "W*page must be at most 2^30");
  if (R > qg::kSharedMaxR || Gn > qg::kSharedMaxR) return fail(QGEMM_EUNSUPPORTED, "more than %d requests or groups", qg::kSharedMaxR);
  // the kernel counts (16-row tile, key/value head, 128 keys) of all units of a kind in 32 bits
  const double grans = (double)std::max<long>(1, qg::ceil_div((long)W * page, 1L << qg::kKv4GranuleLog2)) + qg::kKv4Start;
  if ((double)((long)T * (H / Hkv) / 16 + std::max(R, Gn)) * Hkv * grans >= 2147483648.0)
    return fail(QGEMM_EUNSUPPORTED, "T, R, Hkv and W*page are too large together");
  return QGEMM_OK;
}

template <int D, int NP, int NT>
int launch_shared(const qg::SharedArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((qg::kv4_shared_kernel<D, NP, NT>), dim3((unsigned)a.k.nwg), dim3(qg::kKv4Threads), (size_t)qg::shared_lds(a.k.R, a.Gn) * sizeof(int32_t), s, a);
  int rc = check_launch("qgemm_attention_kv4_shared");
  if (rc != QGEMM_OK) return rc;
  const long groups = qg::ceil_div((long)a.k.T * a.k.H, qg::kSharedJoinRows);
  hipLaunchKernelGGL((qg::kv4_shared_join_kernel<D, NP, NT>), dim3((unsigned)groups), dim3(64 * qg::kSharedJoinRows), 0, s, a);
  return check_launch("qgemm_attention_kv4_shared (join)");
}

template <int D>
int launch_shared_form(const qg::SharedArgs& a, int np, int nt, hipStream_t s) {
  constexpr int kWide = qg::kKv4Wide;
  if (nt == kWide) return launch_shared<D, kWide, kWide>(a, s);
  if (nt == 2) return np == kWide ? launch_shared<D, kWide, 2>(a, s) : launch_shared<D, 2, 2>(a, s);
  return np == kWide ? launch_shared<D, kWide, 1>(a, s) : np == 2 ? launch_shared<D, 2, 1>(a, s) : launch_shared<D, 1, 1>(a, s);
}

// ---------------------------------------------------------------------------
// beams
// ---------------------------------------------------------------------------

struct BeamPlan {
  int pieces, piece;
  long bytes;
};

// A row goes to as many workgroups as leave each of its waves a step, while 768 of all rows are not passed, nor the 1024
// candidates that the second kernel takes fast; of more rows than that to three, so that the last workgroups are short.
// (us, both kernels, by pieces: 4 rows of 32000, K = 4: 2 12.8, 4 11.2, 8 10.5; 85 of 50021, K = 10: 1 26.1, 3 17.4, 7 15.8,
// 13 16.6; 384 of 128000, K = 16: 1 58.0, 2 47.3, 3 50.8, 8 53.1; 1200 of 32000, K = 8: 1 42.1, 3 39.5, 8 48.6; 8 of
// 128000, K = 16: 4 21.3, 8 18.6, 16 19.4, 32 24.1.)
BeamPlan beam_plan(int R, int B, int V, int K) {
  BeamPlan p{};
  const long rows = (long)R * B;
  long pieces = std::min<long>(qg::ceil_div(V, qg::kBeamPiece), rows <= 768 ? 768 / rows : 3);
  pieces = std::max<long>(1, std::min<long>(pieces, qg::kBeamMost / ((long)B * K)));
  p.piece = (int)(qg::ceil_div(qg::ceil_div(V, pieces), qg::kBeamPiece) * qg::kBeamPiece);
  p.pieces = (int)qg::ceil_div(V, p.piece);
  p.bytes = rows * p.pieces * ((long)sizeof(qg::BeamStat) + (long)K * (long)sizeof(uint64_t));
  return p;
}

int check_beams(int R, int B, int V, int K) {
  if (R < 0) return fail(QGEMM_EINVAL, "R must be >= 0 (got %d)", R);
  if (B < 1 || V < 1 || K < 1) return fail(QGEMM_EINVAL, "B, V and K must be >= 1 (got %d, %d, %d)", B, V, K);
  if (B > qg::kBeamMaxB) return fail(QGEMM_EUNSUPPORTED, "B = %d exceeds the supported %d beams", B, qg::kBeamMaxB);
  if (K > qg::kBeamMaxK) return fail(QGEMM_EUNSUPPORTED, "K = %d exceeds the supported %d candidates", K, qg::kBeamMaxK);
  if ((long)R * B > (1 << 20)) return fail(QGEMM_EUNSUPPORTED, "more than 2^20 beams in all");
  if (V > (1 << 30)) return fail(QGEMM_EUNSUPPORTED, "V must be at most 2^30");
  return QGEMM_OK;
}

// int32 entries of the workspace: a count for each workgroup, and room for all of its columns' pages
int64_t reorder_entries(int64_t blocks, int B) { return blocks * (1 + (int64_t)qg::kReorderThreads * B); }

int reorder_blocks(int W) { return (int)std::max<long>(1, qg::ceil_div(W, qg::kReorderThreads)); }

int check_reorder(int R, int B, int W, int F, int Q, int page) {
  if (R < 0 || W < 0 || F < 0 || Q < 0) return fail(QGEMM_EINVAL, "R, W, F and Q must be >= 0 (got %d, %d, %d, %d)", R, W, F, Q);
  if (B < 1) return fail(QGEMM_EINVAL, "B must be >= 1 (got %d)", B);
  if (B > qg::kBeamMaxB) return fail(QGEMM_EUNSUPPORTED, "B = %d exceeds the supported %d beams", B, qg::kBeamMaxB);
  if (!good_page(page)) return fail(QGEMM_EINVAL, "page must be a power of two in [16, 1024] (got %d)", page);
  if ((long)R * B > qg::kReorderMaxRows) return fail(QGEMM_EUNSUPPORTED, "R*B = %ld exceeds the supported %d rows", (long)R * B, qg::kReorderMaxRows);
  if ((long)R * B * W > 0x7fffffffL) return fail(QGEMM_EUNSUPPORTED, "R*B*W must be below 2^31");
  return QGEMM_OK;
}

// ---------------------------------------------------------------------------
// adapters
// ---------------------------------------------------------------------------

struct AdapterPlan {
  int mt_down, jt, splits, k_split, lists;
  int mt_up, nt, s, chunks;
  long at_mid, bytes;
};

AdapterPlan adapter_plan(int M, int N, int K, int r) {
  AdapterPlan p{};
  // mid: K is split over workgroups while they are few; the second kernel adds the parts up, each of its workgroups those of
  // its rows. (us of the first kernel and the second, for splits of 1, 2, 4; K = 2048, 8192 columns: 96 rows, rank 32 9.8, 7.3,
  // 6.9, and 13.0, 13.3, 14.2; 2048 rows, rank 16 7.0, 6.4, 6.8 and 30.4, 30.8, 31.5; 2500 rows, rank 64 15.1, 10.1, 10.0 and
  // 41.9, 44.7, 48.9; 8500 rows, rank 64 25.5, 22.0, 23.3 and 130, 135, 152; each kernel by itself, again
  // and again.) Tiles of 32 rows read A half as often (8500 rows, rank 64 26.2 and 38.6 us; 1252 rows, two splits 9.8 and
  // 12.6), those of 16 have fewer adapters.
  p.mt_down = M > 1024 ? 2 : 1;
  p.jt = r <= 16 ? 1 : r <= 32 ? 2 : 4;
  // A tile's adapters side by side: each row may have its own (96 rows, 64 adapters: 1, 4, 16 at once 35.8, 11.9, 6.9 us); of
  // prompts a tile has two or three where they meet, and the kernel waits for it (1252 rows of 14 prompts, rank 64: 1, 2, 4 at
  // once 18.6, 13.5, 12.6 us).
  p.lists = M <= 256 ? 16 : 4;
  const long tiles = qg::ceil_div(r, 16L * p.jt);
  const long want = M <= 256 ? 256 / (M * tiles) : M <= 4096 ? 2 : 1;
  p.splits = (int)std::max<long>(1, std::min<long>({4, want, K / 256}));
  p.k_split = (int)(qg::ceil_div(qg::ceil_div(K, p.splits), qg::kAdRun) * qg::kAdRun);
  p.splits = (int)qg::ceil_div(K, p.k_split);
  // y: of few rows 16 columns to a wave and eight adapters at once (96 rows with 64 adapters, 8192 columns: 10.2 us, with 64
  // columns 14.7 and 11.7 for one and two at once; 64 rows with 32, 4096 columns 5.6, with two at once 6.4). Else tiles of 32 by
  // 32, two of them to a wave in turn where that leaves four workgroups to a CU (8500 rows of 8192, rank 64: 1, 2, 4 in turn 141,
  // 129, 133 us, with tiles of 16 rows 32% slower at two; 1252 rows, rank 64 26.2, 24.8, 26.8). At a rank up to 32 the
  // operands are soon made, and few tiles are of 16 rows (1252 rows of 5003, rank 8 14.0, 12.2 us, of 32 rows 15.3, 13.3; 540
  // rows of 4096, rank 16 6.3 and 7.0; but 2048 rows of 8192 31.2 and 30.4).
  const bool small = r <= 32 && qg::ceil_div(M, 32) * qg::ceil_div(N, 256) < 4 * kCUs;
  p.nt = M <= 256 ? 1 : 2;
  p.mt_up = M <= 256 || small ? 1 : 2;
  p.chunks = M > 256 && qg::ceil_div(M, 16L * p.mt_up) * qg::ceil_div(N, 256) >= 4 * kCUs ? 2 : 1;
  p.s = r <= 32 ? 1 : r <= 64 ? 2 : 4;
  p.at_mid = round16((long)M * (long)sizeof(int32_t));
  p.bytes = p.at_mid + (long)p.splits * M * r * (long)sizeof(float);
  return p;
}

int check_adapters(int M, int N, int K, int r, int n, int R) {
  if (M < 0 || R < 0) return fail(QGEMM_EINVAL, "M and R must be >= 0 (got %d, %d)", M, R);
  if (N < 1 || n < 1) return fail(QGEMM_EINVAL, "N and n must be >= 1 (got %d, %d)", N, n);
  if (K < 8 || K % 8 != 0) return fail(QGEMM_EINVAL, "K must be a positive multiple of 8 (got %d)", K);
  if (r < 8 || r % 8 != 0) return fail(QGEMM_EINVAL, "the rank must be a positive multiple of 8 (got %d)", r);
  if (r > qg::kAdMaxRank) return fail(QGEMM_EUNSUPPORTED, "rank %d exceeds the supported %d", r, qg::kAdMaxRank);
  if (N > (1 << 28) || K > (1 << 28) || R > (1 << 28)) return fail(QGEMM_EUNSUPPORTED, "N, K and R must be at most 2^28");
  if (M > (1 << 25)) return fail(QGEMM_EUNSUPPORTED, "M must be at most 2^25");        // the first kernel's grid, with its lists and rank tiles
  return QGEMM_OK;
}

}  // namespace

extern "C" {

int qgemm_attention_kv4_shared_workspace(int T, int R, int G, int H, int Hkv, int D, int W, int page, int64_t* bytes) {
  if (!bytes) return fail(QGEMM_EINVAL, "null pointer argument");
  const int rc = check_shared(T, R, G, H, Hkv, D, W, page);
  if (rc != QGEMM_OK) return rc;
  *bytes = T == 0 || R == 0 ? 0 : shared_plan(T, R, G, H, Hkv, D, W, page).bytes;
  return ok();
}

int qgemm_attention_kv4_shared(const void* q, const void* cache, const int32_t* block_table, const int32_t* kv_len,
                               const int32_t* cu_q, const int32_t* groups, const int32_t* prefix_len, void* o, void* workspace,
                               int64_t workspace_bytes, int T, int R, int G, int H, int Hkv, int D, int W, int pages, int page,
                               int64_t q_stride, float scale, hipStream_t stream) {
  int rc = check_shared(T, R, G, H, Hkv, D, W, page);
  if (rc != QGEMM_OK) return rc;
  rc = check_cache(Hkv, D, pages, page);
  if (rc != QGEMM_OK) return rc;
  qg::SharedArgs a{};
  rc = check_scale(scale, &a.k.sl2);
  if (rc != QGEMM_OK) return rc;
  if (!cu_q && T != R) return fail(QGEMM_EINVAL, "without cu_q every request has one token: T = %d, R = %d", T, R);
  if (T == 0 || R == 0) return ok();
  if (!q || !cache || (W && !block_table) || !kv_len || !groups || (G && !prefix_len) || !o || !workspace)
    return fail(QGEMM_EINVAL, "null pointer argument");
  rc = check_rows("q", q, q_stride, (int64_t)H * D, 2);
  if (rc != QGEMM_OK) return rc;
  if (!aligned16(cache) || !aligned16(o) || !aligned16(workspace))
    return fail(QGEMM_EALIGN, "the cache, o and the workspace must be 16-byte aligned");
  if (!aligned(block_table, 4) || !aligned(kv_len, 4) || !aligned(cu_q, 4) || !aligned(groups, 4) || !aligned(prefix_len, 4))
    return fail(QGEMM_EALIGN, "the tables must be 4-byte aligned");
  const SharedPlan plan = shared_plan(T, R, G, H, Hkv, D, W, page);
  if (workspace_bytes < plan.bytes)
    return fail(QGEMM_EINVAL, "a workspace of %lld bytes is needed (got %lld)", (long long)plan.bytes, (long long)workspace_bytes);
  char* ws = static_cast<char*>(workspace);
  a.k.q = static_cast<const uint16_t*>(q);
  a.k.cache = static_cast<const uint8_t*>(cache);
  a.k.table = block_table;
  a.k.kv_len = kv_len;
  a.k.cu = cu_q;
  a.k.o = static_cast<uint16_t*>(o);
  a.k.part = reinterpret_cast<float*>(ws + plan.at_part);
  a.k.T = T;
  a.k.R = R;
  a.k.H = H;
  a.k.Hkv = Hkv;
  a.k.W = W;
  a.k.pages = pages;
  a.k.page_log2 = page_log2(page);
  a.k.nwg = plan.groups;
  a.k.gran_log2 = qg::kKv4GranuleLog2;
  a.k.qs = q_stride;
  a.groups = groups;
  a.prefix = prefix_len;
  a.Gn = G;
  a.cost = plan.cost;
  a.cut = reinterpret_cast<qg::SharedCut*>(ws);
  a.rows = reinterpret_cast<qg::SharedRow*>(ws + plan.at_rows);
  a.whole = reinterpret_cast<float*>(ws + plan.at_whole);
  a.whole_ml = reinterpret_cast<float*>(ws + plan.at_ml);
  a.part_floats = plan.part_floats;
  (void)hipGetLastError();
  rc = D == 128 ? launch_shared_form<128>(a, plan.np, plan.nt, stream) : launch_shared_form<64>(a, plan.np, plan.nt, stream);
  return rc == QGEMM_OK ? ok() : rc;
}

int qgemm_beam_select_workspace(int R, int B, int V, int K, int64_t* bytes) {
  if (!bytes) return fail(QGEMM_EINVAL, "null pointer argument");
  const int rc = check_beams(R, B, V, K);
  if (rc != QGEMM_OK) return rc;
  *bytes = R == 0 ? 0 : beam_plan(R, B, V, K).bytes;
  return ok();
}

int qgemm_beam_select(const void* logits, int type, const float* scores, const uint8_t* finished, float* out_scores,
                      int32_t* out_parents, int32_t* out_tokens, void* workspace, int64_t workspace_bytes, int R, int B, int V,
                      int K, int64_t stride, int end, hipStream_t stream) {
  int rc = check_beams(R, B, V, K);
  if (rc != QGEMM_OK) return rc;
  if (type != QGEMM_F32 && type != QGEMM_BF16) return fail(QGEMM_EINVAL, "unknown type %d of the logits", type);
  if (end < 0 || end >= V) return fail(QGEMM_EINVAL, "end must be a token in [0, V) (got %d)", end);
  if (stride < V) return fail(QGEMM_EINVAL, "rows of %d logits overlap at stride %lld", V, (long long)stride);
  if (R == 0) return ok();
  if (!logits || !scores || !out_scores || !out_parents || !out_tokens || !workspace) return fail(QGEMM_EINVAL, "null pointer argument");
  if (!aligned(logits, type == QGEMM_F32 ? 4 : 2) || !aligned(scores, 4) || !aligned(out_scores, 4) || !aligned(out_parents, 4) ||
      !aligned(out_tokens, 4))
    return fail(QGEMM_EALIGN, "logits, scores and outputs must be aligned to their elements");
  if (!aligned16(workspace)) return fail(QGEMM_EALIGN, "the workspace must be 16-byte aligned");
  const BeamPlan plan = beam_plan(R, B, V, K);
  if (workspace_bytes < plan.bytes)
    return fail(QGEMM_EINVAL, "a workspace of %lld bytes is needed (got %lld)", (long long)plan.bytes, (long long)workspace_bytes);
  const long rows = (long)R * B;
  if (!qg::grid_fits(rows * plan.pieces, qg::kBeamThreads)) return fail(QGEMM_EUNSUPPORTED, "too many workgroups");
  qg::BeamArgs a{};
  a.x = logits;
  a.scores = scores;
  a.finished = finished;
  a.out_scores = out_scores;
  a.out_beams = out_parents;
  a.out_tokens = out_tokens;
  a.stat = static_cast<qg::BeamStat*>(workspace);
  a.cand = reinterpret_cast<uint64_t*>(a.stat + rows * plan.pieces);
  a.stride = stride;
  a.R = R;
  a.B = B;
  a.V = V;
  a.K = K;
  a.pieces = plan.pieces;
  a.piece = plan.piece;
  a.end = end;
  while (a.pieces_log2 < 6 && (1 << a.pieces_log2) < plan.pieces) ++a.pieces_log2;
  const long per = (long)plan.pieces * K;
  a.per_inv = per == 1 ? 0u : (uint32_t)(((1L << 32) + per - 1) / per);
  (void)hipGetLastError();
  const dim3 grid((unsigned)(rows * plan.pieces)), block(qg::kBeamThreads);
  if (type == QGEMM_F32) hipLaunchKernelGGL(qg::beam_rows_kernel<float>, grid, block, 0, stream, a);
  else hipLaunchKernelGGL(qg::beam_rows_kernel<uint16_t>, grid, block, 0, stream, a);
  rc = check_launch("qgemm_beam_select");
  if (rc != QGEMM_OK) return rc;
  if ((long)B * plan.pieces * K <= qg::kBeamMost) hipLaunchKernelGGL(qg::beam_join_kernel<qg::kBeamMost>, dim3((unsigned)R), block, 0, stream, a);
  else hipLaunchKernelGGL((qg::beam_join_kernel<qg::kBeamMaxB * qg::kBeamMaxK>), dim3((unsigned)R), block, 0, stream, a);
  rc = check_launch("qgemm_beam_select (join)");
  return rc == QGEMM_OK ? ok() : rc;
}

int qgemm_kv_reorder_workspace(int R, int B, int W, int64_t* bytes) {
  if (!bytes) return fail(QGEMM_EINVAL, "null pointer argument");
  const int rc = check_reorder(R, B, W, 0, 0, 16);
  if (rc != QGEMM_OK) return rc;
  *bytes = reorder_entries((int64_t)R * reorder_blocks(W), B) * (int64_t)sizeof(int32_t);
  return ok();
}

int qgemm_kv_reorder(const int32_t* block_table, const int32_t* kv_len, const int32_t* parents, const int32_t* free_pages,
                     const int32_t* keep, int32_t* new_table, int32_t* new_len, int32_t* src, int32_t* dst, int32_t* used,
                     int32_t* released, int32_t* n_released, void* workspace, int64_t workspace_bytes, int R, int B, int W, int F,
                     int Q, int page, hipStream_t stream) {
  int rc = check_reorder(R, B, W, F, Q, page);
  if (rc != QGEMM_OK) return rc;
  if (R == 0) return ok();
  if (!kv_len || !parents || (W && (!block_table || !new_table)) || (F && !free_pages) || !new_len || !src || !dst || !used ||
      (Q && !released) || !n_released || !workspace)
    return fail(QGEMM_EINVAL, "null pointer argument");
  for (const void* p : {(const void*)block_table, (const void*)kv_len, (const void*)parents, (const void*)free_pages, (const void*)keep,
                        (const void*)new_table, (const void*)new_len, (const void*)src, (const void*)dst, (const void*)used,
                        (const void*)released, (const void*)n_released, (const void*)workspace})
    if (!aligned(p, 4)) return fail(QGEMM_EALIGN, "the tables must be 4-byte aligned");
  const int64_t rows = (int64_t)R * B, blocks = reorder_blocks(W), counts = R * blocks;
  const int64_t entries = reorder_entries(counts, B);
  if (workspace_bytes < entries * (int64_t)sizeof(int32_t))
    return fail(QGEMM_EINVAL, "a workspace of %lld bytes is needed (got %lld)", (long long)(entries * 4), (long long)workspace_bytes);
  const PlanTable written[] = {{"new_table", new_table, rows * W}, {"new_len", new_len, rows}, {"src", src, rows}, {"dst", dst, rows}, {"used", used, 1},
                               {"released", released, Q}, {"n_released", n_released, 1}, {"workspace", static_cast<int32_t*>(workspace), entries}};
  const PlanTable read[] = {{"block_table", block_table, rows * W}, {"kv_len", kv_len, rows}, {"parents", parents, rows},
                            {"free_pages", free_pages, F}, {"keep", keep, keep ? R : 0}};
  rc = check_apart(written, 8, read, 5);
  if (rc != QGEMM_OK) return rc;
  const qg::ReorderSplit split = qg::reorder_split(R, blocks);
  qg::ReorderArgs a{block_table, kv_len, parents, free_pages, keep, new_table, new_len, src, dst, used, released, n_released,
                    static_cast<int32_t*>(workspace), static_cast<int32_t*>(workspace) + counts, R, B, W, F, Q, page_log2(page), (int)blocks,
                    (int)split.each, (int)split.parts, (int)split.release_each, (int)split.release};
  if (!qg::grid_fits(R * split.parts, qg::kReorderThreads)) return fail(QGEMM_EUNSUPPORTED, "too many workgroups");
  (void)hipGetLastError();
  const dim3 block(qg::kReorderThreads);
  const size_t lds = (size_t)B * qg::kReorderThreads * sizeof(int32_t);
  const dim3 grid((unsigned)(R * split.parts)), release((unsigned)split.release);
  if (split.each == 1) hipLaunchKernelGGL(qg::kv_reorder_kernel<false>, grid, block, lds, stream, a);
  else hipLaunchKernelGGL(qg::kv_reorder_kernel<true>, grid, block, lds, stream, a);
  rc = check_launch("qgemm_kv_reorder");
  if (rc != QGEMM_OK) return rc;
  if (split.release_each == 1) hipLaunchKernelGGL(qg::kv_release_kernel<false>, release, block, 0, stream, a);
  else hipLaunchKernelGGL(qg::kv_release_kernel<true>, release, block, 0, stream, a);
  rc = check_launch("qgemm_kv_reorder (released pages)");
  return rc == QGEMM_OK ? ok() : rc;
}

int qgemm_kv4_copy(void* cache, const int32_t* src, const int32_t* dst, int n, int Hkv, int D, int pages, int page, hipStream_t stream) {
  int rc = check_cache(Hkv, D, pages, page);
  if (rc != QGEMM_OK) return rc;
  if (n < 0) return fail(QGEMM_EINVAL, "n must be >= 0 (got %d)", n);
  if (n == 0) return ok();
  if (!cache || !src || !dst) return fail(QGEMM_EINVAL, "null pointer argument");
  if (!aligned16(cache) || !aligned(src, 4) || !aligned(dst, 4))
    return fail(QGEMM_EALIGN, "the cache must be 16-byte and the lists 4-byte aligned");
  const qg::CopyArgs a{static_cast<uint8_t*>(cache), src, dst, (long)Hkv * page * (D + D / 16), n, pages};
  const long parts = qg::ceil_div(a.page_bytes, qg::kCopyBytes);
  if (parts > 65535 || !qg::grid_fits(n * parts, qg::kCopyThreads)) return fail(QGEMM_EUNSUPPORTED, "too many workgroups");
  (void)hipGetLastError();
  hipLaunchKernelGGL(qg::kv4_copy_kernel, dim3((unsigned)n, (unsigned)parts), dim3(qg::kCopyThreads), 0, stream, a);
  rc = check_launch("qgemm_kv4_copy");
  return rc == QGEMM_OK ? ok() : rc;
}

int qgemm_adapters_workspace(int M, int N, int K, int r, int64_t* bytes) {
  if (!bytes) return fail(QGEMM_EINVAL, "null pointer argument");
  const int rc = check_adapters(M, N, K, r, 1, 0);
  if (rc != QGEMM_OK) return rc;
  *bytes = M == 0 ? 0 : adapter_plan(M, N, K, r).bytes;
  return ok();
}

int qgemm_adapters(const void* x, const void* a_w, const void* b_w, const int32_t* ids, const int32_t* cu_q, const float* gain, float* y,
                   void* workspace, int64_t workspace_bytes, int M, int N, int K, int r, int n, int R, int64_t x_stride, int64_t y_stride,
                   hipStream_t stream) {
  int rc = check_adapters(M, N, K, r, n, R);
  if (rc != QGEMM_OK) return rc;
  if (!cu_q && M != R) return fail(QGEMM_EINVAL, "without cu_q every request has one row: M = %d, R = %d", M, R);
  if (M == 0 || R == 0) return ok();
  if (!x || !a_w || !b_w || !ids || !y || !workspace) return fail(QGEMM_EINVAL, "null pointer argument");
  rc = check_rows("x", x, x_stride, K, 2);
  if (rc != QGEMM_OK) return rc;
  if (!aligned16(a_w) || !aligned16(b_w) || !aligned16(workspace)) return fail(QGEMM_EALIGN, "a, b and the workspace must be 16-byte aligned");
  if (!aligned(ids, 4) || !aligned(cu_q, 4) || !aligned(gain, 4) || !aligned(y, 4))
    return fail(QGEMM_EALIGN, "ids, cu_q, gain and y must be 4-byte aligned");
  if (y_stride < N) return fail(QGEMM_EINVAL, "rows of %d columns overlap at stride %lld", N, (long long)y_stride);
  const AdapterPlan plan = adapter_plan(M, N, K, r);
  if (workspace_bytes < plan.bytes)
    return fail(QGEMM_EINVAL, "a workspace of %lld bytes is needed (got %lld)", (long long)plan.bytes, (long long)workspace_bytes);
  qg::AdapterArgs g{};
  g.x = static_cast<const uint16_t*>(x);
  g.a = static_cast<const uint16_t*>(a_w);
  g.b = static_cast<const uint16_t*>(b_w);
  g.ids = ids;
  g.cu = cu_q;
  g.gain = gain;
  g.y = y;
  g.row_id = static_cast<int32_t*>(workspace);
  g.mid = reinterpret_cast<float*>(static_cast<char*>(workspace) + plan.at_mid);
  g.xs = x_stride;
  g.ys = y_stride;
  g.M = M;
  g.N = N;
  g.K = K;
  g.r = r;
  g.n = n;
  g.R = R;
  g.splits = plan.splits;
  g.k_split = plan.k_split;
  g.lists = plan.lists;
  g.chunks = plan.chunks;
  const long down = qg::ceil_div(M, 16L * plan.mt_down) * plan.lists * plan.splits * qg::ceil_div(r, 16L * plan.jt);
  const long up = qg::ceil_div(M, 16L * plan.mt_up) * qg::ceil_div(N, 16L * plan.nt * plan.chunks * qg::kAdWaves);
  if (!qg::grid_fits(down, qg::kAdThreads) || !qg::grid_fits(up, qg::kAdThreads)) return fail(QGEMM_EUNSUPPORTED, "too many workgroups");
  (void)hipGetLastError();
  auto launch = [&](auto kernel, long groups) { hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(qg::kAdThreads), 0, stream, g); };
  if (plan.mt_down == 1) {
    if (plan.jt == 1) launch(qg::adapter_down_kernel<1, 1, qg::kAdWaves>, down);
    else if (plan.jt == 2) launch(qg::adapter_down_kernel<1, 2, qg::kAdWaves>, down);
    else launch(qg::adapter_down_kernel<1, 4, qg::kAdWaves>, down);
  } else {
    if (plan.jt == 1) launch(qg::adapter_down_kernel<2, 1, qg::kAdWaves>, down);
    else if (plan.jt == 2) launch(qg::adapter_down_kernel<2, 2, qg::kAdWaves>, down);
    else launch(qg::adapter_down_kernel<2, 4, qg::kAdWaves>, down);
  }
  rc = check_launch("qgemm_adapters");
  if (rc != QGEMM_OK) return rc;
  if (plan.nt == 1) {
    if (plan.s == 1) launch(qg::adapter_up_kernel<1, 1, 1, 8>, up);
    else if (plan.s == 2) launch(qg::adapter_up_kernel<1, 1, 2, 8>, up);
    else launch(qg::adapter_up_kernel<1, 1, 4, 4>, up);
  } else {
    if (plan.mt_up == 1) launch(qg::adapter_up_kernel<1, 2, 1, 1>, up);
    else if (plan.s == 1) launch(qg::adapter_up_kernel<2, 2, 1, 1>, up);
    else if (plan.s == 2) launch(qg::adapter_up_kernel<2, 2, 2, 1>, up);
    else launch(qg::adapter_up_kernel<2, 2, 4, 1>, up);
  }
  rc = check_launch("qgemm_adapters (up)");
  return rc == QGEMM_OK ? ok() : rc;
}

}  // extern "C"
