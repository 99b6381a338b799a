// Attention over the paged 4-bit cache for requests that share their first keys: a group's common keys are read once
// for all of its rows.
//
// The rows of a group, one request after another, are the rows of one unit over the shared keys (a tile of them, a
// key/value head), and every request's rows are those of a unit over the keys behind them. Both leave (output, maximum,
// sum) of their rows, and a second kernel joins the two. The softmax of a row is one over both sets of keys:
//   m = max(m_p, m_t),  l = l_p e^(m_p - m) + l_t e^(m_t - m),  o = (o_p e^(m_p - m) + o_t e^(m_t - m)) / l.
// A shared key is read once instead of once per request, so what bounds the call is no longer the cache's bytes but the steps
// of unpacking and multiplying, of which 16 to 128 rows share one where a few query heads did. Times (us, captured, both
// kernels; in brackets attention_kv4, whose reads of the shared keys for each request come from the L2 caches): 64 requests
// behind 7919 keys, 32/8 heads of 128 34.8 (78.2); 24 x 8 beams over prompts of 200 to 5000 keys, 32/4 of 64 25.2 (27.0); 4
// beams over 1000 keys 12.6 (10.9: there all requests' keys fit into one round of workgroups, and the look-up of groups
// costs more than it saves). Of the first's 34.8, 5 join the parts; in the rest VALU instructions (unpacking and softmax)
// are a third of a SIMD's time, matrix instructions a seventh, with two waves to hide the loads, and 3.5 are the look-up.
//
// Units over shared keys and units behind them are two sequences of granules, each cut evenly over workgroups of its
// own, as the units of the kernel over single requests are; the workgroups are dealt to the two by what their granules
// cost, and alternate over the chip, so that a CU holds some of both: one kind is bound by its arithmetic, the
// other by loads.
//
// Shared are the keys that all of a group's rows see: the prefix as given is cut to the shortest history before the
// new tokens, and to blocks of 64, so that no unit over shared keys needs a mask and no unit behind them begins inside
// a block.
#pragma once

#include "attn_kv4.hpp"

namespace qg {
namespace {

constexpr int kSharedMaxR = 2048;          // requests, and groups
// int32 of LDS in which a workgroup looks them up: 72 KiB at most, beside the tiles' 66
__host__ __device__ constexpr int shared_lds(int R, int Gn) { return 4 * R + 4 * Gn + Gn + 1; }
constexpr int kSharedBlock = 64;           // shared keys come in blocks of so many

struct SharedRow {          // where a request's rows have their results
  int c0, n, first;         // its first row and rows; shared keys
  unsigned base, grans;     // of the keys behind them: first granule of its first unit, granules of each
  int pre_c0;               // first row of its group
  unsigned pre_base, pre_grans;
};

struct SharedCut {          // of the workgroups: `np` over shared keys; each + 1 granules for the first `more` of a kind
  int ok, np;
  unsigned each[2], more[2];
};

struct SharedArgs {
  Kv4Args k;
  const int32_t* groups;    // [Gn + 1]
  const int32_t* prefix;    // [Gn]
  int Gn;
  int cost;                 // of a granule over shared keys, in sixteenths of one behind them
  SharedCut* cut;
  SharedRow* rows;          // [R]
  float* whole;             // [2][T * H][D] rows of units that one workgroup has finished: shared keys, others
  float* whole_ml;          // [2][T * H][2] their maxima and sums
  long part_floats;         // of one slot of k.part
};

// A unit's rows and keys as the tile functions see them.
struct SharedUnit {
  int c0, n, kv, len, tiles, grans;
  int first;                // key of its granule 0
  bool pre;                 // over shared keys, of which every row sees all
  template <int NT>
  __device__ __forceinline__ void size(const Kv4Args& a, int G) {
    tiles = (n * G + 16 * NT - 1) / (16 * NT);
    grans = (len - first + (1 << kKv4GranuleLog2) - 1) >> kKv4GranuleLog2;
    grans = pre ? grans : max(1, grans);
  }
  __device__ __forceinline__ unsigned weight(int Hkv) const {
    return grans == 0 ? 0u : (unsigned)tiles * (unsigned)Hkv * (unsigned)(kKv4Start + grans);
  }
  __device__ __forceinline__ int position(int i) const { return kv - n + i; }
  __device__ __forceinline__ int sees(int i) const { return pre ? len : clamp_i(kv - n + i + 1, 0, len); }
  __device__ __forceinline__ bool past(int i) const { return !pre && kv - n + i >= len; }
};

// Rows that are whole go, unscaled, to the place of their own; the others to the workgroup's slot.
template <int D>
struct SharedFinish {
  bool whole;
  float* slot;
  float* rows;
  float* ml;
  __device__ __forceinline__ float begin_row(const Kv4Args&, size_t row, float m, float sum, int, bool once) const {
    if (once) *reinterpret_cast<float2*>(ml + 2 * row) = make_float2(m, sum);
    return 1.0f;
  }
  __device__ __forceinline__ float* at(const Kv4Args&, size_t i) const { return rows + i; }
  template <int N>
  static __device__ __forceinline__ void store(float* p, const float (&v)[N]) {
#pragma unroll
    for (int e = 0; e < N; e += 4) *reinterpret_cast<f32x4*>(p + e) = f32x4{v[e], v[e + 1], v[e + 2], v[e + 3]};
  }
};

template <int D, int NT>
struct SharedTileLds {
  uint16_t vbuf[kKv4Waves][32 * D];
  float ml[kKv4Waves][16 * NT][2];
};
template <int D>
struct SharedWideLds {
  uint16_t tile[4][64 * D];
  unsigned long long nans[2][kKv4Waves];
};

// A workgroup's granules of a sequence: `more` workgroups of each + 1, then of each.
__device__ __forceinline__ unsigned cut_begin(unsigned w, unsigned each, unsigned more) { return each * w + min(w, more); }
__device__ __forceinline__ unsigned cut_owner(unsigned g, unsigned each, unsigned more) {
  const unsigned wide = more * (each + 1);
  return g < wide ? g / (each + 1) : more + (g - wide) / each;
}

// NP, NT: 16-row tiles of a unit over shared keys, and of one behind them.
template <int D, int NP, int NT>
__global__ __launch_bounds__(kKv4Threads, (kKv4PerCU<D, (NP > NT ? NP : NT)>)) void kv4_shared_kernel(SharedArgs sa) {
  constexpr bool kAnyWide = NP == kKv4Wide || NT == kKv4Wide;
  constexpr int kMostTile = (NP == kKv4Wide ? 1 : NP) > (NT == kKv4Wide ? 1 : NT) ? (NP == kKv4Wide ? 1 : NP) : (NT == kKv4Wide ? 1 : NT);
  using TileLds = SharedTileLds<D, kMostTile>;
  using WideLds = SharedWideLds<D>;
  constexpr size_t kLds = kAnyWide && sizeof(WideLds) > sizeof(TileLds) ? sizeof(WideLds) : sizeof(TileLds);
  __shared__ __attribute__((aligned(16))) char lds[kLds];
  extern __shared__ int4 group_lds[];        // (its type is its alignment: requests and groups are read 16 bytes at once)
  __shared__ unsigned wsum[2][kKv4Waves];
  __shared__ struct {
    int v;
    unsigned off;
  } where;
  const Kv4Args& a = sa.k;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int G = a.H / a.Hkv, R = a.R, Gn = sa.Gn;
  int4* const req = group_lds;                                 // [R] first row, rows, keys, group (-1: none)
  int4* const grp = req + R;                                   // [Gn] first row, rows, shared keys, first granule of its units
  int32_t* const gstart = reinterpret_cast<int32_t*>(grp + Gn);          // [Gn + 1] first requests of the groups

  // ---- requests and groups, in one round of loads
  bool ascends = true;
  const int most_keys = a.W << a.page_log2;
  for (int i = tid; i < max(R, Gn) + 1; i += kKv4Threads) {
    const int r = min(i, R), g = min(i, Gn);
    const int c = a.cu ? a.cu[r] : r, c1 = a.cu ? a.cu[min(i + 1, R)] : min(i + 1, R);
    const int kv = a.kv_len[min(i, R - 1)];
    const int at = sa.groups[g], at1 = sa.groups[min(i + 1, Gn)], keys = Gn > 0 ? sa.prefix[min(i, Gn - 1)] : 0;
    ascends = ascends && c <= c1 && at <= at1;
    const int c0 = clamp_i(c, 0, a.T);
    if (i < R) req[i] = make_int4(c0, max(clamp_i(c1, 0, a.T) - c0, 0), max(kv, 0), -1);
    if (i <= Gn) gstart[i] = clamp_i(at, 0, R);
    if (i < Gn) grp[i].z = clamp_i(keys, 0, most_keys);
  }
  const bool good = !__syncthreads_or(!ascends);
  // ---- the requests' groups, the groups' rows and shared keys
  const int per = (R + kKv4Threads - 1) / kKv4Threads;
  const int r0 = min(R, tid * per), r1 = min(R, r0 + per);
  if (Gn > 0 && r0 < r1) {
    int g = 0;
    for (int hi = Gn - 1; g < hi;) {             // the last group that begins at or before the request
      const int mid = (g + hi + 1) >> 1;
      if (gstart[mid] <= r0) g = mid;
      else hi = mid - 1;
    }
    for (int r = r0; r < r1; ++r) {
      while (g + 1 < Gn && gstart[g + 1] <= r) ++g;
      if (gstart[g] > r || r >= gstart[g + 1]) continue;
      req[r].w = g;
      if (req[r].y > 0) atomicMin(&grp[g].z, max(req[r].z - req[r].y, 0));
    }
  }
  const int gper = (Gn + kKv4Threads - 1) / kKv4Threads;
  const int p0 = min(Gn, tid * gper), p1 = min(Gn, p0 + gper);
  for (int g = p0; g < p1; ++g) {
    const int first = gstart[g], last = gstart[g + 1];
    const int c0 = last > first ? req[first].x : 0;
    grp[g].x = c0;
    grp[g].y = last > first ? req[last - 1].x + req[last - 1].y - c0 : 0;
  }
  __syncthreads();
  auto tail_unit = [&](int r) {
    const int4 q = req[r];
    SharedUnit u;
    u.c0 = q.x;
    u.n = q.y;
    u.kv = q.z;
    u.len = (int)min((long)u.kv, (long)most_keys);
    u.first = min(q.w >= 0 ? grp[max(q.w, 0)].z : 0, u.len) & -kSharedBlock;         // (a request of no rows may have fewer)
    u.pre = false;
    u.size<NT>(a, G);
    return u;
  };
  auto pre_unit = [&](int g) {
    const int4 q = grp[g];
    SharedUnit u;
    u.c0 = q.x;
    u.n = q.y;
    u.len = u.kv = q.z & -kSharedBlock;
    u.first = 0;
    u.pre = true;
    u.size<NP>(a, G);
    return u;
  };
  // ---- where the units are in the two sequences of granules
  unsigned mine[2] = {0, 0};
  for (int g = p0; g < p1; ++g) mine[0] += pre_unit(g).weight(a.Hkv);
  for (int r = r0; r < r1; ++r) mine[1] += tail_unit(r).weight(a.Hkv);
  unsigned base[2], total[2];
#pragma unroll
  for (int kind = 0; kind < 2; ++kind) {
    unsigned inc = mine[kind];
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const unsigned up = __shfl_up(inc, d);
      if (lane >= d) inc += up;
    }
    if (lane == 63) wsum[kind][wave] = inc;
    base[kind] = inc - mine[kind];
  }
  __syncthreads();
#pragma unroll
  for (int kind = 0; kind < 2; ++kind) {
    total[kind] = 0;
#pragma unroll
    for (int i = 0; i < kKv4Waves; ++i) {
      if (i < wave) base[kind] += wsum[kind][i];
      total[kind] += wsum[kind][i];
    }
    total[kind] = __builtin_amdgcn_readfirstlane(good ? total[kind] : 0u);
  }
  // ---- the workgroups: of nwg, np over shared keys
  int np;
  {
    const float cp = (float)total[0] * (float)sa.cost, ct = (float)total[1] * 16.0f;
    np = cp + ct > 0.0f ? (int)((float)a.nwg * cp / (cp + ct) + 0.5f) : 0;
    if (total[0] && np < 1) np = 1;
    if (total[1] && np > a.nwg - 1) np = a.nwg - 1;
    np = min(np, (int)min(total[0], (unsigned)a.nwg));
    np = __builtin_amdgcn_readfirstlane(np);
  }
  const unsigned nwgs[2] = {(unsigned)np, min((unsigned)(a.nwg - np), total[1])};
  unsigned each[2], more[2];
#pragma unroll
  for (int kind = 0; kind < 2; ++kind) {
    each[kind] = nwgs[kind] ? total[kind] / nwgs[kind] : 1u;
    more[kind] = nwgs[kind] ? total[kind] - each[kind] * nwgs[kind] : 0u;
  }
  // the kinds alternate over the launch
  const unsigned bid = blockIdx.x;
  const unsigned pb = bid * (unsigned)np / (unsigned)a.nwg;           // (at most 1024 workgroups)
  const unsigned pe = (bid + 1) * (unsigned)np / (unsigned)a.nwg;
  const int kind = pe > pb ? 0 : 1;
  const unsigned w = kind == 0 ? pb : bid - pb;
  const unsigned ww = kind == 0 ? w : (unsigned)np + w;        // its place among all, and its slots'
  unsigned gs = 0, ge = 0;
  if (w < nwgs[kind]) {
    gs = cut_begin(w, each[kind], more[kind]);
    ge = gs + each[kind] + (w < more[kind] ? 1u : 0u);
  }
  if (bid == 0) {                              // what the second kernel goes by
    if (tid == 0) *sa.cut = {good && total[1] ? 1 : 0, np, {each[0], each[1]}, {more[0], more[1]}};
    unsigned at = base[0];
    for (int g = p0; g < p1; ++g) {
      grp[g].w = (int)at;
      at += pre_unit(g).weight(a.Hkv);
    }
    __syncthreads();
    at = base[1];
    for (int r = r0; r < r1; ++r) {
      const SharedUnit u = tail_unit(r);
      SharedRow row{u.c0, u.n, u.first, at, (unsigned)u.grans, 0, 0, 0};
      if (const int g = req[r].w; g >= 0) {
        const SharedUnit p = pre_unit(g);
        row.pre_c0 = p.c0, row.pre_base = (unsigned)grp[g].w, row.pre_grans = p.weight(a.Hkv) ? (unsigned)p.grans : 0u;
      }
      sa.rows[r] = row;
      at += u.weight(a.Hkv);
    }
  }
  if (gs >= ge) return;
  if (base[kind] <= gs && gs < base[kind] + mine[kind]) {
    unsigned off = gs - base[kind];
    int v = kind == 0 ? p0 : r0;
    if (kind == 0 ? p1 - p0 > 1 : r1 - r0 > 1)        // (one unit to a thread is that one)
      for (unsigned wt; off >= (wt = kind == 0 ? pre_unit(v).weight(a.Hkv) : tail_unit(v).weight(a.Hkv)); ++v) off -= wt;
    where = {v, off};
  }
  __syncthreads();
  // ---- the workgroup's units
  int v = __builtin_amdgcn_readfirstlane(where.v);
  auto uniform = [&](SharedUnit u) {
    u.c0 = __builtin_amdgcn_readfirstlane(u.c0), u.n = __builtin_amdgcn_readfirstlane(u.n);
    u.kv = __builtin_amdgcn_readfirstlane(u.kv), u.len = __builtin_amdgcn_readfirstlane(u.len);
    u.tiles = __builtin_amdgcn_readfirstlane(u.tiles), u.grans = __builtin_amdgcn_readfirstlane(u.grans);
    u.first = __builtin_amdgcn_readfirstlane(u.first);
    u.pre = kind == 0;
    return u;
  };
  auto unit_at = [&]() { return uniform(kind == 0 ? pre_unit(v) : tail_unit(v)); };
  // the request whose table a unit reads: of a group the first that has rows
  auto table_of = [&]() {
    if (kind == 1) return v;
    int r = gstart[v];
    while (r + 1 < gstart[v + 1] && req[r].y == 0) ++r;
    return __builtin_amdgcn_readfirstlane(r);
  };
  SharedUnit u = unit_at();
  int r = table_of();
  int tile, h, gi;
  {
    const unsigned off = (unsigned)__builtin_amdgcn_readfirstlane((int)where.off);
    const unsigned len = (unsigned)(kKv4Start + u.grans), heads = off / len;
    gi = (int)(off - heads * len);
    tile = (int)(heads / (unsigned)a.Hkv);
    h = (int)(heads - (unsigned)tile * (unsigned)a.Hkv);
  }
  const size_t nrows = (size_t)a.T * a.H;
  unsigned at = gs;
  bool first_segment = true;
  while (at < ge) {
    const int v1 = (int)min((unsigned)(kKv4Start + u.grans), (unsigned)gi + (ge - at));
    const int a0 = max(0, gi - kKv4Start), a1 = v1 - kKv4Start;
    if (a1 > a0) {
      const SharedFinish<D> fin{a0 == 0 && a1 == u.grans, a.part + (size_t)(2 * ww + (first_segment ? 0 : 1)) * sa.part_floats,
                                sa.whole + kind * nrows * D, sa.whole_ml + kind * nrows * 2};
      int t = tid;                           // opaque, so that what follows from it is computed for each unit anew and not
      asm volatile("" : "+v"(t));           // held in registers, for both kinds of tiles, from the kernel's start
      auto tiles = [&](auto nt) {
        constexpr int N = decltype(nt)::value;
        if constexpr (N == kKv4Wide) {
          WideLds& wl = *reinterpret_cast<WideLds*>(lds);
          kv4_wide<D>(a, u, r, tile, h, a0, a1, fin, Kv4WideLds{wl.tile[0], wl.tile[1], wl.tile[2], wl.tile[3], {wl.nans[0], wl.nans[1]}}, t);
          __syncthreads();
        } else {
          const Kv4Lane<D> places(a, t);
          SharedTileLds<D, N>& tl = *reinterpret_cast<SharedTileLds<D, N>*>(lds);
          kv4_tile<D, N>(a, u, r, tile, h, a0, a1, fin, places, tl.vbuf, tl.ml);
        }
      };
      if (NP == NT || kind == 0) tiles(std::integral_constant<int, NP>{});
      else tiles(std::integral_constant<int, NT>{});
      first_segment = false;
    }
    at += (unsigned)(v1 - gi);
    gi = 0;
    if (at < ge && ++h == a.Hkv) {
      h = 0;
      if (++tile == u.tiles) {
        tile = 0;
        do {
          ++v;
          u = unit_at();
        } while (u.weight(a.Hkv) == 0);       // (granules are left, so a unit with some is)
        r = table_of();
      }
    }
  }
}

constexpr int kSharedJoinRows = 4;         // rows of a workgroup, one to a wave

// A row's parts: over shared keys, then behind them, each in granule order; 16 lanes across the dimensions, and every
// fourth part to each quarter of the wave.
template <int D, int NP, int NT>
__global__ __launch_bounds__(64 * kSharedJoinRows) void kv4_shared_join_kernel(SharedArgs sa) {
  constexpr int CH = D / 16;
  const Kv4Args& a = sa.k;
  const int lane = threadIdx.x & 63, ch = lane & 15, quarter = lane >> 4;
  const unsigned row = blockIdx.x * kSharedJoinRows + (unsigned)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6);      // (token, head), below 2^31
  if (row >= (unsigned)a.T * (unsigned)a.H) return;
  const SharedCut cut = *sa.cut;
  const int G = a.H / a.Hkv, t = (int)(row / (unsigned)a.H), hq = (int)(row - (unsigned)t * (unsigned)a.H), h = (int)((unsigned)hq / (unsigned)G);
  int r = t;
  if (a.cu) {                  // requests that end at or before the row: two looks of 64 entries each
    const int step = (a.R + 63) / 64;
    const int mark = min((lane + 1) * step, a.R);
    const int blocks = __builtin_popcountll(__ballot(lane * step < a.R && a.cu[mark] <= t));
    r = blocks * step;
    const int i = r + lane + 1;
    r += __builtin_popcountll(__ballot(lane < step && i <= a.R && a.cu[i] <= t));
    if (r >= a.R) return;
  }
  const SharedRow of = sa.rows[r];
  if (!cut.ok) return;
  if (t < of.c0 || t >= of.c0 + of.n) return;
  float top = -__builtin_inff(), sum = 0.0f, out[CH] = {};
  constexpr int DEEP = 4;                 // parts whose loads are on their way at once
  struct Part {
    float m, l;
    f32x4 x[CH / 4];
  };
  auto load = [&](const float* ml, const float* x) {
    Part p;
    const float2 v = *reinterpret_cast<const float2*>(ml);
    p.m = v.x, p.l = v.y;
#pragma unroll
    for (int c = 0; c < CH / 4; ++c) p.x[c] = *reinterpret_cast<const f32x4*>(x + ch * CH + 4 * c);
    return p;
  };
  auto add = [&](const Part& p) {
    const float to = fmaxf(top, p.m);
    const float was = part_weight(top, to, a.sl2), wt = part_weight(p.m, to, a.sl2);
    sum = (top == -__builtin_inff() ? sum : was * sum) + (p.m == -__builtin_inff() ? p.l : wt * p.l);    // (NaN of an empty part stays)
#pragma unroll
    for (int c = 0; c < CH / 4; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e) out[4 * c + e] = out[4 * c + e] * was + wt * p.x[c][e];
    top = to;
  };
  auto parts = [&](int kind, int n16, unsigned base, unsigned grans, int c0) {
    if (grans == 0) return;
    const int rho = (t - c0) * G + (hq - h * G), tile = (int)((unsigned)rho / (unsigned)n16), lr = rho - tile * n16;
    const unsigned unit = base + ((unsigned)tile * (unsigned)a.Hkv + (unsigned)h) * (kKv4Start + grans);
    const unsigned w0 = cut_owner(unit + kKv4Start, cut.each[kind], cut.more[kind]);
    const unsigned w1 = cut_owner(unit + kKv4Start + grans - 1, cut.each[kind], cut.more[kind]);
    if (w0 == w1) {
      const size_t at = (size_t)kind * a.T * a.H + row;
      if (quarter == kind) add(load(sa.whole_ml + 2 * at, sa.whole + at * D));
      return;
    }
    // in its first workgroup the unit is the second segment where one before it has granules there
    const unsigned second = cut_begin(w0, cut.each[kind], cut.more[kind]) < unit ? 1 : 0;
    const unsigned np = kind ? (unsigned)cut.np : 0u;
    for (unsigned i0 = w0 + quarter; i0 <= w1; i0 += 4 * DEEP) {
      Part p[DEEP];
#pragma unroll
      for (int k = 0; k < DEEP; ++k) {
        const unsigned w = min(i0 + 4 * k, w1);
        const float* sl = a.part + (size_t)(2 * (np + w) + (w == w0 ? second : 0u)) * sa.part_floats;
        p[k] = load(sl + 2 * lr, sl + 2 * n16 + lr * D);
      }
#pragma unroll
      for (int k = 0; k < DEEP; ++k)
        if (i0 + 4 * k <= w1) add(p[k]);
    }
  };
  parts(0, 16 * NP, of.pre_base, of.pre_grans, of.pre_c0);
  parts(1, 16 * NT, of.base, of.grans, of.c0);
  const float all = max_over_groups(top);
  const float wt = part_weight(top, all, a.sl2);
  sum = sum_over_groups(top == -__builtin_inff() ? sum : wt * sum);
#pragma unroll
  for (int e = 0; e < CH; ++e) out[e] = sum_over_groups(wt * out[e]);
  if (quarter != 0) return;
  const float inv = row_factor(sum, max(a.kv_len[r], 0) - of.n + (t - of.c0));
#pragma unroll
  for (int e = 0; e < CH; ++e) out[e] *= inv;
  store_row<CH>(a.o + (size_t)row * D + ch * CH, out);
}

}  // namespace
}  // namespace qg
