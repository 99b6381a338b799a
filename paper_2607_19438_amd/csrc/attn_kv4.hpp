// Attention of new tokens over the paged 4-bit cache, for gfx950.
//
// Bound by the cache's bytes for single tokens (0.53 bytes per element, each read once) and by the vector
// ALU that unpacks them where several query rows share a pass. The mathematics is the online softmax of the
// prompt kernel; what differs is the work split and how the 4-bit operands reach the matrix cores.
//
// Work: a unit is (request, tile of 16 NT query rows, key/value head); the rows of a tile are the query heads
// of the group times the request's new tokens. A unit's keys are cut into granules of 128, the granules of all
// units (and a few more for the start of each) are numbered in one sequence, and workgroup w of n takes the w-th
// n-th of them; n is what the CUs hold at once. So requests of any mix of lengths load every workgroup alike, a long
// one is split over many, and the host needs to know no length. (Where the table is short a granule holds all of a
// unit's keys: nothing is split then.)
// A unit that lies in one workgroup is finished there; the others leave (output, maximum, sum) in the caller's
// workspace, at most two per workgroup, and a second kernel joins them in granule order.
//
// A wave takes every fourth run of 32 keys of the workgroup's range:
//   S^T = K Q^T  v_mfma_f32_16x16x32_bf16; lane (key, g) loads its quarter of the key's row (one scale block at
//                D = 128, half of one at D = 64) and unpacks it straight into A operands: the contraction takes
//                the dimensions in the order in which the lanes hold them, and the queries are loaded to match.
//   O^T += V^T P^T  the values need four keys of one dimension in a lane, so the unpacked rows go through
//                a wave's own 32-row LDS tile and come back with the transposing read; no barrier is needed.
// v_cvt_scalef32_pk_bf16_fp4 unpacks two levels and applies the block's scale in one instruction.
//
// Measured: 64 requests of 20 to 16000 keys, 32/8 heads of 128, 176 MB in 43 us (4.1 TB/s) and 4.5 us to join; one
// request of 4097 keys, 32/4 heads, 6.3 us and 4.5 (of the 6.3: workgroups started 0.7, lengths scanned 1.4, page numbers
// and first loads 1.6, its keys 1.2 to 2.2, waves joined 0.9); two chunks of 550 rows over 5000 keys, 32/8 heads, 131 us in all
// (650 TFLOP/s; with pairs of tiles 150).
#pragma once

#include "attn_kernels.hpp"
#include "kv4_levels.hpp"

namespace qg {
namespace {

constexpr int kKv4Threads = 256;
constexpr int kKv4Waves = kKv4Threads / 64;
constexpr int kKv4StepLog2 = 5;
constexpr int kKv4Step = 1 << kKv4StepLog2;           // keys of a wave's step
constexpr int kKv4GranuleLog2 = 7;                    // keys of a granule at least: a step of every wave
static_assert(1 << kKv4GranuleLog2 == kKv4Step * kKv4Waves, "a granule");
constexpr int kKv4Bufs = 2;                           // steps of keys and values that a wave has in registers
// What a unit's start (its queries and page numbers to fetch, its waves to join) counts in the split, in granules.
// With 0 a workgroup of many short units is the last to end. Measured (us; 0, 1, 2, 4): 64 requests of 20 to 16000
// keys 56.7, 48.9, 49.3, 50.5; 9 requests of 3 to 9 tokens 18.8, 18.2, 17.4, 17.4; one of 4097 keys 10.6, 11.0,
// 11.3, 11.2.
constexpr int kKv4Start = 2;

// Value blocks from this scale on count as NaN: 4 and 6 times 2^126 are infinite in bf16, and a weight of 0 would not
// keep an infinity out of the product either. (The store gives at most 252, or 255.)
constexpr uint32_t kKv4NaN = 253;

// The unit that a workgroup's last segment begins and does not end: where its other parts are, and its rows.
struct Kv4Head {
  int r;              // request, -1: there is no such unit
  int last;           // workgroup of its last part
  int slot;           // of the first part, among the workgroup's two; the others are in their workgroup's first
  int c0, nrows;      // the request's first row of q, and its rows of a head
  int row0, h;        // first row of the tile among them; key/value head
  int pad;
};

struct Kv4Args {
  const uint16_t* q;
  const uint8_t* cache;
  const int32_t* table;     // [R][W]
  const int32_t* kv_len;
  const int32_t* cu;        // null: one new token per request
  uint16_t* o;
  Kv4Head* head;            // [nwg]
  float* part;              // [nwg][2] partial results
  int T, R, H, Hkv, W, pages, page_log2, nwg;
  int gran_log2;            // of the keys of a granule
  long qs;
  float sl2;
};

template <int D, int NT>
constexpr int kKv4PartFloats = 16 * NT * (D + 2);

__device__ __forceinline__ int clamp_i(int x, int lo, int hi) { return min(max(x, lo), hi); }

// Tables that the kernels only read, as memory that scalar loads may fetch where the address is uniform.
typedef const __attribute__((address_space(4))) int32_t* const_i32;
__device__ __forceinline__ const_i32 as_const(const int32_t* p) { return (const_i32)p; }

// A request: its first row, its new tokens, its keys as given and those that the table has pages for, and how many
// tiles of rows and granules of keys that is; what its units count in the split.
struct Kv4Request {
  int c0, n, kv, len, tiles, grans;
  template <int NT>
  __device__ __forceinline__ void size(const Kv4Args& a, int G) {
    len = (int)min((long)kv, (long)a.W << a.page_log2);
    tiles = (n * G + 16 * NT - 1) / (16 * NT);
    grans = max(1, (len + (1 << a.gran_log2) - 1) >> a.gran_log2);
  }
  __device__ __forceinline__ unsigned int weight(int Hkv) const {
    return (unsigned)tiles * (unsigned)Hkv * (unsigned)(kKv4Start + grans);
  }
  __device__ __forceinline__ int position(int i) const { return kv - n + i; }                        // of its new token i
  __device__ __forceinline__ int sees(int i) const { return clamp_i(kv - n + i + 1, 0, len); }       // keys
  __device__ __forceinline__ bool past(int i) const { return kv - n + i >= len; }                    // sees keys past the table
  static constexpr int first = 0;                                                                    // key of its granule 0
};

template <int NT>
__device__ __forceinline__ Kv4Request kv4_request(const Kv4Args& a, int r, int G) {
  Kv4Request q;
  if (a.cu) {
    q.c0 = clamp_i(as_const(a.cu)[r], 0, a.T);
    q.n = clamp_i(as_const(a.cu)[r + 1], q.c0, a.T) - q.c0;
  } else {
    q.c0 = r;
    q.n = 1;
  }
  q.kv = max(as_const(a.kv_len)[r], 0);
  q.size<NT>(a, G);
  return q;
}

// The largest of three, NaN if one is (v_maximum3_f32: fmaxf would first quiet each of its arguments).
__device__ __forceinline__ float max3(float x, float y, float z) {
  return __builtin_elementwise_maximum(__builtin_elementwise_maximum(x, y), z);
}

__device__ __forceinline__ float max_over_groups(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float sum_over_groups(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// exp2((m - top) sl2), 0 for an empty part (which has seen no key)
__device__ __forceinline__ float part_weight(float m, float top, float sl2) {
  return m == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f((m - top) * sl2);
}

// What a row's weighted values are multiplied by at the end: one over the weights' sum, and 0 for a row before the
// cache's start. A row that sees keys of score -inf only has the sum 0 too: its 0 times infinity is NaN, as its softmax.
__device__ __forceinline__ float row_factor(float sum, int position) {
  return sum == 0.0f && position < 0 ? 0.0f : 1.0f / sum;
}

template <int N>
__device__ __forceinline__ void store_row(uint16_t* p, const float (&v)[N]) {
  static_assert(N == 4 || N == 8, "8 or 16 bytes");
  if constexpr (N == 8)
    *reinterpret_cast<u32x4*>(p) =
        u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
  else
    *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
}

// Where a unit's result goes: finished rows to the output, a share's (output, maximum, sum) to a slot.
struct Kv4Finish {
  bool whole;
  float* slot;
  // what a row's weighted values are multiplied by before they are stored, and (once a row) the row's other results
  __device__ __forceinline__ float begin_row(const Kv4Args&, size_t, float, float sum, int position, bool) const {
    return row_factor(sum, position);
  }
  __device__ __forceinline__ uint16_t* at(const Kv4Args& a, size_t i) const { return a.o + i; }
  template <int N>
  static __device__ __forceinline__ void store(uint16_t* p, const float (&v)[N]) {
    store_row<N>(p, v);
  }
};

template <int D>
struct Kv4Keys {                  // 32 keys and values as a wave's lanes hold them
  static constexpr int DW = D / 32;
  uint32_t k[2][DW], v[2][DW];
  uint32_t ks[2], vs[2];
  bool ok[2];                     // whether the 16 keys' page is one (uniform)
};

constexpr int kKv4Wide = 8;          // NT of the wide form: 128 query rows

// A unit's share of a wide tile, 128 query rows: the four waves take 32 rows each and walk the same keys, 64 to a
// block. The block is unpacked once for all of them, a quarter of a row to a thread, into LDS; the products are the
// prompt kernel's (v_mfma_f32_32x32x16_bf16). The next block's levels are in registers while a block is computed.
// Bound by the matrix cores and the softmax as that kernel is, and by the parts: 64 KiB each, written and read again, for
// two chunks of 550 rows over 5000 keys 27 of 131 us. (The value fragments a whole step ahead, as there, take 12
// registers too many at D = 128: 134 us.)
struct Kv4WideLds {
  uint16_t *ks0, *ks1, *vt0, *vt1;                // [64 * D] each
  unsigned long long* nans[2];                    // value blocks of NaN: bit 4 key + quarter of each wave's 16 keys
};

template <int D, typename Rq, typename Finish>
__device__ __forceinline__ void kv4_wide(const Kv4Args& a, const Rq& rq, int r, int tile, int h, int a0, int a1, const Finish& fin,
                                         const Kv4WideLds& lds, int tid) {
  constexpr int BK = 64, DW = D / 32, KSTEPS = D / 16, DT = D / 32;
  uint16_t *const ks0 = lds.ks0, *const ks1 = lds.ks1, *const vt0 = lds.vt0, *const vt1 = lds.vt1;
  unsigned long long* const nans[2] = {lds.nans[0], lds.nans[1]};
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, hh = lane >> 5;
  const int G = a.H / a.Hkv;
  const int row0 = tile * 16 * kKv4Wide, nrows = rq.n * G;
  const int rho = row0 + 32 * wave + col;
  const bool live = rho < nrows;
  auto seen_by = [&](int row) { return rq.sees(row / G); };                       // keys that a row sees
  const int lim = live ? seen_by(rho) : 0;
  const int kmax = seen_by(min(row0 + 16 * kKv4Wide, nrows) - 1);                 // keys that any row sees,
  const int wrow = row0 + 32 * wave;
  const int wmax = wrow < nrows ? seen_by(min(wrow + 32, nrows) - 1) : 0;         // any of the wave's,
  const int wall = wrow < nrows ? seen_by(wrow) : 0;                              // every one of the wave's
  bf16x8 qf[KSTEPS];
  {
    const int token = rho / G;
    const uint16_t* qp = a.q + (size_t)(rq.c0 + token) * a.qs + (size_t)(h * G + (rho - token * G)) * D + 8 * hh;
#pragma unroll
    for (int t = 0; t < KSTEPS; ++t)
      qf[t] = live ? __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(qp + 16 * t)) : bf16x8{};
  }
  f32x16 acc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) acc[dt] = f32x16{};
  float m_run = -__builtin_inff();
  float l_run = live && rq.past(rho / G) ? __builtin_nanf("") : 0.0f;

  const const_i32 trow = as_const(a.table) + (size_t)r * a.W;     // (indexed only if there is a key, so W >= 1)
  const int page_mask = (1 << a.page_log2) - 1;
  const uint32_t record = (uint32_t)(D + D / 16) << a.page_log2;
  const uint32_t page_bytes = (uint32_t)a.Hkv * record;
  const uint8_t* cache_h = a.cache + (size_t)h * record;
  const int kq = lane >> 2, quarter = lane & 3;                   // this thread's key of the wave's 16, quarter of its row
  const uint32_t k_off = (uint32_t)(kq * (D / 2) + quarter * (D / 8));
  const uint32_t v_off = k_off + ((uint32_t)(D / 2) << a.page_log2);
  const uint32_t ks_off = ((uint32_t)D << a.page_log2) + (uint32_t)(kq * (D / 32) + (D == 128 ? quarter : quarter >> 1));
  const uint32_t vs_off = ks_off + ((uint32_t)(D / 32) << a.page_log2);
  auto kswz = [](int key) { return D == 128 ? (key & 15) : row_swizzle(key); };
  // (as the prompt kernel's, and the four keys of 16 writing threads on different 16-byte groups too)
  auto vswz = [](int key) { return D == 128 ? 5 * (key & 3) : 5 * ((key >> 1) & 1); };

  const int base = rq.first / BK;
  const int jb0 = base + (a0 << (a.gran_log2 - 6)), jb1 = min(base + (a1 << (a.gran_log2 - 6)), (kmax + BK - 1) / BK);
  struct Levels {
    uint32_t k[DW], v[DW], ks, vs;
    bool ok;
  };
  auto page_of = [&](int jb) { return trow[min((BK * jb + 16 * wave) >> a.page_log2, a.W - 1)]; };
  auto load = [&](int jb, int id) {
    Levels b;
    b.ok = (unsigned)id < (unsigned)a.pages;
    const uint8_t* rec = cache_h + (uint64_t)(b.ok ? (uint32_t)id : 0u) * page_bytes;
    const uint32_t in_page = (uint32_t)((BK * jb + 16 * wave) & page_mask);
    const uint8_t* codes = rec + in_page * (D / 2);
    const uint8_t* scales = rec + in_page * (D / 32);
    if constexpr (DW == 4) {
      const u32x4 k4 = *reinterpret_cast<const u32x4*>(codes + k_off), v4 = *reinterpret_cast<const u32x4*>(codes + v_off);
#pragma unroll
      for (int t = 0; t < DW; ++t) b.k[t] = k4[t], b.v[t] = v4[t];
    } else {
      const uint2 k2 = *reinterpret_cast<const uint2*>(codes + k_off), v2 = *reinterpret_cast<const uint2*>(codes + v_off);
      b.k[0] = k2.x, b.k[1] = k2.y, b.v[0] = v2.x, b.v[1] = v2.y;
    }
    b.ks = scales[ks_off];
    b.vs = scales[vs_off];
    return b;
  };
  // The levels of a block into LDS. Values that no row may see are taken as zero, and NaN blocks too (a weight of 0
  // would not keep a NaN out of the product); rows that do see a NaN block get it after the product.
  auto unpack = [&](Levels& b, int jb, uint16_t* ksn, uint16_t* vtn, unsigned long long* nan) {
    const int key = 16 * wave + kq;
    const uint32_t ks = b.ok ? b.ks : 255u, vs = b.ok ? b.vs : 255u;
    const float ku = __builtin_bit_cast(float, ks << 23);
#pragma unroll
    for (int t = 0; t < DW; ++t)
      *reinterpret_cast<u32x4*>(&ksn[key * D + (((quarter * DW + t) ^ kswz(key)) << 3)]) = fp4_unit(b.k[t], ku);
    const bool hidden = BK * jb + key >= kmax;
    const unsigned long long bad = __ballot(!hidden && vs >= kKv4NaN);
    const bool zero = hidden || vs >= kKv4NaN;
    const float vu = __builtin_bit_cast(float, zero ? 0u : vs << 23);
#pragma unroll
    for (int t = 0; t < DW; ++t)
      *reinterpret_cast<u32x4*>(&vtn[key * D + (((quarter * DW + t) ^ vswz(key)) << 3)]) = fp4_unit(zero ? 0u : b.v[t], vu);
    if (lane == 0) nan[wave] = bad;
  };
  auto rd_k = [&](const uint16_t* ksc, int t, int kt) {
    const int key = kt * 32 + col;
    return *reinterpret_cast<const bf16x8*>(&ksc[key * D + (((2 * t + hh) ^ kswz(key)) << 3)]);
  };
  const int trk = (lane & 15) >> 2, trd = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
  auto rd_v = [&](const uint16_t* vtc, int u, int dt) {
    uint32_t f[4];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int key = 16 * u + 8 * half + 4 * hh + trk;
      const int dim = 32 * dt + trd;
      typedef short v4i16 __attribute__((ext_vector_type(4)));
      const v4i16 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4i16*)(
          const_cast<uint16_t*>(vtc) + key * D + (((dim >> 3) ^ vswz(key)) << 3) + (dim & 7)));
      const uint2 xx = __builtin_bit_cast(uint2, x);
      f[2 * half] = xx.x;
      f[2 * half + 1] = xx.y;
    }
    return __builtin_bit_cast(bf16x8, u32x4{f[0], f[1], f[2], f[3]});
  };
  auto product = [&](int jb, const uint16_t* ksc, const uint16_t* vtc, const unsigned long long* nan) {
    const int j0 = BK * jb;
    f32x16 sc[2] = {f32x16{}, f32x16{}};
    bf16x8 kf[2][2];
#pragma unroll
    for (int c = 0; c < 2; ++c) kf[0][c] = rd_k(ksc, 0, c);
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int t = 0; t < KSTEPS; ++t) {
#pragma unroll
      for (int c = 0; c < 2; ++c)
        if (t + 1 < KSTEPS) kf[(t + 1) & 1][c] = rd_k(ksc, t + 1, c);
#pragma unroll
      for (int c = 0; c < 2; ++c) sc[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[t & 1][c], qf[t], sc[c], 0, 0, 0);
      if (t + 1 < KSTEPS) QG_SG(kSchedDSRead, 2);
      QG_SG(kSchedMFMA, 2);
    }
    __builtin_amdgcn_s_setprio(0);
    if (j0 + BK > wall) {
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (j0 + kt * 32 + (e >> 2) * 8 + 4 * hh + (e & 3) >= lim) sc[kt][e] = -__builtin_inff();
    }
    float mloc = -__builtin_inff();
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int e = 0; e < 16; ++e) mloc = fmaxf(mloc, sc[kt][e]);
    mloc = fmaxf(mloc, other_half(mloc));
    const float m_new = fmaxf(m_run, mloc);
    if ((m_new - m_run) * a.sl2 > 8.0f) {            // as everywhere: the reference maximum moves seldom
      const float alpha = __builtin_amdgcn_exp2f((m_run - m_new) * a.sl2);
      l_run *= alpha;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) acc[dt] *= alpha;
      m_run = m_new;
    }
    const float ms = m_run == -__builtin_inff() ? 0.0f : m_run * a.sl2;
    float lsum = 0.0f;
    uint32_t pf[2][8];
    auto exps = [&](int kt) {
#pragma unroll
      for (int e = 0; e < 16; e += 2) {
        const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[kt][e], a.sl2, -ms));
        const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[kt][e + 1], a.sl2, -ms));
        lsum += p0 + p1;
        pf[kt][e >> 1] = pack_bf16x2(p0, p1);
      }
    };
    exps(0);
    // (the fragments one product ahead; a step ahead they would not fit in the registers)
    bf16x8 vf[2];
    vf[0] = rd_v(vtc, 0, 0);
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int e0 = (u & 1) * 4;
      const bf16x8 pb = __builtin_bit_cast(bf16x8, u32x4{pf[u >> 1][e0], pf[u >> 1][e0 + 1], pf[u >> 1][e0 + 2], pf[u >> 1][e0 + 3]});
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const int n = u * DT + dt + 1;
        if (n < 4 * DT) vf[n & 1] = rd_v(vtc, n / DT, n % DT);
        acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[(n - 1) & 1], pb, acc[dt], 0, 0, 0);
      }
      if (u == 0) exps(1);
    }
    __builtin_amdgcn_s_setprio(0);
    l_run += lsum;
    for (int i = 0; i < kKv4Waves; ++i) {
      const unsigned long long bad = nan[i];
      if (__builtin_expect(bad != 0, 0)) {
        const int n = clamp_i(lim - j0 - 16 * i, 0, 16);
        const unsigned long long seen = bad & (n == 16 ? ~0ull : (1ull << (4 * n)) - 1ull);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
          if ((seen >> (D == 128 ? dt : 2 * dt)) & 0x1111111111111111ull) acc[dt] = f32x16{} + __builtin_nanf("");
      }
    }
  };

  if (jb0 < jb1) {
    // past the last block loads go on with that one, so that each step's are issued
    auto at = [&](int jb) { return min(jb, jb1 - 1); };
    Levels cur = load(jb0, page_of(jb0));
    Levels next = load(at(jb0 + 1), page_of(at(jb0 + 1)));
    int id = page_of(at(jb0 + 2));
    unpack(cur, jb0, ks0, vt0, nans[0]);
    __syncthreads();
    auto step = [&](int jb, const uint16_t* ksc, const uint16_t* vtc, const unsigned long long* nanc, uint16_t* ksn, uint16_t* vtn,
                    unsigned long long* nann) {
      if (jb + 1 < jb1) unpack(next, jb + 1, ksn, vtn, nann);
      next = load(at(jb + 2), id);
      id = page_of(at(jb + 3));
      if (BK * jb < wmax) product(jb, ksc, vtc, nanc);
      __syncthreads();
    };
    for (int jb = jb0; jb < jb1; jb += 2) {
      step(jb, ks0, vt0, nans[0], ks1, vt1, nans[1]);
      if (jb + 1 < jb1) step(jb + 1, ks1, vt1, nans[1], ks0, vt0, nans[0]);
    }
  }

  // lane (col, hh) holds o[row][32 dt + 8 e + 4 hh + {0..3}] in acc[dt][4 e ..]
  const float sum = l_run + other_half(l_run);
  if (fin.whole) {
    if (live) {
      const int token = rho / G;
      const size_t row = (size_t)(rq.c0 + token) * a.H + (size_t)(h * G + (rho - token * G));
      const float by = fin.begin_row(a, row, m_run, sum, rq.position(token), hh == 0);
      auto* out = fin.at(a, row * D);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float v[4] = {acc[dt][4 * e] * by, acc[dt][4 * e + 1] * by, acc[dt][4 * e + 2] * by, acc[dt][4 * e + 3] * by};
          fin.store(out + dt * 32 + 8 * e + 4 * hh, v);
        }
    }
  } else {
    const int row = 32 * wave + col;
    float* po = fin.slot + 2 * 16 * kKv4Wide + row * D;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        *reinterpret_cast<f32x4*>(po + dt * 32 + 8 * e + 4 * hh) =
            f32x4{acc[dt][4 * e], acc[dt][4 * e + 1], acc[dt][4 * e + 2], acc[dt][4 * e + 3]};
    if (hh == 0) {
      fin.slot[2 * row] = m_run;
      fin.slot[2 * row + 1] = sum;
    }
  }
}

// A thread's places: in the workgroup, and within a record (key or value col of 16, its quarter of the row, that quarter's scale).
template <int D>
struct Kv4Lane {
  int tid, lane, wave, col, grp, G, page_mask;
  uint32_t page_bytes, k_off, v_off, ks_off, vs_off;
  __device__ __forceinline__ Kv4Lane(const Kv4Args& a, int t) {
    tid = t, lane = tid & 63;
    wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    col = lane & 15, grp = lane >> 4;
    G = a.H / a.Hkv;
    page_mask = (1 << a.page_log2) - 1;
    page_bytes = (uint32_t)a.Hkv * ((uint32_t)(D + D / 16) << a.page_log2);     // (the host keeps it below 2^31)
    k_off = (uint32_t)(col * (D / 2) + grp * (D / 8));
    v_off = k_off + ((uint32_t)(D / 2) << a.page_log2);
    ks_off = ((uint32_t)D << a.page_log2) + (uint32_t)(col * (D / 32) + (D == 128 ? grp : grp >> 1));
    vs_off = ks_off + ((uint32_t)(D / 32) << a.page_log2);
  }
};

// A unit's share of 16 NT query rows: the four waves take every fourth run of 32 keys and are joined at the end.
template <int D, int NT, typename Rq, typename Finish>
__device__ __forceinline__ void kv4_tile(const Kv4Args& a, const Rq& rq, int r, int tile, int h, int a0, int a1, const Finish& fin,
                                         const Kv4Lane<D>& L, uint16_t (&vbuf)[kKv4Waves][32 * D], float (&ml)[kKv4Waves][16 * NT][2]) {
  constexpr int DW = D / 32;            // dwords of packed levels in a lane: a quarter of a key's row
  constexpr int DT = D / 16;            // 16-row tiles of O^T
  constexpr int CH = D / 16;            // dimensions of a thread where parts are joined
  const int row0 = tile * 16 * NT;
  const int lane = L.lane, wave = L.wave, col = L.col, grp = L.grp, G = L.G, tid = L.tid;
  const int page_mask = L.page_mask;
  const uint32_t page_bytes = L.page_bytes, k_off = L.k_off, v_off = L.v_off, ks_off = L.ks_off, vs_off = L.vs_off;
  uint16_t* vw = vbuf[wave];
  auto vswz = [](int key) {
    const int low = 2 * (key & 3) | ((key >> 2) & 1);
    return D == 128 ? low | (key & 8) : low;
  };

  // this lane's query rows
  const int nrows = rq.n * G;
  int lim[NT];                                    // keys that the row sees
  bf16x8 qf[NT][DW];
  f32x4 l_run[NT];                              // sum of the weights as they enter the product, four times
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int rho = row0 + 16 * nt + col;
    const int i = rho / G;
    const bool live = rho < nrows;
    lim[nt] = live ? rq.sees(i) : 0;
    l_run[nt] = f32x4{} + (live && rq.past(i) ? __builtin_nanf("") : 0.0f);
    const uint16_t* qp = a.q + (size_t)(rq.c0 + i) * a.qs + (size_t)(h * G + (rho - i * G)) * D + grp * (D / 4);
#pragma unroll
    for (int t = 0; t < DW; ++t)
      qf[nt][t] = live ? __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(qp + 8 * t)) : bf16x8{};
  }
  const int last = (min(row0 + 16 * NT, nrows) - 1) / G;
  const int kmax = rq.sees(last);                             // keys that any row sees
  const int kall = rq.sees(row0 / G);                         // keys that every row sees

  f32x4 acc[NT][DT];
  float m_run[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    m_run[nt] = -__builtin_inff();
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) acc[nt][dt] = f32x4{};
  }

  const const_i32 trow = as_const(a.table) + (size_t)r * a.W;      // (indexed only if there is a key, so W >= 1)
  const int base = rq.first / kKv4Step;
  const int s_end = min(base + (a1 << (a.gran_log2 - kKv4StepLog2)), (kmax + kKv4Step - 1) / kKv4Step);
  const uint8_t* cache_h = a.cache + (size_t)h * ((uint32_t)(D + D / 16) << a.page_log2);
  // pages of the two halves of a step (the last step's second half, or the step after it, may be past the table)
  auto pages_of = [&](int s) {
    const int key = kKv4Step * s;
    return make_int2(trow[min(key >> a.page_log2, a.W - 1)], trow[min((key + 16) >> a.page_log2, a.W - 1)]);
  };
  auto load = [&](int s, int2 ids) {
    Kv4Keys<D> b;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int key = kKv4Step * s + 16 * i;
      const int id = i ? ids.y : ids.x;
      b.ok[i] = (unsigned)id < (unsigned)a.pages;
      // the addresses' parts that all lanes share are scalar, the lanes' own do not change
      const uint8_t* rec = cache_h + (uint64_t)(b.ok[i] ? (uint32_t)id : 0u) * page_bytes;
      const uint32_t in_page = (uint32_t)(key & page_mask);
      const uint8_t* codes = rec + in_page * (D / 2);
      const uint8_t* scales = rec + in_page * (D / 32);
      if constexpr (DW == 4) {
        const u32x4 k4 = *reinterpret_cast<const u32x4*>(codes + k_off);
        const u32x4 v4 = *reinterpret_cast<const u32x4*>(codes + v_off);
#pragma unroll
        for (int t = 0; t < DW; ++t) b.k[i][t] = k4[t], b.v[i][t] = v4[t];
      } else {
        const uint2 k2 = *reinterpret_cast<const uint2*>(codes + k_off);
        const uint2 v2 = *reinterpret_cast<const uint2*>(codes + v_off);
        b.k[i][0] = k2.x, b.k[i][1] = k2.y, b.v[i][0] = v2.x, b.v[i][1] = v2.y;
      }
      b.ks[i] = scales[ks_off];
      b.vs[i] = scales[vs_off];
    }
    return b;
  };

  auto step = [&](Kv4Keys<D>& b, int s) {
    const int key0 = kKv4Step * s;
    const bool need_mask = key0 + kKv4Step > kall;
    if (!(b.ok[0] && b.ok[1])) {          // a page that is none reads as NaN
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (!b.ok[i]) b.ks[i] = b.vs[i] = 255u;
    }
    f32x4 sc[NT][2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float unit = __builtin_bit_cast(float, b.ks[i] << 23);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) sc[nt][i] = f32x4{};
#pragma unroll
      for (int t = 0; t < DW; ++t) {
        const bf16x8 kf = __builtin_bit_cast(bf16x8, fp4_unit(b.k[i][t], unit));
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
          sc[nt][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[nt][t], sc[nt][i], 0, 0, 0);
      }
    }
    // Values that no row may see are taken as zero, and NaN blocks too (a weight of 0 would not keep a NaN
    // out of the product); rows that do see a NaN block get it below.
    if (need_mask) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const bool hidden = key0 + 16 * i + col >= kmax;
        b.vs[i] = hidden ? 0u : b.vs[i];
#pragma unroll
        for (int t = 0; t < DW; ++t) b.v[i][t] = hidden ? 0u : b.v[i][t];
      }
    }
    const unsigned long long nan_at[2] = {__ballot(b.vs[0] >= kKv4NaN), __ballot(b.vs[1] >= kKv4NaN)};
    if (nan_at[0] | nan_at[1]) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const bool nan = b.vs[i] >= kKv4NaN;
        b.vs[i] = nan ? 0u : b.vs[i];
#pragma unroll
        for (int t = 0; t < DW; ++t) b.v[i][t] = nan ? 0u : b.v[i][t];
      }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float unit = __builtin_bit_cast(float, b.vs[i] << 23);
      const int key = 16 * i + col;
#pragma unroll
      for (int t = 0; t < DW; ++t)
        *reinterpret_cast<u32x4*>(&vw[key * D + (((grp * DW + t) ^ vswz(key)) << 3)]) = fp4_unit(b.v[i][t], unit);
    }
    bf16x8 pb[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      if (need_mask) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (key0 + 16 * i + 4 * grp + e >= lim[nt]) sc[nt][i][e] = -__builtin_inff();
      }
      float mloc = max3(max3(sc[nt][0][0], sc[nt][0][1], sc[nt][0][2]), max3(sc[nt][0][3], sc[nt][1][0], sc[nt][1][1]),
                        max3(sc[nt][1][2], sc[nt][1][3], sc[nt][1][3]));
      // The reference maximum moves, for all rows of the wave, only when some score passes its row's by more
      // than 8 in exp2 units: weights stay <= 2^8, and most steps exchange nothing between lanes.
      if (__any((mloc - m_run[nt]) * a.sl2 > 8.0f)) {
        const float m_new = fmaxf(m_run[nt], max_over_groups(mloc));
        const float alpha = m_new == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f((m_run[nt] - m_new) * a.sl2);
        l_run[nt] *= alpha;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) acc[nt][dt] *= alpha;
        m_run[nt] = m_new;
      }
      const float ms = m_run[nt] == -__builtin_inff() ? 0.0f : m_run[nt] * a.sl2;
      float p[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[nt][e >> 2][e & 3], a.sl2, -ms));
      pb[nt] = __builtin_bit_cast(bf16x8, u32x4{pack_bf16x2(p[0], p[1]), pack_bf16x2(p[2], p[3]),
                                                pack_bf16x2(p[4], p[5]), pack_bf16x2(p[6], p[7])});
    }
    // the weights' sum as a product with ones: rounded as they are, so that their rounding cancels where few weigh
    const bf16x8 ones = __builtin_bit_cast(bf16x8, u32x4{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u});
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) l_run[nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pb[nt], l_run[nt], 0, 0, 0);
    asm volatile("" ::: "memory");       // the tile's writes stay before its reads; a wave's LDS accesses run in order
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      uint32_t f[4];
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int key = 16 * half + 4 * grp + (col >> 2);
        const int dim = 16 * dt + 4 * (lane & 3);
        typedef short v4i16 __attribute__((ext_vector_type(4)));
        const v4i16 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) v4i16*)(vw + key * D + (((dim >> 3) ^ vswz(key)) << 3) + (dim & 7)));
        const uint2 xx = __builtin_bit_cast(uint2, x);
        f[2 * half] = xx.x;
        f[2 * half + 1] = xx.y;
      }
      const bf16x8 vf = __builtin_bit_cast(bf16x8, u32x4{f[0], f[1], f[2], f[3]});
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
        acc[nt][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pb[nt], acc[nt][dt], 0, 0, 0);
    }
    asm volatile("" ::: "memory");       // and the next tile's writes after them
    if (nan_at[0] | nan_at[1]) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint32_t seen = (1u << clamp_i(lim[nt] - key0 - 16 * i, 0, 16)) - 1u;
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) {
            const uint32_t keys = (uint32_t)(nan_at[i] >> (D == 128 ? 16 * (dt >> 1) : 32 * (dt >> 1))) & 0xffffu;
            if (keys & seen) acc[nt][dt] = f32x4{} + __builtin_nanf("");
          }
        }
    }
  };

  // kKv4Bufs steps of keys and values in registers: while one is computed the others are in flight, and the page
  // numbers of the next to be loaded. Every refill is issued, past the last step once more for that step: were
  // it skipped, the compiler could not tell how many loads are behind the one a step waits for, and would wait
  // for all of them.
  if (base + (a0 << (a.gran_log2 - kKv4StepLog2)) + wave < s_end) {
    int s = base + (a0 << (a.gran_log2 - kKv4StepLog2)) + wave, sl = s;
    const int s_last = s + ((s_end - 1 - s) & ~(kKv4Waves - 1));
    int2 ids = pages_of(s);
    Kv4Keys<D> buf[kKv4Bufs];
    auto refill = [&](Kv4Keys<D>& b) {
      b = load(sl, ids);
      sl = min(sl + kKv4Waves, s_last);
      ids = pages_of(sl);
    };
#pragma unroll
    for (int j = 0; j < kKv4Bufs; ++j) refill(buf[j]);
    for (bool more = true; more;) {
#pragma unroll
      for (int j = 0; j < kKv4Bufs; ++j) {
        step(buf[j], s);
        s += kKv4Waves;
        if (s >= s_end) {
          more = false;
          break;
        }
        refill(buf[j]);
      }
    }
  }

  // join the four waves, 16 rows at a time
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    float* ow = reinterpret_cast<float*>(vw);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
      *reinterpret_cast<f32x4*>(&ow[col * D + (((4 * dt + grp) ^ (col & 7)) << 2)]) = acc[nt][dt];
    if (grp == 0) {
      ml[wave][16 * nt + col][0] = m_run[nt];
      ml[wave][16 * nt + col][1] = l_run[nt][0];
    }
    __syncthreads();
    const int row = tid >> 4, ch = tid & 15;
    float mw[kKv4Waves], top = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < kKv4Waves; ++i) {
      mw[i] = ml[i][16 * nt + row][0];
      top = fmaxf(top, mw[i]);
    }
    float sum = 0.0f, out[CH] = {};
#pragma unroll
    for (int i = 0; i < kKv4Waves; ++i) {
      const float wt = part_weight(mw[i], top, a.sl2);
      const float li = ml[i][16 * nt + row][1];
      sum += mw[i] == -__builtin_inff() ? li : wt * li;     // an empty part's 0, or NaN
      const float* oi = reinterpret_cast<const float*>(vbuf[i]);
#pragma unroll
      for (int c = 0; c < CH / 4; ++c) {
        const f32x4 x = *reinterpret_cast<const f32x4*>(&oi[row * D + (((ch * (CH / 4) + c) ^ (row & 7)) << 2)]);
#pragma unroll
        for (int e = 0; e < 4; ++e) out[4 * c + e] += wt * x[e];
      }
    }
    const int rho = row0 + 16 * nt + row;
    if (fin.whole) {
      if (rho < nrows) {
        const int i = rho / G;
        const size_t at = (size_t)(rq.c0 + i) * a.H + (size_t)(h * G + (rho - i * G));
        const float by = fin.begin_row(a, at, top, sum, rq.position(i), ch == 0);
#pragma unroll
        for (int e = 0; e < CH; ++e) out[e] *= by;
        fin.store(fin.at(a, at * D + ch * CH), out);
      }
    } else {
      float* po = fin.slot + 2 * 16 * NT + (16 * nt + row) * D + ch * CH;
#pragma unroll
      for (int c = 0; c < CH / 4; ++c)
        *reinterpret_cast<f32x4*>(po + 4 * c) = f32x4{out[4 * c], out[4 * c + 1], out[4 * c + 2], out[4 * c + 3]};
      if (ch == 0) {
        fin.slot[2 * (16 * nt + row)] = top;
        fin.slot[2 * (16 * nt + row) + 1] = sum;
      }
    }
    __syncthreads();
  }
}

template <int D, int NT>
__device__ __forceinline__ void kv4_body(const Kv4Args& a) {
  constexpr bool kWide = NT == kKv4Wide;
  __shared__ __attribute__((aligned(16))) uint16_t vbuf[kKv4Waves][kWide ? 8 : 32 * D];     // also 16 rows of O in fp32
  __shared__ float ml[kKv4Waves][kWide ? 1 : 16 * NT][2];
  __shared__ __attribute__((aligned(16))) uint16_t ks0[kWide ? 64 * D : 8], ks1[kWide ? 64 * D : 8], vt0[kWide ? 64 * D : 8],
      vt1[kWide ? 64 * D : 8];
  __shared__ unsigned long long nans[2][kKv4Waves];
  __shared__ unsigned int wsum[kKv4Waves];
  __shared__ struct {
    int r, off, c0, n, kv;
  } where;

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int G = a.H / a.Hkv;
  const int w = xcd_tile((int)blockIdx.x, a.nwg);

  // the workgroup's range of granules (a unit's start counted in), and the request that it begins in
  unsigned int total = 0, gs = 0, ge = 0;         // (the host keeps the largest possible total below 2^31)
  constexpr unsigned int kNoSum = 0xffffffffu;
  unsigned int parts, each, more;                 // workgroups with work: `more` of each + 1 granules, then of each
  {
    const int per = (a.R + kKv4Threads - 1) / kKv4Threads;
    const int r0 = min(a.R, tid * per), r1 = min(a.R, r0 + per);
    unsigned int mine = 0;
    bool ascends = true;          // else requests share rows, and their work could pass what the host has bounded
    for (int r = r0; r < r1; ++r) {
      mine += kv4_request<NT>(a, r, G).weight(a.Hkv);
      if (a.cu) ascends = ascends && as_const(a.cu)[r] <= as_const(a.cu)[r + 1];
    }
    const bool descent = __any(!ascends);
    unsigned int inc = mine;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const unsigned int up = __shfl_up(inc, d);
      if (lane >= d) inc += up;
    }
    if (lane == 63) wsum[wave] = descent ? kNoSum : inc;
    __syncthreads();
    unsigned int base = inc - mine, most = 0;
#pragma unroll
    for (int i = 0; i < kKv4Waves; ++i) {
      if (i < wave) base += wsum[i];
      total += wsum[i];
      most = max(most, wsum[i]);
    }
    total = __builtin_amdgcn_readfirstlane(most == kNoSum ? 0u : total);      // then nothing is done
    parts = min((unsigned)a.nwg, total);
    each = parts ? total / parts : 0u;
    more = total - each * parts;
    if ((unsigned)w < parts) {
      gs = each * (unsigned)w + min((unsigned)w, more);
      ge = gs + each + ((unsigned)w < more ? 1u : 0u);
    }
    if (gs < ge && base <= gs && gs < base + mine) {
      unsigned int off = gs - base;
      int r = r0;
      Kv4Request q = kv4_request<NT>(a, r, G);
      while (off >= q.weight(a.Hkv)) {
        off -= q.weight(a.Hkv);
        q = kv4_request<NT>(a, ++r, G);
      }
      where = {r, (int)off, q.c0, q.n, q.kv};
    }
    __syncthreads();
  }
  if (gs >= ge) {
    if (tid == 0) a.head[w].r = -1;
    return;
  }
  int r = __builtin_amdgcn_readfirstlane(where.r);
  Kv4Request rq;
  rq.c0 = __builtin_amdgcn_readfirstlane(where.c0);
  rq.n = __builtin_amdgcn_readfirstlane(where.n);
  rq.kv = __builtin_amdgcn_readfirstlane(where.kv);
  rq.size<NT>(a, G);
  int tile, h, gi;
  {
    const unsigned int off = (unsigned)__builtin_amdgcn_readfirstlane(where.off);
    const unsigned int heads = off / (unsigned)(kKv4Start + rq.grans);      // (tile, head) in one number
    gi = (int)(off - heads * (unsigned)(kKv4Start + rq.grans));
    tile = (int)(heads / (unsigned)a.Hkv);
    h = (int)(heads - (unsigned)tile * (unsigned)a.Hkv);
  }
  unsigned int g = gs;
  bool first_segment = true;
  Kv4Head header{-1};

  const Kv4Lane<D> places(a, tid);
  while (g < ge) {
    // the unit's share, its start's granules left out: with nothing but those it is left to the next workgroup
    const int v1 = (int)min((unsigned)(kKv4Start + rq.grans), (unsigned)gi + (ge - g));
    const int a0 = max(0, gi - kKv4Start), a1 = v1 - kKv4Start;
    if (a1 > a0) {
      const bool whole = a0 == 0 && a1 == rq.grans;
      const Kv4Finish fin{whole, a.part + (size_t)(2 * w + (first_segment ? 0 : 1)) * kKv4PartFloats<D, NT>};
      if constexpr (NT == kKv4Wide) {
        kv4_wide<D>(a, rq, r, tile, h, a0, a1, fin, Kv4WideLds{ks0, ks1, vt0, vt1, {nans[0], nans[1]}}, tid);
      } else {
        kv4_tile<D, NT>(a, rq, r, tile, h, a0, a1, fin, places, vbuf, ml);
      }
      if (a0 == 0 && a1 < rq.grans) {          // the unit goes on: this workgroup's block of the second kernel joins it
        const unsigned int end = g + (unsigned)(kKv4Start + rq.grans - gi) - 1, wide = more * (each + 1);   // its last granule,
        const unsigned int last_w = end < wide ? end / (each + 1) : more + (end - wide) / each;             // in workgroup:
        header = {r, (int)last_w, first_segment ? 0 : 1, rq.c0, rq.n * G, tile * 16 * NT, h, 0};
      }
      first_segment = false;
    }
    g += (unsigned)(v1 - gi);
    gi = 0;
    if (g < ge && ++h == a.Hkv) {
      h = 0;
      if (++tile == rq.tiles) {
        tile = 0;
        do {
          ++r;
          rq = kv4_request<NT>(a, r, G);
        } while (rq.n == 0 && r + 1 < a.R);
      }
    }
  }
  if (tid == 0) a.head[w] = header;
}

template <int D, int NT>
constexpr int kKv4PerCU = NT == kKv4Wide ? 2 : (D == 128 ? 3 : 4) - (NT - 1);      // workgroups that a CU holds, by the registers

template <int D, int NT>
__global__ __launch_bounds__(kKv4Threads, (kKv4PerCU<D, NT>)) void kv4_attn_kernel(Kv4Args a) {
  kv4_body<D, NT>(a);
}

constexpr int kKv4JoinRows = 4;        // rows of a workgroup, one to a wave

// Joins the parts of the unit that workgroup w began and did not end: those of w and of the workgroups up to
// the last. A wave takes one row: 16 lanes across the dimensions, and every fourth part to each quarter of the
// wave, eight parts' loads in flight per lane; the quarters are joined last. The order is fixed.
template <int D, int NT>
__global__ __launch_bounds__(64 * kKv4JoinRows) void kv4_join_kernel(Kv4Args a) {
  constexpr int CH = D / 16;
  constexpr int DEEP = 8;
  const int w = blockIdx.x;
  const Kv4Head head = a.head[w];
  if (head.r < 0) return;
  const int G = a.H / a.Hkv;
  const int last = head.last;
  const int lane = threadIdx.x & 63, ch = lane & 15;
  const int lr = blockIdx.y * kKv4JoinRows + (threadIdx.x >> 6);
  const int rho = head.row0 + lr;
  if (rho >= head.nrows) return;
  float top = -__builtin_inff(), sum = 0.0f, out[CH] = {};
  for (int i0 = w + (lane >> 4); i0 <= last; i0 += 4 * DEEP) {
    float m[DEEP], l[DEEP];
    f32x4 x[DEEP][CH / 4];
#pragma unroll
    for (int j = 0; j < DEEP; ++j) {
      const int i = min(i0 + 4 * j, last);
      const float* sl = a.part + (size_t)(2 * i + (i == w ? head.slot : 0)) * kKv4PartFloats<D, NT>;
      const float2 ml = *reinterpret_cast<const float2*>(sl + 2 * lr);
      m[j] = ml.x;
      l[j] = ml.y;
#pragma unroll
      for (int c = 0; c < CH / 4; ++c) x[j][c] = *reinterpret_cast<const f32x4*>(sl + 32 * NT + lr * D + ch * CH + 4 * c);
    }
    float t = top;
#pragma unroll
    for (int j = 0; j < DEEP; ++j) t = fmaxf(t, i0 + 4 * j <= last ? m[j] : -__builtin_inff());
    const float was = part_weight(top, t, a.sl2);
    sum *= top == -__builtin_inff() ? 1.0f : was;       // (NaN of a part that has seen no key stays)
#pragma unroll
    for (int e = 0; e < CH; ++e) out[e] *= was;
#pragma unroll
    for (int j = 0; j < DEEP; ++j) {
      if (i0 + 4 * j > last) continue;
      const float wt = part_weight(m[j], t, a.sl2);
      sum += m[j] == -__builtin_inff() ? l[j] : wt * l[j];
#pragma unroll
      for (int c = 0; c < CH / 4; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) out[4 * c + e] += wt * x[j][c][e];
    }
    top = t;
  }
  const float all = max_over_groups(top);
  const float wt = part_weight(top, all, a.sl2);
  sum = sum_over_groups(top == -__builtin_inff() ? sum : wt * sum);
#pragma unroll
  for (int e = 0; e < CH; ++e) out[e] = sum_over_groups(wt * out[e]);
  if (lane >= 16) return;
  const int i = rho / G;
  const float inv = row_factor(sum, max(a.kv_len[head.r], 0) - head.nrows / G + i);
#pragma unroll
  for (int e = 0; e < CH; ++e) out[e] *= inv;
  store_row<CH>(a.o + ((size_t)(head.c0 + i) * a.H + (size_t)(head.h * G + (rho - i * G))) * D + ch * CH, out);
}

}  // namespace
}  // namespace qg
