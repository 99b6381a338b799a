// Attention of new tokens over the paged 4-bit cache, for gfx950.
//
// Bound by the cache's bytes for single tokens (0.53 bytes per element, each read once) and by the vector
// ALU that unpacks them where several query rows share a pass. The mathematics is the online softmax of the
// prompt kernel; what differs is the work split and how the 4-bit operands reach the matrix cores.
//
// Work: a unit is (request, tile of 16 NT query rows, key/value head); the rows of a tile are the query heads
// of the group times the request's new tokens. A unit's keys are cut into granules of 128, the granules of all
// units are numbered in one sequence, and workgroup w of n takes the w-th n-th of them. So requests of any mix
// of lengths load every workgroup alike, a long one is split over many, and the host needs to know no length.
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
#pragma once

#include "attn_kernels.hpp"
#include "serve_kernels.hpp"

namespace qg {
namespace {

constexpr int kKv4Threads = 256;
constexpr int kKv4Waves = kKv4Threads / 64;
constexpr int kKv4Step = 32;                          // keys of a wave's step
constexpr int kKv4Granule = kKv4Step * kKv4Waves;     // keys of a granule

struct Kv4Args {
  const uint16_t* q;
  const uint8_t* cache;
  const int32_t* table;     // [R][W]
  const int32_t* kv_len;
  const int32_t* cu;        // null: one new token per request
  uint16_t* o;
  int4* head;               // [nwg] the unit a workgroup's last segment starts and does not end
  float* part;              // [nwg][2] partial results
  int T, R, H, Hkv, W, pages, page_log2, nwg;
  long qs;
  float sl2;
};

template <int D, int NT>
constexpr int kKv4PartFloats = 16 * NT * (D + 2);

__device__ __forceinline__ int clamp_i(int x, int lo, int hi) { return min(max(x, lo), hi); }

// Tables that the kernels only read, as memory that scalar loads may fetch where the address is uniform.
typedef const __attribute__((address_space(4))) int32_t* const_i32;
__device__ __forceinline__ const_i32 as_const(const int32_t* p) { return (const_i32)p; }

// A request: its first row, its new tokens, its keys (as given, and those that the table has pages for).
struct Kv4Request {
  int c0, n, kv, len, tiles, grans;
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
  q.len = (int)min((long)q.kv, (long)a.W << a.page_log2);
  q.tiles = (q.n * G + 16 * NT - 1) / (16 * NT);
  q.grans = max(1, (q.len + kKv4Granule - 1) / kKv4Granule);
  return q;
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

template <int N>
__device__ __forceinline__ void store_row(uint16_t* p, const float (&v)[N]) {
  static_assert(N == 4 || N == 8, "8 or 16 bytes");
  if constexpr (N == 8)
    *reinterpret_cast<u32x4*>(p) =
        u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
  else
    *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
}

template <int D>
struct Kv4Keys {                  // 32 keys and values as a wave's lanes hold them
  static constexpr int DW = D / 32;
  uint32_t k[2][DW], v[2][DW];
  uint32_t ks[2], vs[2];
};

template <int D, int NT>
__device__ __forceinline__ void kv4_body(const Kv4Args& a) {
  constexpr int DW = D / 32;            // dwords of packed levels in a lane: a quarter of a key's row
  constexpr int DT = D / 16;            // 16-row tiles of O^T
  constexpr int CH = D / 16;            // dimensions of a thread where parts are joined
  __shared__ __attribute__((aligned(16))) uint16_t vbuf[kKv4Waves][32 * D];     // also 16 rows of O in fp32
  __shared__ float ml[kKv4Waves][16 * NT][2];
  __shared__ unsigned long long wsum[kKv4Waves];
  __shared__ int where_r;
  __shared__ unsigned long long where_off;

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, grp = lane >> 4;
  const int G = a.H / a.Hkv;
  const int w = xcd_tile((int)blockIdx.x, a.nwg);

  // the workgroup's range of granules, and the request that it begins in
  unsigned long long total = 0, gs, ge;
  {
    const int per = (a.R + kKv4Threads - 1) / kKv4Threads;
    const int r0 = min(a.R, tid * per), r1 = min(a.R, r0 + per);
    unsigned long long mine = 0;
    for (int r = r0; r < r1; ++r) {
      const Kv4Request q = kv4_request<NT>(a, r, G);
      mine += (unsigned long long)q.tiles * a.Hkv * q.grans;
    }
    unsigned long long inc = mine;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const unsigned long long up = __shfl_up(inc, d);
      if (lane >= d) inc += up;
    }
    if (lane == 63) wsum[wave] = inc;
    __syncthreads();
    unsigned long long base = inc - mine;
#pragma unroll
    for (int i = 0; i < kKv4Waves; ++i) {
      if (i < wave) base += wsum[i];
      total += wsum[i];
    }
    gs = total * (unsigned)w / (unsigned)a.nwg;
    ge = total * ((unsigned)w + 1u) / (unsigned)a.nwg;
    if (gs < ge && base <= gs && gs < base + mine) {
      unsigned long long off = gs - base;
      int r = r0;
      for (; r < r1; ++r) {
        const Kv4Request q = kv4_request<NT>(a, r, G);
        const unsigned long long n = (unsigned long long)q.tiles * a.Hkv * q.grans;
        if (off < n) break;
        off -= n;
      }
      where_r = r;
      where_off = off;
    }
    __syncthreads();
  }
  if (gs >= ge) {
    if (tid == 0) a.head[w] = make_int4(-2, 0, 0, 0);       // takes part in nothing
    return;
  }
  int r = __builtin_amdgcn_readfirstlane(where_r);
  Kv4Request rq = kv4_request<NT>(a, r, G);
  int tile, h, gi;
  {
    const unsigned long long off = where_off;
    const unsigned long long heads = off / (unsigned)rq.grans;      // (tile, head) in one number
    gi = __builtin_amdgcn_readfirstlane((int)(off - heads * (unsigned)rq.grans));
    tile = __builtin_amdgcn_readfirstlane((int)(heads / (unsigned)a.Hkv));
    h = __builtin_amdgcn_readfirstlane((int)(heads - (unsigned long long)tile * (unsigned)a.Hkv));
  }
  unsigned long long g = gs;
  bool first_segment = true;
  int4 header = make_int4(-1, 0, 0, 0);

  const int page_mask = (1 << a.page_log2) - 1;
  const size_t record = (size_t)(D + D / 16) << a.page_log2;
  uint16_t* vw = vbuf[wave];
  auto vswz = [](int key) {
    const int low = 2 * (key & 3) | ((key >> 2) & 1);
    return D == 128 ? low | (key & 8) : low;
  };

  while (g < ge) {
    const int a0 = gi;
    const int a1 = (int)min((unsigned long long)rq.grans, (unsigned long long)a0 + (ge - g));

    // this lane's query rows
    const int row0 = tile * 16 * NT;
    const int nrows = rq.n * G;
    int lim[NT];                                    // keys that the row sees
    bf16x8 qf[NT][DW];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int rho = row0 + 16 * nt + col;
      const int i = rho / G;
      const bool live = rho < nrows;
      lim[nt] = live ? clamp_i(rq.kv - rq.n + i + 1, 0, rq.len) : 0;
      const uint16_t* qp = a.q + (size_t)(rq.c0 + i) * a.qs + (size_t)(h * G + (rho - i * G)) * D + grp * (D / 4);
#pragma unroll
      for (int t = 0; t < DW; ++t)
        qf[nt][t] = live ? __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(qp + 8 * t)) : bf16x8{};
    }
    const int last = (min(row0 + 16 * NT, nrows) - 1) / G;
    const int kmax = clamp_i(rq.kv - rq.n + last + 1, 0, rq.len);           // keys that any row sees
    const int kall = clamp_i(rq.kv - rq.n + row0 / G + 1, 0, rq.len);       // keys that every row sees

    f32x4 acc[NT][DT];
    float m_run[NT], l_run[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      m_run[nt] = -__builtin_inff();
      l_run[nt] = rq.kv > rq.len ? __builtin_nanf("") : 0.0f;   // keys without a page to look in
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) acc[nt][dt] = f32x4{};
    }

    const const_i32 trow = as_const(a.table) + (size_t)r * a.W;
    const int s_end = min(a1 * kKv4Waves, (kmax + kKv4Step - 1) / kKv4Step);
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
        const bool ok = (unsigned)id < (unsigned)a.pages;
        const uint8_t* rec = a.cache + ((size_t)(ok ? id : 0) * a.Hkv + h) * record;
        const uint32_t off = (uint32_t)((key & page_mask) + col);
        const uint32_t voff = off + (1u << a.page_log2);
        const uint32_t sbase = (uint32_t)D << a.page_log2;
        const uint32_t blk = D == 128 ? grp : grp >> 1;
        if constexpr (DW == 4) {
          const u32x4 k4 = *reinterpret_cast<const u32x4*>(rec + (off * (D / 2) + grp * (D / 8)));
          const u32x4 v4 = *reinterpret_cast<const u32x4*>(rec + (voff * (D / 2) + grp * (D / 8)));
#pragma unroll
          for (int t = 0; t < DW; ++t) b.k[i][t] = k4[t], b.v[i][t] = v4[t];
        } else {
          const uint2 k2 = *reinterpret_cast<const uint2*>(rec + (off * (D / 2) + grp * (D / 8)));
          const uint2 v2 = *reinterpret_cast<const uint2*>(rec + (voff * (D / 2) + grp * (D / 8)));
          b.k[i][0] = k2.x, b.k[i][1] = k2.y, b.v[i][0] = v2.x, b.v[i][1] = v2.y;
        }
        const uint32_t ks = rec[sbase + off * (D / 32) + blk], vs = rec[sbase + voff * (D / 32) + blk];
        b.ks[i] = ok ? ks : 255u;             // a page that is none reads as NaN
        b.vs[i] = ok ? vs : 255u;
      }
      return b;
    };

    auto step = [&](Kv4Keys<D>& b, int s) {
      const int key0 = kKv4Step * s;
      const bool need_mask = key0 + kKv4Step > kall;
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
      unsigned long long nan_at[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (need_mask && key0 + 16 * i + col >= kmax) {
          b.vs[i] = 0;
#pragma unroll
          for (int t = 0; t < DW; ++t) b.v[i][t] = 0;
        }
        nan_at[i] = __ballot(b.vs[i] == 255u);
        if (b.vs[i] == 255u) {
          b.vs[i] = 0;
#pragma unroll
          for (int t = 0; t < DW; ++t) b.v[i][t] = 0;
        }
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
        float mloc = fmaxf(fmaxf(fmaxf(sc[nt][0][0], sc[nt][0][1]), fmaxf(sc[nt][0][2], sc[nt][0][3])),
                           fmaxf(fmaxf(sc[nt][1][0], sc[nt][1][1]), fmaxf(sc[nt][1][2], sc[nt][1][3])));
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
        for (int e = 0; e < 8; ++e) {
          p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[nt][e >> 2][e & 3], a.sl2, -ms));
          l_run[nt] += p[e];
        }
        pb[nt] = __builtin_bit_cast(bf16x8, u32x4{pack_bf16x2(p[0], p[1]), pack_bf16x2(p[2], p[3]),
                                                  pack_bf16x2(p[4], p[5]), pack_bf16x2(p[6], p[7])});
      }
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

    int s = a0 * kKv4Waves + wave;
    if (s < s_end) {
      // the next step's keys and values are in flight during a step, and the page numbers of the one after it
      int2 ids = pages_of(s);
      Kv4Keys<D> cur = load(s, ids);
      ids = pages_of(s + kKv4Waves);
      for (;;) {
        const int sn = s + kKv4Waves;
        Kv4Keys<D> nxt;
        if (sn < s_end) {
          nxt = load(sn, ids);
          ids = pages_of(sn + kKv4Waves);
        }
        step(cur, s);
        if (sn >= s_end) break;
        cur = nxt;
        s = sn;
      }
    }

    // join the four waves, 16 rows at a time
    const bool whole = a0 == 0 && a1 == rq.grans;
    float* slot = a.part + (size_t)(2 * w + (first_segment ? 0 : 1)) * kKv4PartFloats<D, NT>;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float* ow = reinterpret_cast<float*>(vw);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
        *reinterpret_cast<f32x4*>(&ow[col * D + (((4 * dt + grp) ^ (col & 7)) << 2)]) = acc[nt][dt];
      const float l = sum_over_groups(l_run[nt]);
      if (grp == 0) {
        ml[wave][16 * nt + col][0] = m_run[nt];
        ml[wave][16 * nt + col][1] = l;
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
      if (whole) {
        if (rho < nrows) {
          const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
          for (int e = 0; e < CH; ++e) out[e] *= inv;
          const int i = rho / G;
          store_row<CH>(a.o + ((size_t)(rq.c0 + i) * a.H + (size_t)(h * G + (rho - i * G))) * D + ch * CH, out);
        }
      } else {
        float* po = slot + 2 * 16 * NT + (16 * nt + row) * D + ch * CH;
#pragma unroll
        for (int c = 0; c < CH / 4; ++c)
          *reinterpret_cast<f32x4*>(po + 4 * c) = f32x4{out[4 * c], out[4 * c + 1], out[4 * c + 2], out[4 * c + 3]};
        if (ch == 0) {
          slot[2 * (16 * nt + row)] = top;
          slot[2 * (16 * nt + row) + 1] = sum;
        }
      }
      __syncthreads();
    }

    if (a0 == 0 && a1 < rq.grans) {          // the unit goes on: this workgroup's block of the second kernel joins it
      const unsigned long long end = g + (unsigned)rq.grans - 1;      // its last granule, in workgroup:
      unsigned int wl = (unsigned int)(end * (unsigned)a.nwg / total);
      while (wl + 1 < (unsigned)a.nwg && total * (wl + 1) / (unsigned)a.nwg <= end) ++wl;
      header = make_int4(r, tile, h, (int)(wl << 1) | (first_segment ? 0 : 1));
    }
    first_segment = false;
    g += (unsigned)(a1 - a0);
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
__global__ __launch_bounds__(kKv4Threads) void kv4_attn_kernel(Kv4Args a) {
  kv4_body<D, NT>(a);
}

// Joins the parts of the unit that workgroup w began and did not end: those of w and of the workgroups up to
// the last, in that order.
template <int D, int NT>
__global__ __launch_bounds__(kKv4Threads) void kv4_join_kernel(Kv4Args a) {
  constexpr int CH = D / 16;
  const int w = blockIdx.x;
  const int4 head = a.head[w];
  if (head.x < 0) return;
  const int G = a.H / a.Hkv;
  const Kv4Request rq = kv4_request<NT>(a, head.x, G);
  const int wl = head.w >> 1;
  const int tid = threadIdx.x, row = tid >> 4, ch = tid & 15;
  for (int nt = 0; nt < NT; ++nt) {
    const int lr = 16 * nt + row;
    const int rho = head.y * 16 * NT + lr;
    if (rho >= rq.n * G) continue;
    auto slot_of = [&](int i) {
      return a.part + (size_t)(2 * i + (i == w ? head.w & 1 : 0)) * kKv4PartFloats<D, NT>;
    };
    float top = -__builtin_inff();
    for (int i = w; i <= wl; ++i)
      if (i == w || a.head[i].x != -2) top = fmaxf(top, slot_of(i)[2 * lr]);
    float sum = 0.0f, out[CH] = {};
    for (int i = w; i <= wl; ++i) {
      if (i != w && a.head[i].x == -2) continue;
      const float* sl = slot_of(i);
      const float m = sl[2 * lr], l = sl[2 * lr + 1];
      const float wt = part_weight(m, top, a.sl2);
      sum += m == -__builtin_inff() ? l : wt * l;
      const float* x = sl + 2 * 16 * NT + lr * D + ch * CH;
#pragma unroll
      for (int c = 0; c < CH / 4; ++c) {
        const f32x4 v = *reinterpret_cast<const f32x4*>(x + 4 * c);
#pragma unroll
        for (int e = 0; e < 4; ++e) out[4 * c + e] += wt * v[e];
      }
    }
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
    for (int e = 0; e < CH; ++e) out[e] *= inv;
    const int i = rho / G;
    store_row<CH>(a.o + ((size_t)(rq.c0 + i) * a.H + (size_t)(head.z * G + (rho - i * G))) * D + ch * CH, out);
  }
}

}  // namespace
}  // namespace qg
