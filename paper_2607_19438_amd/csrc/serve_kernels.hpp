// Kernels of a serving step around the projections: the plan of a ragged batch, rotary positions, and the
// paged 4-bit cache's store and load. All are bound by HBM or, at a few tokens, by launch and load latency.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kv4_levels.hpp"
#include "qgemm_kernels.hpp"

namespace qg {
namespace {

// ---------------------------------------------------------------------------
// plan: where the tokens of a ragged batch sit
// ---------------------------------------------------------------------------

constexpr int kPlanThreads = 256;
constexpr int kPlanTokens = 256;       // tokens of a workgroup
constexpr int kPlanMaxR = 4096;        // requests: three int32 per request in LDS (48 KiB)

struct PlanArgs {
  const int32_t* kv_len;
  const int32_t* q_len;
  int32_t* table;         // [R][W]
  const int32_t* free_pages;
  int32_t* cu_q;
  int32_t* positions;
  int32_t* slots;
  int32_t* total_len;
  int32_t* used;
  int R, W, F, page_log2, T;
};

// One launch: every workgroup scans the lengths of all requests for itself (R <= 4096: a few loads and one
// scan per thread) and then finds the request of each of its tokens in LDS, so nothing waits for another
// workgroup. A page that the step adds has its first token in the step (its first position is at or past
// kv_len), and the thread of that token writes its table entry.
// Bound by its chain of loads: 64 requests of a token 2.6 us, 500 requests and 34410 rows 3.4 (1024 tokens to a
// workgroup 6.8, 512 5.0, 256 4.2 between launches).
__global__ __launch_bounds__(kPlanThreads) void kv_plan_kernel(PlanArgs a) {
  extern __shared__ int32_t plan_lds[];
  __shared__ int32_t wave_q[kPlanThreads / 64], wave_p[kPlanThreads / 64];
  int32_t* cu = plan_lds;              // [R] first token of each request
  int32_t* first = plan_lds + a.R;     // [R] pages that the requests before it take from the free list
  int32_t* kv = plan_lds + 2 * a.R;    // [R]
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int R = a.R, mask = (1 << a.page_log2) - 1;
  auto pages = [&](int n) { return (int)(((unsigned)n + (unsigned)mask) >> a.page_log2); };
  const int per = (R + kPlanThreads - 1) / kPlanThreads;
  const int r0 = tid * per, r1 = min(R, r0 + per);
  int sq = 0, sp = 0;
  for (int r = r0; r < r1; ++r) {
    const int n = max(a.kv_len[r], 0), m = max(a.q_len[r], 0);
    kv[r] = n;
    cu[r] = sq;                        // within the thread's requests; the threads before are added below
    first[r] = sp;
    sq += m;
    sp += pages(n + m) - pages(n);
  }
  int iq = sq, ip = sp;                // inclusive over the wave
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int uq = __shfl_up(iq, d), up = __shfl_up(ip, d);
    if (lane >= d) {
      iq += uq;
      ip += up;
    }
  }
  if (lane == 63) {
    wave_q[wave] = iq;
    wave_p[wave] = ip;
  }
  __syncthreads();
  int bq = iq - sq, bp = ip - sp, tq = 0, tp = 0;
#pragma unroll
  for (int w = 0; w < kPlanThreads / 64; ++w) {
    if (w < wave) {
      bq += wave_q[w];
      bp += wave_p[w];
    }
    tq += wave_q[w];
    tp += wave_p[w];
  }
  for (int r = r0; r < r1; ++r) {
    cu[r] += bq;
    first[r] += bp;
    if (blockIdx.x == 0) {
      a.cu_q[r] = cu[r];
      a.total_len[r] = kv[r] + max(a.q_len[r], 0);
    }
  }
  if (blockIdx.x == 0 && tid == 0) {
    a.cu_q[R] = tq;
    a.used[0] = tp;
  }
  __syncthreads();
  const int t0 = blockIdx.x * kPlanTokens;
#pragma unroll
  for (int i = 0; i < kPlanTokens / kPlanThreads; ++i) {
    const int t = t0 + i * kPlanThreads + tid;
    if (t >= a.T) break;
    int pos = 0;
    long slot = -1;
    if (t < tq) {
      int lo = 0, hi = R - 1;          // the last request that starts at or before t: one of no tokens starts
      while (lo < hi) {                // where the next one does
        const int mid = (lo + hi + 1) >> 1;
        if (cu[mid] <= t) lo = mid;
        else hi = mid - 1;
      }
      const int n = kv[lo];
      pos = n + t - cu[lo];
      const int j = pos >> a.page_log2;
      const int fresh = j - pages(n);
      if (j >= 0 && j < a.W) {
        int id = -1;
        int32_t* entry = a.table + (size_t)lo * a.W + j;
        if (fresh < 0) {
          id = *entry;
        } else {
          const long at = (long)first[lo] + fresh;
          if (at >= 0 && at < a.F) id = a.free_pages[at];
          if ((pos & mask) == 0) *entry = id;
        }
        if (id >= 0) slot = ((long)id << a.page_log2) + (pos & mask);
      }
    }
    a.positions[t] = pos;
    a.slots[t] = slot > 0x7fffffffL ? -1 : (int32_t)slot;
  }
}

// ---------------------------------------------------------------------------
// rotary positions
// ---------------------------------------------------------------------------

constexpr int kRopeThreads = 256;
constexpr int kRopeMaxPairs = 256;     // (sine, cosine) of a workgroup's tokens in LDS: 4 x 256 x 8 bytes

struct RopeArgs {
  const void* x;
  const int32_t* positions;
  const double* inv_freq;
  uint16_t* y;
  int T, heads, rot_heads, D, rot;
  long xs, ys;             // elements between tokens
  float gain;
  int tokens;              // of a workgroup
  int parts;               // workgroups that share the heads of those tokens
};

__device__ __forceinline__ float load_one(const float* p) { return *p; }
__device__ __forceinline__ float load_one(const uint16_t* p) { return __builtin_bit_cast(float, (uint32_t)*p << 16); }

__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
  const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
}
__device__ __forceinline__ void load8(const uint16_t* p, float (&v)[8]) {
  const u32x4 w = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __builtin_bit_cast(float, w[i] << 16);
    v[2 * i + 1] = __builtin_bit_cast(float, w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void store8(uint16_t* p, const float (&v)[8]) {
  *reinterpret_cast<u32x4*>(p) =
      u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
}

// (a, b) turned by w = (cosine, sine), each with one product rounded and one fused; written out, so that every form of
// the kernel gives the same bits.
__device__ __forceinline__ void rotate(float& a, float& b, float2 w) {
  const float a0 = a;
  a = __builtin_fmaf(a0, w.x, -(b * w.y));
  b = __builtin_fmaf(a0, w.y, b * w.x);
}

// The sine and cosine of every (token, pair) are evaluated once per workgroup and shared by all heads through
// LDS. The angle is taken in turns in fp64 (position x frequency / 2 pi, less its whole turns): at position
// 10^6 an fp32 product is off by 0.06 radians. What is left is below half a turn, so fp32 keeps 2^-25 of one.
// Bound by HBM: 8192 rows of 40 x 128 from fp32 in 46.4 us, 5.4 TB/s (40 into the buffer that the call before wrote, which
// is still in the memory-side cache); at 16 rows by its one launch, 3.2 us.
// WIDE: 16 elements per thread and step, with 16-byte accesses, where sizes, strides and addresses allow it;
// else two elements. (The first step's loads before the sines, and each next step's before the last one's work:
// 3000 rows of 24 x 64 5.2 -> 5.5 us, 8000 rows 10.0 -> 11.8, 16 rows of 40 x 128 3.1 -> 3.3. The waves are
// enough to cover them.)
template <typename TX, bool INTER, bool WIDE>
__global__ __launch_bounds__(kRopeThreads) void rope_kernel(RopeArgs a) {
  constexpr int N = WIDE ? 8 : 1;      // elements of a thread's two pieces
  __shared__ float2 cs[4 * kRopeMaxPairs];
  const int tid = threadIdx.x;
  const int group = blockIdx.x / a.parts, part = blockIdx.x - group * a.parts;
  const int t0 = group * a.tokens;
  const int nt = min(a.tokens, a.T - t0);
  const int pairs = a.rot >> 1;
  const int units = a.D / (2 * N);                    // of a head
  const int turned = a.rot / (2 * N);                 // of them rotated, in the heads that are
  const int per = (a.heads + a.parts - 1) / a.parts;
  const int h0 = part * per, nh = min(per, a.heads - h0);
  const int n = nt * nh * units;
  struct Item {
    int t, u, o1, o2;      // token, unit, offsets of its two pieces in the head
    bool rot;
    size_t head;           // head x D
    float p[N], q[N];
  };
  auto fetch = [&](int i) {
    Item m;
    m.u = i % units;
    const int hu = i / units;
    const int h = h0 + hu % nh;
    m.t = hu / nh;
    m.rot = h < a.rot_heads && m.u < turned;
    m.o1 = m.rot && !INTER ? N * m.u : 2 * N * m.u;
    m.o2 = m.rot && !INTER ? N * m.u + pairs : 2 * N * m.u + N;
    m.head = (size_t)h * a.D;
    const TX* x = static_cast<const TX*>(a.x) + (size_t)(t0 + m.t) * a.xs + m.head;
    if constexpr (WIDE) {
      load8(x + m.o1, m.p);
      load8(x + m.o2, m.q);
    } else {
      m.p[0] = load_one(x + m.o1);
      m.q[0] = load_one(x + m.o2);
    }
    return m;
  };
  for (int i = tid; i < nt * pairs; i += kRopeThreads) {
    const int t = i / pairs;
    double turn = (double)a.positions[t0 + t] * (a.inv_freq[i - t * pairs] * 0.15915494309189535);
    turn -= rint(turn);
    float s, c;
    sincospif(2.0f * (float)turn, &s, &c);
    cs[i] = make_float2(c * a.gain, s * a.gain);
  }
  __syncthreads();
  for (int i = tid; i < n; i += kRopeThreads) {
    Item item = fetch(i);
    if (item.rot) {
      const float2* w = cs + item.t * pairs + N * item.u;
      if constexpr (WIDE && INTER) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          rotate(item.p[2 * k], item.p[2 * k + 1], w[k]);
          rotate(item.q[2 * k], item.q[2 * k + 1], w[4 + k]);
        }
      } else {
#pragma unroll
        for (int k = 0; k < N; ++k) rotate(item.p[k], item.q[k], w[k]);
      }
    }
    uint16_t* y = a.y + (size_t)(t0 + item.t) * a.ys + item.head;
    if constexpr (WIDE) {
      store8(y + item.o1, item.p);
      store8(y + item.o2, item.q);
    } else {
      const uint32_t w = pack_bf16x2(item.p[0], item.q[0]);
      y[item.o1] = (uint16_t)w;
      y[item.o2] = (uint16_t)(w >> 16);
    }
  }
}

// ---------------------------------------------------------------------------
// the paged 4-bit cache
// ---------------------------------------------------------------------------

constexpr int kCacheThreads = 256;

// Byte offsets within the record of one (page, head): key codes, value codes, key scales, value scales.
struct Kv4Layout {
  int D, page_log2;
  __device__ __forceinline__ int codes(int which, int off, int unit) const {       // of 8 elements
    return ((which << page_log2) + off) * (D >> 1) + 4 * unit;
  }
  __device__ __forceinline__ int scale(int which, int off, int block) const {
    return (D << page_log2) + ((which << page_log2) + off) * (D >> 5) + block;
  }
  __device__ __forceinline__ size_t record() const { return (size_t)(D + (D >> 4)) << page_log2; }
};

struct CacheArgs {
  const uint16_t* k;
  const uint16_t* v;
  uint16_t* ko;
  uint16_t* vo;
  uint8_t* cache;
  const int32_t* slots;
  long ks, vs;             // elements between tokens
  unsigned n;              // threads: tokens x 2 x heads x (D / 8)
  int Hkv, nslots;
  int units_log2;          // of D / 8
  Kv4Layout lay;
};

// A thread moves 8 elements: 16 bytes of bf16 and 4 of codes, so that a wave's accesses on either side are contiguous
// within a token; four neighbouring threads share a block of 32 and its scale. (A block to a thread, 64 bytes of it 16
// at a time: store and load of 8191 rows of 8 x 64 16.0 us, so 12.9, 3.3 TB/s over both; of 64 rows 8.1, 6.3.)
struct CacheItem {
  long t;
  int which, h, unit;      // keys or values, head, 8 elements of it
};
__device__ __forceinline__ CacheItem cache_item(const CacheArgs& a, unsigned i) {
  const unsigned row = i >> a.units_log2, per = 2u * (unsigned)a.Hkv;
  const unsigned t = row / per;
  unsigned h = row - t * per;
  const bool second = h >= (unsigned)a.Hkv;
  if (second) h -= (unsigned)a.Hkv;
  return {(long)t, second ? 1 : 0, (int)h, (int)(i & ((1u << a.units_log2) - 1u))};
}

// A block's exponent: that of its largest magnitude rounded to two significant bits (so 1.75 and up counts as
// the next power of two, whose half is the level 4; the plain exponent would cut those to 6 of 8), less 2 for
// the largest level's 4 <= 6 < 8. Zero and the smallest blocks take 2^-126, the largest 2^125 (6 of it are the most
// below bf16's end); a block with an infinity or NaN 255, which reads as NaN.
__device__ __forceinline__ uint32_t block_exponent(uint32_t top) {   // bits of the largest |x|
  if (top >= 0x7f800000u) return 255u;
  const uint32_t e = (top + 0x200000u) >> 23;
  return min(max(e, 3u) - 2u, 252u);
}

__global__ __launch_bounds__(kCacheThreads) void kv4_store_kernel(CacheArgs a) {
  const unsigned i = blockIdx.x * kCacheThreads + threadIdx.x;
  if (i >= a.n) return;          // (n is a multiple of 4: the threads of a block are all here or all gone)
  const CacheItem it = cache_item(a, i);
  const int slot = a.slots[it.t];
  const u32x4 w = *reinterpret_cast<const u32x4*>((it.which ? a.v + it.t * a.vs : a.k + it.t * a.ks) + (size_t)it.h * a.lay.D + 8 * it.unit);
  uint32_t top = 0;              // bf16 magnitudes order as integers, NaN above infinity
#pragma unroll
  for (int c = 0; c < 4; ++c) top = max(top, max((w[c] << 16) & 0x7fff0000u, w[c] & 0x7fff0000u));
  top = max(top, (uint32_t)__shfl_xor((int)top, 1));
  top = max(top, (uint32_t)__shfl_xor((int)top, 2));
  if ((unsigned)slot >= (unsigned)a.nslots) return;
  const uint32_t e = block_exponent(top);
  uint32_t codes = 0;
  if (e != 255u) {
    const float unit = __builtin_bit_cast(float, e << 23);
    // v_cvt_scalef32_pk_fp4_bf16: x / unit to the next level, ties to the even code
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(bf16x2, (uint32_t)w[0]), unit, 0);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(bf16x2, (uint32_t)w[1]), unit, 1);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(bf16x2, (uint32_t)w[2]), unit, 2);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(bf16x2, (uint32_t)w[3]), unit, 3);
  }
  const int page = slot >> a.lay.page_log2, off = slot & ((1 << a.lay.page_log2) - 1);
  uint8_t* rec = a.cache + ((size_t)page * a.Hkv + it.h) * a.lay.record();
  *reinterpret_cast<uint32_t*>(rec + a.lay.codes(it.which, off, it.unit)) = codes;
  if ((it.unit & 3) == 0) rec[a.lay.scale(it.which, off, it.unit >> 2)] = (uint8_t)e;
}

__global__ __launch_bounds__(kCacheThreads) void kv4_load_kernel(CacheArgs a) {
  const unsigned i = blockIdx.x * kCacheThreads + threadIdx.x;
  if (i >= a.n) return;
  const CacheItem it = cache_item(a, i);
  const int slot = a.slots[it.t];
  if ((unsigned)slot >= (unsigned)a.nslots) return;
  const int page = slot >> a.lay.page_log2, off = slot & ((1 << a.lay.page_log2) - 1);
  const uint8_t* rec = a.cache + ((size_t)page * a.Hkv + it.h) * a.lay.record();
  const uint32_t codes = *reinterpret_cast<const uint32_t*>(rec + a.lay.codes(it.which, off, it.unit));
  const uint32_t e = rec[a.lay.scale(it.which, off, it.unit >> 2)];
  *reinterpret_cast<u32x4*>((it.which ? a.vo : a.ko) + ((size_t)it.t * a.Hkv + it.h) * a.lay.D + 8 * it.unit) =
      fp4_unit(codes, __builtin_bit_cast(float, e << 23));
}

}  // namespace
}  // namespace qg
