// Kernels of beam search: the selection over beams and vocabulary, and the tables and pages of the beams after it.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "qgemm_kernels.hpp"

namespace qg {
namespace {

// ---------------------------------------------------------------------------
// selection
// ---------------------------------------------------------------------------
//
// A candidate (beam b, token v) is worth score[b] + x[b][v] - lse[b], lse = log sum_v exp x[b][v]. Within a beam the
// order is that of the logits, so the first kernel needs no lse: a workgroup takes a piece of a row in one pass over
// it, carries maximum and sum as an online softmax does, and keeps the piece's K largest logits. The second kernel
// has the B * pieces * K of a request that are left and computes their values in 64 bits: what beams differ by
// decides between candidates, and at a score of -100 steps of 32 bits are 2^-17.
// Bound by the logits' bytes; with few rows by the chain load - bound - selection - second launch.

constexpr int kBeamThreads = 256;
constexpr int kBeamMaxB = 64;          // beams of a request
constexpr int kBeamMaxK = 128;         // candidates that are taken
constexpr int kBeamElems = 16;         // logits of a thread and step
constexpr int kBeamStep = kBeamThreads * kBeamElems;
constexpr int kBeamList = 16 * kBeamMaxK + kBeamMaxK;      // logits that a workgroup holds before it selects
constexpr int kBeamMost = 8192;        // of a request that are left for the second kernel, at most
static_assert(kBeamList % kBeamThreads == 128, "see beam_keep");
constexpr int kBeamKept = kBeamMaxK * ((kBeamList + kBeamThreads - 1) / kBeamThreads);

// A logit and its token as one number, larger logits first, then lower tokens. 0 stands for none.
__device__ __forceinline__ uint64_t beam_key(float x, uint32_t v) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x + 0.0f);         // -0 as 0
  return ((uint64_t)(u ^ ((u >> 31) ? 0xffffffffu : 0x80000000u)) << 32) | (0xffffffffu - v);
}
__device__ __forceinline__ float beam_logit(uint64_t key) {
  const uint32_t u = (uint32_t)(key >> 32);
  return __builtin_bit_cast(float, u ^ ((u >> 31) ? 0x80000000u : 0xffffffffu));
}
__device__ __forceinline__ int beam_token(uint64_t key) { return (int)(0xffffffffu - (uint32_t)key); }

// A number of 64 bits as one whose order as an integer is its own. (No NaN comes here.)
__device__ __forceinline__ uint64_t beam_order(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x + 0.0);
  return u ^ ((u >> 63) ? ~0ull : 1ull << 63);
}

struct BeamStat {
  double sum;         // of exp(x - top) over a piece
  float top;
  float pad;
};

struct BeamArgs {
  const void* x;            // [R * B][V] at `stride`
  const float* scores;      // [R][B]
  const uint8_t* finished;  // [R][B] or null
  float* out_scores;        // [R][K]
  int32_t* out_beams;
  int32_t* out_tokens;
  BeamStat* stat;           // [R * B][pieces]
  uint64_t* cand;           // [R * B][pieces][K]
  long stride;
  int R, B, V, K, pieces, piece;      // piece: logits of one, a multiple of kBeamStep
  int end;
};

// Whether a beam's logits are candidates: not those of an ended one, nor of one whose score leaves nothing.
__device__ __forceinline__ bool beam_reads(const BeamArgs& a, int row) {
  return a.scores[row] > -__builtin_inff() && !(a.finished && a.finished[row]);
}

struct BeamLds {
  uint64_t list[kBeamList];
  uint64_t kept[kBeamKept];
  uint64_t each[kBeamThreads];
  uint64_t bound;
  int count, first_out, kept_n;
};

// How many threads' keys are larger than this one's.
__device__ __forceinline__ int beam_place(BeamLds& s, uint64_t mine) {
  s.each[threadIdx.x] = mine;
  __syncthreads();
  int n = 0;
#pragma unroll 16
  for (int i = 0; i < kBeamThreads; ++i) n += s.each[i] > mine;
  __syncthreads();
  return n;
}

// The K-th largest of the threads' keys, 1 if there are fewer: a lower bound of the K-th largest of all that they
// hold, which K threads at most reach. (Keys are distinct, but for 0.)
__device__ __forceinline__ uint64_t beam_bound(BeamLds& s, uint64_t mine, int K) {
  if (threadIdx.x == 0) s.bound = 1;
  const int place = beam_place(s, mine);      // (its barriers are behind the write above)
  if (place == K - 1 && mine) s.bound = mine;
  __syncthreads();
  const uint64_t bound = s.bound;
  __syncthreads();
  return bound;
}

// The K largest of list[0 .. n) to its front, in order; how many there are. list[.. K) behind them is 0.
__device__ __forceinline__ int beam_keep(BeamLds& s, int n, int K) {
  const int tid = threadIdx.x;
  uint64_t top = 0;
  for (int i = tid; i < n; i += kBeamThreads) top = max(top, s.list[i]);
  if (tid == 0) s.kept_n = 0;
  const uint64_t from = beam_bound(s, top, K);
  for (int i = tid; i < n; i += kBeamThreads) {
    const uint64_t k = s.list[i];
    if (k >= from) s.kept[atomicAdd(&s.kept_n, 1)] = k;       // a set: their order does not matter
  }
  __syncthreads();
  const int m = s.kept_n;
  for (int i = tid; i < K; i += kBeamThreads) s.list[i] = 0;
  __syncthreads();
  for (int i = tid; i < m; i += kBeamThreads) {
    const uint64_t k = s.kept[i];
    int p = 0;
    for (int j = 0; j < m; ++j) p += s.kept[j] > k;
    if (p < K) s.list[p] = k;
  }
  __syncthreads();
  return min(m, K);
}

typedef uint32_t u32x4_by4 __attribute__((ext_vector_type(4), aligned(4)));      // rows need no more than their elements' alignment
typedef uint32_t u32x4_by2 __attribute__((ext_vector_type(4), aligned(2)));

template <typename T>
struct BeamLoad {
  static constexpr int kWide = 16 / sizeof(T);      // logits of a load
  static constexpr int kLoads = kBeamElems / kWide;
  using vec = std::conditional_t<sizeof(T) == 4, u32x4_by4, u32x4_by2>;
  static __device__ __forceinline__ float one(const T* p) {
    if constexpr (sizeof(T) == 4) return *p;
    else return __builtin_bit_cast(float, (uint32_t)*p << 16);
  }
  static __device__ __forceinline__ void spread(const u32x4& w, float* x) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t u = w[e];
      if constexpr (sizeof(T) == 4) {
        x[e] = __builtin_bit_cast(float, u);
      } else {
        x[2 * e] = __builtin_bit_cast(float, u << 16);
        x[2 * e + 1] = __builtin_bit_cast(float, u & 0xffff0000u);
      }
    }
  }
};

template <typename T>
__global__ __launch_bounds__(kBeamThreads) void beam_rows_kernel(BeamArgs a) {
  using L = BeamLoad<T>;
  __shared__ BeamLds s;
  __shared__ double wave_sum[kBeamThreads / 64];
  __shared__ float wave_top[kBeamThreads / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int row = blockIdx.x / a.pieces, piece = blockIdx.x - row * a.pieces;
  if (!beam_reads(a, row)) return;                  // the second kernel asks the same
  const T* x0 = static_cast<const T*>(a.x) + (size_t)row * a.stride;
  const int v_begin = piece * a.piece, v_end = min(a.V, v_begin + a.piece);
  const float ninf = -__builtin_inff(), log2e = 1.4426950408889634f;
  float top = ninf;
  double sum = 0.0;
  uint64_t from = 0;             // candidates are above it
  if (tid == 0) s.count = 0, s.first_out = kBeamList;
  __syncthreads();
  for (int v0 = v_begin; v0 < v_end; v0 += kBeamStep) {
    float x[kBeamElems];
    auto token = [&](int i) { return v0 + ((i / L::kWide) * kBeamThreads + tid) * L::kWide + i % L::kWide; };
#pragma unroll
    for (int j = 0; j < L::kLoads; ++j) {
      const int v = token(j * L::kWide);
      if (v + L::kWide <= v_end) {
        L::spread(__builtin_bit_cast(u32x4, *reinterpret_cast<const typename L::vec*>(x0 + v)), x + j * L::kWide);
      } else {
#pragma unroll
        for (int e = 0; e < L::kWide; ++e) x[j * L::kWide + e] = v + e < v_end ? L::one(x0 + v + e) : ninf;
      }
    }
    float most = x[0];
#pragma unroll
    for (int i = 1; i < kBeamElems; ++i) most = fmaxf(most, x[i]);
    if (most > top) {
      sum *= (double)__builtin_amdgcn_exp2f((top - most) * log2e);
      top = most;
    }
    const float ref = top == ninf ? 0.0f : top;
    float part = 0.0f;
#pragma unroll
    for (int i = 0; i < kBeamElems; ++i) part += __builtin_amdgcn_exp2f((x[i] - ref) * log2e);
    sum += (double)part;
    // what is above the bound, into the list
    uint32_t pending = 0;
    uint64_t mine = 0;
#pragma unroll
    for (int i = 0; i < kBeamElems; ++i) {
      const uint64_t k = x[i] > ninf ? beam_key(x[i], (uint32_t)token(i)) : 0;
      if (k > from) pending |= 1u << i;
      mine = max(mine, k);
    }
    if (v0 == v_begin) {
      from = beam_bound(s, mine, a.K) - 1;
#pragma unroll
      for (int i = 0; i < kBeamElems; ++i)
        if (!(x[i] > ninf) || beam_key(x[i], (uint32_t)token(i)) <= from) pending &= ~(1u << i);
    }
    while (__syncthreads_or(pending != 0)) {
      if (pending) {
        const int n = __builtin_popcount(pending);
        int at = atomicAdd(&s.count, n);
        if (at + n <= kBeamList) {
#pragma unroll
          for (int i = 0; i < kBeamElems; ++i)
            if (pending >> i & 1) s.list[at++] = beam_key(x[i], (uint32_t)token(i));
          pending = 0;
        } else {
          atomicMin(&s.first_out, at);        // from here on the list holds nothing
        }
      }
      __syncthreads();
      if (s.count > kBeamList) {              // full: keep the best, and try again with what is still above them
        const int n = beam_keep(s, min(s.first_out, kBeamList), a.K);
        if (n == a.K) from = s.list[a.K - 1];
        __syncthreads();
        if (tid == 0) s.count = n, s.first_out = kBeamList;
#pragma unroll
        for (int i = 0; i < kBeamElems; ++i)
          if (beam_key(x[i], (uint32_t)token(i)) <= from) pending &= ~(1u << i);
      }
    }
  }
  beam_keep(s, s.count, a.K);
  uint64_t* out = a.cand + (size_t)blockIdx.x * a.K;
  for (int i = tid; i < a.K; i += kBeamThreads) out[i] = s.list[i];
  // the threads' maxima and sums as one
  float all = top;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) all = fmaxf(all, __shfl_xor(all, d));
  if (lane == 0) wave_top[wave] = all;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kBeamThreads / 64; ++i) all = fmaxf(all, wave_top[i]);
  sum = top == ninf ? sum : sum * exp((double)top - (double)all);
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d);
  if (lane == 0) wave_sum[wave] = sum;
  __syncthreads();
  if (tid == 0) {
    double t = 0.0;
#pragma unroll
    for (int i = 0; i < kBeamThreads / 64; ++i) t += wave_sum[i];
    a.stat[blockIdx.x] = {t, all, 0.0f};
  }
}

// One workgroup to a request. Candidate e = (beam, piece, place in the piece's list); equal values go to the lower e.
__global__ __launch_bounds__(kBeamThreads) void beam_join_kernel(BeamArgs a) {
  extern __shared__ uint64_t kept_value[];
  __shared__ double lse[kBeamMaxB];
  __shared__ float score[kBeamMaxB];
  __shared__ uint64_t each[kBeamThreads];
  __shared__ int each_at[kBeamThreads];
  __shared__ uint64_t bound;
  __shared__ int bound_at, kept_n;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = blockIdx.x;
  const int per = a.pieces * a.K, n = a.B * per;
  int* kept_at = reinterpret_cast<int*>(kept_value + min(n, a.K * ((n + kBeamThreads - 1) / kBeamThreads)));
  const float ninf = -__builtin_inff();
  for (int b = wave; b < a.B; b += kBeamThreads / 64) {
    const int row = r * a.B + b;
    if (lane == 0) score[b] = a.scores[row];
    double sum = 0.0;
    float top = ninf;
    if (beam_reads(a, row)) {
      for (int p = lane; p < a.pieces; p += 64) top = fmaxf(top, a.stat[(size_t)row * a.pieces + p].top);
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
      for (int p = lane; p < a.pieces; p += 64) {
        const BeamStat st = a.stat[(size_t)row * a.pieces + p];
        sum += st.top == ninf ? st.sum : st.sum * exp((double)st.top - (double)top);
      }
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d);
    }
    if (lane == 0) lse[b] = (double)top + log(sum);       // NaN where a logit is NaN or +inf: its beam has no candidates
  }
  if (tid == 0) bound = 1, bound_at = n, kept_n = 0;
  __syncthreads();
  const uint64_t* cand = a.cand + (size_t)r * n;
  // a candidate's value as an ordered integer, 0 for none
  auto value = [&](int e) -> uint64_t {
    const int b = e / per;
    if (!beam_reads(a, r * a.B + b)) {
      const bool one = e == b * per && score[b] > ninf;   // an ended beam's only candidate
      return one ? beam_order((double)score[b]) : 0;
    }
    const uint64_t k = cand[e];
    if (!k) return 0;
    const double v = (double)score[b] + ((double)beam_logit(k) - lse[b]);
    return v > (double)ninf ? beam_order(v) : 0;
  };
  uint64_t top = 0;
  int top_at = n;
  for (int e = tid; e < n; e += kBeamThreads) {
    const uint64_t v = value(e);
    if (v > top) top = v, top_at = e;
  }
  each[tid] = top;
  each_at[tid] = top_at;
  __syncthreads();
  int place = 0;
#pragma unroll 8
  for (int i = 0; i < kBeamThreads; ++i) place += each[i] > top || (each[i] == top && each_at[i] < top_at);
  if (place == a.K - 1 && top) bound = top, bound_at = top_at;
  __syncthreads();
  const uint64_t from = bound;
  const int from_at = bound_at;
  for (int e = tid; e < n; e += kBeamThreads) {
    const uint64_t v = value(e);
    if (v > from || (v == from && e <= from_at)) {
      const int i = atomicAdd(&kept_n, 1);
      kept_value[i] = v;
      kept_at[i] = e;
    }
  }
  __syncthreads();
  const int m = kept_n;
  float* os = a.out_scores + (size_t)r * a.K;
  int32_t* ob = a.out_beams + (size_t)r * a.K;
  int32_t* ot = a.out_tokens + (size_t)r * a.K;
  for (int i = tid; i < m; i += kBeamThreads) {
    const uint64_t v = kept_value[i];
    const int e = kept_at[i];
    int p = 0;
    for (int j = 0; j < m; ++j) p += kept_value[j] > v || (kept_value[j] == v && kept_at[j] < e);
    if (p >= a.K) continue;
    const int b = e / per;
    os[p] = (float)__builtin_bit_cast(double, v ^ ((v >> 63) ? 1ull << 63 : ~0ull));
    ob[p] = b;
    ot[p] = beam_reads(a, r * a.B + b) ? beam_token(cand[e]) : a.end;
  }
  for (int p = m + tid; p < a.K; p += kBeamThreads) os[p] = ninf, ob[p] = -1, ot[p] = a.end;
}

// ---------------------------------------------------------------------------
// tables and pages after a selection
// ---------------------------------------------------------------------------

constexpr int kReorderThreads = 256;
constexpr int kReorderMaxRows = 1 << 16;       // R * B

struct ReorderArgs {
  const int32_t* table;       // [R * B][W]
  const int32_t* kv_len;
  const int32_t* parents;
  const int32_t* free_pages;
  const int32_t* keep;        // [R] or null
  int32_t* new_table;
  int32_t* new_len;
  int32_t* src;               // [R * B]
  int32_t* dst;
  int32_t* used;
  int32_t* released;          // [Q]
  int32_t* n_released;
  int32_t* counts;            // [R * blocks] pages that a workgroup's columns release
  int R, B, W, F, Q, page_log2, blocks;
};

struct ReorderBeams {
  int len[kBeamMaxB], have[kBeamMaxB];                   // old rows: tokens, and pages (within the table)
  int parent[kBeamMaxB], fresh[kBeamMaxB];               // new rows: old row or -1; place in the free list or -1
  unsigned long long live, childless;                    // old rows that have children; that have pages and none
  int taken;                                             // new rows with a fresh page
  int wave[kReorderThreads / 64];
};

// The request's beams; returns how many pages the requests before it take from the free list. Every workgroup counts for
// itself, so that nothing waits for another.
__device__ __forceinline__ int reorder_beams(const ReorderArgs& a, int r, ReorderBeams& s) {
  const int tid = threadIdx.x, lane = tid & 63, B = a.B, mask = (1 << a.page_log2) - 1;
  // whether new row k of request q takes a fresh page: not its parent's first child, and the parent's last page partly filled
  auto takes_page = [&](int q, int k) {
    const int32_t* of = a.parents + (size_t)q * B;
    const int p = of[k];
    if ((unsigned)p >= (unsigned)B || (max(a.kv_len[(size_t)q * B + p], 0) & mask) == 0) return false;
    bool again = false;
    for (int i = 0; i < k; ++i) again |= of[i] == p;
    return again;
  };
  int mine = 0;
  for (int row = tid; row < r * B; row += kReorderThreads) mine += takes_page(row / B, row % B);
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) mine += __shfl_xor(mine, d);
  if (lane == 0) s.wave[tid >> 6] = mine;
  if (tid < 64) {            // B <= 64: a lane of the first wave to a beam
    const bool in = tid < B;
    const int n = in ? max(a.kv_len[(size_t)r * B + tid], 0) : 0;
    const int have = (int)min(((long)n + mask) >> a.page_log2, (long)a.W);
    const int of = in ? a.parents[(size_t)r * B + tid] : -1;
    const int p = (unsigned)of < (unsigned)B ? of : -1;
    const unsigned long long fresh = __ballot(in && takes_page(r, in ? tid : 0));
    if (in) {
      s.len[tid] = n;
      s.have[tid] = have;
      s.parent[tid] = p;
      s.fresh[tid] = fresh >> tid & 1 ? __builtin_popcountll(fresh & ((1ull << tid) - 1)) : -1;
    }
    unsigned long long live = p >= 0 ? 1ull << p : 0ull;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) live |= __shfl_xor(live, d);
    const unsigned long long held = __ballot(have > 0);
    if (tid == 0) s.live = live, s.childless = held & ~live, s.taken = __builtin_popcountll(fresh);
  }
  __syncthreads();
  int before = 0;
#pragma unroll
  for (int i = 0; i < kReorderThreads / 64; ++i) before += s.wave[i];
  return before;
}

// Of the column's old entries, those that no new row holds any more: bit b for old row b. A page stands in the same column
// of all rows that share it, and a row's children hold all of its pages, so only rows without children can lose one.
__device__ __forceinline__ unsigned long long reorder_gone(const ReorderArgs& a, const ReorderBeams& s, const int32_t* old, int j) {
  unsigned long long gone = 0;
  for (unsigned long long m = s.childless; m; m &= m - 1) {
    const int b = __builtin_ctzll(m);
    if (j >= s.have[b]) continue;
    const int id = old[(size_t)b * a.W + j];
    bool stays = id < 0;
    for (unsigned long long l = s.live; l && !stays; l &= l - 1) {
      const int p = __builtin_ctzll(l);
      stays = j < s.have[p] && old[(size_t)p * a.W + j] == id;
    }
    for (unsigned long long l = s.childless & ((1ull << b) - 1); l && !stays; l &= l - 1) {       // listed once
      const int p = __builtin_ctzll(l);
      stays = j < s.have[p] && old[(size_t)p * a.W + j] == id;
    }
    if (!stays) gone |= 1ull << b;
  }
  return gone;
}

// A workgroup takes 256 columns of a request's tables.
__global__ __launch_bounds__(kReorderThreads) void kv_reorder_kernel(ReorderArgs a) {
  __shared__ ReorderBeams s;
  __shared__ int gone_n[kReorderThreads / 64];
  const int tid = threadIdx.x, lane = tid & 63, B = a.B;
  const int r = blockIdx.x / a.blocks, block = blockIdx.x - r * a.blocks;
  const int before = reorder_beams(a, r, s);
  const int32_t* old = a.table + (size_t)r * B * a.W;
  if (block == 0 && tid < B) {
    const int p = s.parent[tid];
    const size_t row = (size_t)r * B + tid;
    int src = -1, dst = -1;
    if (s.fresh[tid] >= 0) {
      const int last = s.len[p] >> a.page_log2;
      const long at = (long)before + s.fresh[tid];
      if (at < a.F && last < a.W) {
        src = old[(size_t)p * a.W + last];
        dst = a.free_pages[at];
      }
    }
    a.new_len[row] = p < 0 ? 0 : s.len[p];
    a.src[row] = src;
    a.dst[row] = dst;
  }
  if (r == a.R - 1 && block == 0 && tid == 0) a.used[0] = before + s.taken;
  const int j = block * kReorderThreads + tid;
  unsigned long long gone = 0;
  if (j < a.W) {
    for (int k = 0; k < B; ++k) {
      const int p = s.parent[k];
      int id = -1;
      if (p >= 0 && j < s.have[p]) {
        if (s.fresh[k] >= 0 && j == s.len[p] >> a.page_log2) {
          const long at = (long)before + s.fresh[k];
          if (at < a.F) id = a.free_pages[at];
        } else {
          id = old[(size_t)p * a.W + j];
        }
      }
      a.new_table[((size_t)r * B + k) * a.W + j] = id;
    }
    if (j >= (a.keep ? max(a.keep[r], 0) : 0)) gone = reorder_gone(a, s, old, j);
  }
  int n = __builtin_popcountll(gone);
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) n += __shfl_xor(n, d);
  if (lane == 0) gone_n[tid >> 6] = n;
  __syncthreads();
  if (tid == 0) {
    int t = 0;
#pragma unroll
    for (int i = 0; i < kReorderThreads / 64; ++i) t += gone_n[i];
    a.counts[blockIdx.x] = t;
  }
}

// The pages that no row holds any more, by request, column and row, and -1 behind them.
__global__ __launch_bounds__(kReorderThreads) void kv_release_kernel(ReorderArgs a) {
  __shared__ ReorderBeams s;
  __shared__ int sums[kReorderThreads / 64][2];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, nblk = a.R * a.blocks, me = (int)blockIdx.x;
  int before = 0, all = 0;
  for (int i = tid; i < nblk; i += kReorderThreads) {
    const int c = a.counts[i];
    all += c;
    if (i < me) before += c;
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) before += __shfl_xor(before, d), all += __shfl_xor(all, d);
  if (lane == 0) sums[wave][0] = before, sums[wave][1] = all;
  __syncthreads();
  before = all = 0;
#pragma unroll
  for (int i = 0; i < kReorderThreads / 64; ++i) before += sums[i][0], all += sums[i][1];
  if (me == 0 && tid == 0) a.n_released[0] = all;
  for (long i = (long)all + (long)me * kReorderThreads + tid; i < a.Q; i += (long)nblk * kReorderThreads) a.released[i] = -1;
  if (a.counts[me] == 0) return;
  __syncthreads();
  const int r = me / a.blocks, block = me - r * a.blocks, j = block * kReorderThreads + tid;
  reorder_beams(a, r, s);
  const int32_t* old = a.table + (size_t)r * a.B * a.W;
  unsigned long long gone = 0;
  if (j < a.W && j >= (a.keep ? max(a.keep[r], 0) : 0)) gone = reorder_gone(a, s, old, j);
  const int n = __builtin_popcountll(gone);
  int inc = n;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int up = __shfl_up(inc, d);
    if (lane >= d) inc += up;
  }
  if (lane == 63) s.wave[wave] = inc;
  __syncthreads();
  int at = before + inc - n;
  for (int i = 0; i < wave; ++i) at += s.wave[i];
  for (; gone; gone &= gone - 1, ++at)
    if (at < a.Q) a.released[at] = old[(size_t)__builtin_ctzll(gone) * a.W + j];
}

struct CopyArgs {
  uint8_t* cache;
  const int32_t* src;
  const int32_t* dst;
  long page_bytes;          // of all heads, a multiple of 16
  int n, pages;
};

constexpr int kCopyThreads = 256;
constexpr int kCopyBytes = 4 * kCopyThreads * 16;        // of a workgroup

// Whole pages, one (pair, 16 KiB) to a workgroup; pairs with a page outside the cache are none.
__global__ __launch_bounds__(kCopyThreads) void kv4_copy_kernel(CopyArgs a) {
  const int i = blockIdx.x;
  const int from = a.src[i], to = a.dst[i];
  if ((unsigned)from >= (unsigned)a.pages || (unsigned)to >= (unsigned)a.pages || from == to) return;
  const uint8_t* p = a.cache + (size_t)from * a.page_bytes;
  uint8_t* q = a.cache + (size_t)to * a.page_bytes;
  u32x4 x[4];
  const long at = (long)blockIdx.y * kCopyBytes + threadIdx.x * 16;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const long o = at + k * kCopyThreads * 16;
    if (o < a.page_bytes) x[k] = *reinterpret_cast<const u32x4*>(p + o);
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const long o = at + k * kCopyThreads * 16;
    if (o < a.page_bytes) *reinterpret_cast<u32x4*>(q + o) = x[k];
  }
}

}  // namespace
}  // namespace qg
