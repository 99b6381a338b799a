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
// order is that of the logits, so the first kernel needs no lse: it takes a piece of a row in one pass over it,
// carries maximum and sum as an online softmax does, and keeps the piece's K largest logits. The second kernel has the
// B * pieces * K of a request that are left and computes their values in 64 bits: what beams differ by decides
// between candidates, and at a score of -100 steps of 32 bits are 2^-17. (The exponentials of a sum are taken in 32 bits, so
// candidates of different beams may change places where they are closer than 1e-6; sums are off by up to 2e-7 of themselves.)
// Bound by the logits' bytes (48 x 8 beams over 128000 in fp32, K = 16: 39.3 us for the first kernel, 5.0 TB/s, and 7.0 for the
// second); with few rows by the chain load - bound - selection - second launch (4 beams over 32000: 5.9 and 4.8 us).

constexpr int kBeamThreads = 256;
constexpr int kBeamWaves = kBeamThreads / 64;
constexpr int kBeamMaxB = 64;          // beams of a request
constexpr int kBeamMaxK = 128;         // candidates that are taken
constexpr int kBeamElems = 16;         // logits of a lane and step
constexpr int kBeamStep = 64 * kBeamElems;
constexpr int kBeamPiece = kBeamWaves * kBeamStep;         // pieces of a row are multiples of it
constexpr int kBeamList = 640;         // logits that a wave holds before it selects
constexpr int kBeamMost = 1024;        // of a request that are left for the second kernel, where a row has several pieces
static_assert(kBeamList % 64 == 0 && kBeamList >= kBeamMaxK + 64, "a selection makes room for a round");

// A logit as an integer of the same order, above 0 but for NaN.
__device__ __forceinline__ uint32_t beam_bits(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x + 0.0f);         // -0 as 0
  return u ^ ((u >> 31) ? 0xffffffffu : 0x80000000u);
}
// A logit and its token as one number, larger logits first, then lower tokens. 0 stands for none.
__device__ __forceinline__ uint64_t beam_key(float x, uint32_t v) { return (uint64_t)beam_bits(x) << 32 | (0xffffffffu - v); }
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
  uint64_t* cand;           // [R * B][pieces][K] in order, 0 for none
  long stride;
  int R, B, V, K, pieces, piece;      // piece: logits of one, a multiple of kBeamPiece
  int end;
  int pieces_log2;          // of the power of two from `pieces` on, at most 6
  uint32_t per_inv;         // 2^32 / (pieces K), rounded up; 0 for pieces K = 1
};

// Whether a beam's logits are candidates: not those of an ended one, nor of one whose score leaves nothing.
__device__ __forceinline__ bool beam_reads(const BeamArgs& a, int row) {
  return a.scores[row] > -__builtin_inff() && !(a.finished && a.finished[row]);
}

__device__ __forceinline__ int lanes_below(unsigned long long mask) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}

// The largest number that K of the lanes' P numbers each reach, its bits from LOW on: a lower bound of the K-th largest
// of all that the lanes hold (0 if fewer than K hold any). A count of lanes for each bit; comparing every lane's with
// every other's takes eight times as long.
template <int LOW, int P>
__device__ __forceinline__ uint32_t wave_bound(const uint32_t (&mine)[P], int K) {
  uint32_t bound = 0;
#pragma unroll
  for (int bit = 31; bit >= LOW; --bit) {
    const uint32_t more = bound | 1u << bit;
    int n = 0;
#pragma unroll
    for (int p = 0; p < P; ++p) n += __builtin_popcountll(__ballot(mine[p] >= more));
    bound = n >= K ? more : bound;
  }
  return bound;
}

// A wave's list[0 .. n) without what is below a bound that K of it reach: the bound, n as it is then. A wave's LDS
// accesses run in order.
__device__ __forceinline__ uint32_t wave_tighten(uint64_t* list, int& n, int K, int lane) {
  asm volatile("" ::: "memory");
  uint32_t top[2] = {0, 0};
  for (int i = lane, h = 0; i < n; i += 64, h ^= 1) {
    const uint32_t k = (uint32_t)(list[i] >> 32);
    top[0] = max(top[0], h ? 0u : k);
    top[1] = max(top[1], h ? k : 0u);
  }
  const uint32_t bound = wave_bound<12>(top, K);
  int m = 0;
  for (int i = 0; i < n; i += 64) {
    const uint64_t k = i + lane < n ? list[i + lane] : 0;
    const bool in = k && (uint32_t)(k >> 32) >= bound;
    const unsigned long long all = __ballot(in);
    if (in) list[m + lanes_below(all)] = k;
    m += __builtin_popcountll(all);
  }
  n = m;
  asm volatile("" ::: "memory");
  return bound;
}

// The K largest of a wave's list[0 .. n), in order, to its front, by way of sorted[K]; how many there are.
__device__ __forceinline__ int wave_keep(uint64_t* list, uint64_t* sorted, int n, int K, int lane) {
  if (n > K && n > 64) wave_tighten(list, n, K, lane);
  asm volatile("" ::: "memory");
  for (int c = 0; c < n; c += 64) {
    const uint64_t mine = c + lane < n ? list[c + lane] : 0;
    int place = 0;
#pragma unroll 4
    for (int j = 0; j < n; ++j) place += list[j] > mine;
    if (mine && place < K) sorted[place] = mine;
  }
  asm volatile("" ::: "memory");
  for (int i = lane; i < min(n, K); i += 64) list[i] = sorted[i];
  asm volatile("" ::: "memory");
  return min(n, K);
}

typedef uint32_t u32x4_by4 __attribute__((ext_vector_type(4), aligned(4)));      // rows need no more than their elements' alignment
typedef uint32_t u32x4_by2 __attribute__((ext_vector_type(4), aligned(2)));

template <typename T>
struct BeamLoad {
  static constexpr int kWide = 16 / sizeof(T);      // logits of a load
  static constexpr int kLoads = kBeamElems / kWide;
  using vec = std::conditional_t<sizeof(T) == 4, u32x4_by4, u32x4_by2>;
  // the place in a step of a lane's logit i
  static __device__ __forceinline__ int place(int i, int lane) { return (i / kWide * 64 + lane) * kWide + i % kWide; }
  static __device__ __forceinline__ float one(const T* p) {
    if constexpr (sizeof(T) == 4) return *p;
    else return __builtin_bit_cast(float, (uint32_t)*p << 16);
  }
  // A lane's logits of the step at v0, -inf from `end` on.
  static __device__ __forceinline__ void step(const T* row, int v0, int end, int lane, float (&x)[kBeamElems]) {
    if (v0 + kBeamStep <= end) {
      u32x4 w[kLoads];
#pragma unroll
      for (int j = 0; j < kLoads; ++j)
        w[j] = __builtin_bit_cast(u32x4, *reinterpret_cast<const vec*>(row + v0 + place(j * kWide, lane)));
#pragma unroll
      for (int j = 0; j < kLoads; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t u = w[j][e];
          if constexpr (sizeof(T) == 4) {
            x[4 * j + e] = __builtin_bit_cast(float, u);
          } else {
            x[8 * j + 2 * e] = __builtin_bit_cast(float, u << 16);
            x[8 * j + 2 * e + 1] = __builtin_bit_cast(float, u & 0xffff0000u);
          }
        }
    } else {
#pragma unroll
      for (int i = 0; i < kBeamElems; ++i) {
        const int v = v0 + place(i, lane);
        x[i] = v < end ? one(row + v) : -__builtin_inff();
      }
    }
  }
};

// A workgroup takes a piece of a row, each of its waves every fourth step, with a list of its own: no barrier but at
// the end. A wave's first step gives a bound that K logits reach; from then on a logit is kept if it is above the bound,
// which the list raises whenever it has grown by K or 64. One that equals it is not kept: its token is behind those of
// the list. What a step costs beside its 16 exponentials is a round for each lane's logits above the bound: with the first
// step's bound to the end, K of 1024 logits pass in every step (48 x 8 rows of 128000, K = 16: 52.8 us, bf16 49.4).
template <typename T>
__global__ __launch_bounds__(kBeamThreads, 4) void beam_rows_kernel(BeamArgs a) {
  using L = BeamLoad<T>;
  __shared__ uint64_t lists[kBeamWaves][kBeamList], sorted[kBeamWaves][kBeamMaxK];
  __shared__ double wave_sum[kBeamWaves];
  __shared__ float wave_top[kBeamWaves];
  __shared__ int wave_count[kBeamWaves];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int row = blockIdx.x / a.pieces, piece = blockIdx.x - row * a.pieces;
  const T* x0 = static_cast<const T*>(a.x) + (size_t)row * a.stride;
  const int v_begin = piece * a.piece + wave * kBeamStep, v_end = min(a.V, (piece + 1) * a.piece);
  const int K = a.K;
  const float ninf = -__builtin_inff(), log2e = 1.4426950408889634f;
  uint64_t* list = lists[wave];
  float top = ninf;
  double sum = 0.0;
  float from = ninf;             // logits that are kept are above it
  int count = 0, limit = 2 * max(K, 32);
  float x[kBeamElems];
  if (v_begin < v_end) L::step(x0, v_begin, v_end, lane, x);
  if (!beam_reads(a, row)) return;                  // (asked while the loads are on their way; the second kernel asks the same)
  for (int v0 = v_begin; v0 < v_end; v0 += kBeamPiece) {
    float next[kBeamElems];
    if (v0 + kBeamPiece < v_end) L::step(x0, v0 + kBeamPiece, v_end, lane, next);
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
    auto token = [&](int i) { return (uint32_t)(v0 + L::place(i, lane)); };
    uint32_t pending = 0;
    if (v0 == v_begin) {
      float half[2] = {x[0], x[1]};
#pragma unroll
      for (int i = 2; i < kBeamElems; ++i) half[i & 1] = fmaxf(half[i & 1], x[i]);
      const uint32_t two[2] = {half[0] > ninf ? beam_bits(half[0]) : 0u, half[1] > ninf ? beam_bits(half[1]) : 0u};
      const uint32_t one[1] = {max(two[0], two[1])};
      const uint32_t bound = K <= 32 ? wave_bound<12>(one, K) : wave_bound<12>(two, K);
      if (bound) from = beam_logit((uint64_t)bound << 32);
#pragma unroll
      for (int i = 0; i < kBeamElems; ++i) pending |= x[i] > ninf && x[i] >= from ? 1u << i : 0u;
    } else if (__any(most > from)) {
#pragma unroll
      for (int i = 0; i < kBeamElems; ++i) pending |= x[i] > from ? 1u << i : 0u;
    }
    // one logit of each lane to a round
    for (unsigned long long in; (in = __ballot(pending != 0)) != 0;) {
      if (count + 64 > kBeamList) {
        count = wave_keep(list, sorted[wave], count, K, lane);
        const uint64_t last = list[K - 1];
        const uint32_t behind = (uint32_t)beam_token(last);
        from = beam_logit(last);
        uint32_t above = 0;
#pragma unroll
        for (int i = 0; i < kBeamElems; ++i) above |= x[i] > from || (x[i] == from && token(i) < behind) ? 1u << i : 0u;
        pending &= above;
        continue;
      }
      const int i = pending ? __builtin_ctz(pending) : 0;
      // (values, as a choice between two places would put the array into memory)
      auto pick = [](bool second, float p, float q) { return second ? q : p; };
      float v[kBeamElems / 2];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = pick(i & 8, x[j], x[8 + j]);
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = pick(i & 4, v[j], v[4 + j]);
#pragma unroll
      for (int j = 0; j < 2; ++j) v[j] = pick(i & 2, v[j], v[2 + j]);
      const float mine = pick(i & 1, v[0], v[1]);
      if (pending) list[count + lanes_below(in)] = beam_key(mine, token(i));
      count += __builtin_popcountll(in);
      pending &= pending - 1;
    }
    if (count >= limit) {
      from = beam_logit((uint64_t)wave_tighten(list, count, K, lane) << 32);       // (more than K: there is a bound)
      limit = count + max(K, 64);
    }
#pragma unroll
    for (int i = 0; i < kBeamElems; ++i) x[i] = next[i];
  }
  count = wave_keep(list, sorted[wave], count, K, lane);
  for (int i = count + lane; i < K; i += 64) list[i] = 0;
  // the lanes' and the waves' maxima and sums as one
  float all = top;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) all = fmaxf(all, __shfl_xor(all, d));
  sum = top == ninf ? sum : sum * exp((double)top - (double)all);
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d);
  if (lane == 0) wave_top[wave] = all, wave_sum[wave] = sum, wave_count[wave] = count;
  __syncthreads();
  if (tid < kBeamWaves) {
    const float mine = wave_top[tid];
#pragma unroll
    for (int i = 0; i < kBeamWaves; ++i) all = fmaxf(all, wave_top[i]);
    double t = mine == ninf ? wave_sum[tid] : wave_sum[tid] * exp((double)mine - (double)all);
#pragma unroll
    for (int d = 1; d < kBeamWaves; d <<= 1) t += __shfl_xor(t, d);
    if (tid == 0) a.stat[blockIdx.x] = {t, all, 0.0f};
  }
  // and their lists: a logit's place is its own in its list, and how many of each other list are above it
  uint64_t* out = a.cand + (size_t)blockIdx.x * K;
  for (int e = tid; e < kBeamWaves * K; e += kBeamThreads) {
    const int w = e / K, i = e - w * K;
    const uint64_t k = lists[w][i];
    if (!k) continue;
    int place = i, at[kBeamWaves - 1] = {};
    for (int half = 1 << (31 - __builtin_clz(K)); half; half >>= 1)       // at: entries that are above k, of the first so many
#pragma unroll
      for (int o = 1; o < kBeamWaves; ++o) {
        const int to = at[o - 1] + half;
        if (to <= K && lists[(w + o) % kBeamWaves][to - 1] > k) at[o - 1] = to;
      }
#pragma unroll
    for (int o = 1; o < kBeamWaves; ++o) place += at[o - 1];
    if (place < K) out[place] = k;
  }
  int total = 0;
#pragma unroll
  for (int w = 0; w < kBeamWaves; ++w) total += wave_count[w];
  for (int i = total + tid; i < K; i += kBeamThreads) out[i] = 0;
}

// One workgroup to a request. Candidate e = (beam, piece, place in the piece's list). Equal values go to the lower beam, and of
// a beam to the larger logit, then the lower token, as e has it: a large score makes the values of different logits equal, and
// then their order must not follow the pieces. So a beam's candidates come in the order of their keys whatever their values
// round to, and the K of largest key, which its pieces' lists hold, are all that can be chosen.
// MOST: candidates at most.
template <int MOST>
__global__ __launch_bounds__(kBeamThreads) void beam_join_kernel(BeamArgs a) {
  __shared__ uint64_t kept_value[MOST];   // (all of them where all are worth the same)
  __shared__ uint64_t kept_next[MOST];    // what their order goes by next, lower ones first: beam, logit turned round, e
  constexpr int kHeld = 4;                // of a thread's candidates, in registers
  __shared__ double off[kBeamMaxB];       // score - lse
  __shared__ float score[kBeamMaxB];
  __shared__ int reads[kBeamMaxB];
  __shared__ uint32_t each[kBeamThreads];
  __shared__ int kept_n;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = blockIdx.x, K = a.K;
  const int per = a.pieces * K, n = a.B * per;
  const uint64_t* cand = a.cand + (size_t)r * n;
  const float ninf = -__builtin_inff();
  uint64_t held[kHeld];
#pragma unroll
  for (int i = 0; i < kHeld; ++i) held[i] = tid + i * kBeamThreads < n ? cand[tid + i * kBeamThreads] : 0;
  if (tid == 0) kept_n = 0;
  {
    // a row's pieces in neighbouring lanes, as many rows to a wave as fit
    const int lg = a.pieces_log2, sub = lane & ((1 << lg) - 1);
    for (int b = (wave * 64 + lane) >> lg; (b & -(64 >> lg)) < a.B; b += kBeamThreads >> lg) {
      const bool in = b < a.B;
      const int row = r * a.B + (in ? b : 0);
      const BeamStat first = a.stat[(size_t)row * a.pieces + min(sub, a.pieces - 1)];       // (not written for a beam that is not read)
      const bool take = in && beam_reads(a, row);
      const bool some = take && sub < a.pieces;
      double sum = some ? first.sum : 0.0;
      float top = some ? first.top : ninf;
      for (int p = sub + 64; take && p < a.pieces; p += 64) {         // (then a row takes a wave)
        const BeamStat st = a.stat[(size_t)row * a.pieces + p];
        const float to = fmaxf(top, st.top);
        sum = (top == ninf ? sum : sum * exp((double)top - (double)to)) + (st.top == ninf ? st.sum : st.sum * exp((double)st.top - (double)to));
        top = to;
      }
      float all = top;
      for (int d = 1; d < 1 << lg; d <<= 1) all = fmaxf(all, __shfl_xor(all, d));
      sum = top == ninf ? sum : sum * exp((double)top - (double)all);
      for (int d = 1; d < 1 << lg; d <<= 1) sum += __shfl_xor(sum, d);
      if (in && sub == 0) {
        const float s = a.scores[row];
        score[b] = s;
        reads[b] = take;
        off[b] = (double)all + log(sum);      // NaN where a logit is NaN or +inf: its beam has no candidates
      }
    }
  }
  __syncthreads();
  // a candidate's value as an ordered integer, 0 for none
  auto beam_of = [&](int e) { return a.per_inv ? (int)__umulhi((uint32_t)e, a.per_inv) : e; };      // e / per, of e < 2^14
  auto value = [&](int e, uint64_t k) -> uint64_t {
    const int b = beam_of(e);
    if (!reads[b]) {
      const bool one = e == b * per && score[b] > ninf;   // an ended beam's only candidate
      return one ? beam_order((double)score[b]) : 0;
    }
    if (!k) return 0;
    const double v = (double)score[b] + ((double)beam_logit(k) - off[b]);
    return v > (double)ninf ? beam_order(v) : 0;
  };
  auto for_each = [&](auto&& f) {
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      const int e = tid + i * kBeamThreads;
      if (e < n) f(e, value(e, held[i]), held[i]);
    }
    for (int e = tid + kHeld * kBeamThreads; e < n; e += kBeamThreads) f(e, value(e, cand[e]), cand[e]);
  };
  uint32_t top = 0;
  for_each([&](int, uint64_t v, uint64_t) { top = max(top, (uint32_t)(v >> 32)); });
  // a bound that K candidates reach, from the threads' largest: with a candidate or two to a thread about K are left
  uint64_t from = 0;
  if (n > K) {
    each[tid] = top;
    __syncthreads();
    const uint32_t mine[4] = {each[lane], each[64 + lane], each[128 + lane], each[192 + lane]};
    from = (uint64_t)wave_bound<8>(mine, K) << 32;
  }
  for_each([&](int e, uint64_t v, uint64_t k) {
    if (v && v >= from) {
      const int i = atomicAdd(&kept_n, 1);          // a set: its order does not matter
      kept_value[i] = v;
      kept_next[i] = (uint64_t)beam_of(e) << 48 | (uint64_t)~(uint32_t)(k >> 32) << 16 | (uint32_t)e;
    }
  });
  __syncthreads();
  const int m = kept_n;
  float* os = a.out_scores + (size_t)r * K;
  int32_t* ob = a.out_beams + (size_t)r * K;
  int32_t* ot = a.out_tokens + (size_t)r * K;
  for (int i = tid; i < m; i += kBeamThreads) {
    const uint64_t v = kept_value[i];
    const uint64_t next = kept_next[i];
    const int e = (int)(next & 0xffff), b = beam_of(e);
    const uint64_t k = cand[e];
    int p = 0;
#pragma unroll 4
    for (int j = 0; j < m; ++j) p += kept_value[j] > v || (kept_value[j] == v && kept_next[j] < next);
    if (p >= K) continue;
    os[p] = (float)__builtin_bit_cast(double, v ^ ((v >> 63) ? 1ull << 63 : ~0ull));
    ob[p] = b;
    ot[p] = reads[b] ? beam_token(k) : a.end;
  }
  for (int p = m + tid; p < K; p += kBeamThreads) os[p] = ninf, ob[p] = -1, ot[p] = a.end;
}

// ---------------------------------------------------------------------------
// tables and pages after a selection
// ---------------------------------------------------------------------------
//
// A workgroup takes blocks of 256 columns of a request's tables, one unless there are very many. Every one counts for itself the
// pages that the requests before take from the free list (a thread to a row: a few loads), so that nothing waits for
// another. Pages that no row holds any more are left in the caller's workspace, and a second kernel, which knows how many
// the blocks before have left, moves them to their places in the list.
// Bound by chains of loads: lengths and parents, old entries, then the counts of the first kernel (4 x 4 beams of up to 3100 tokens
// 6.1 and 2.2 us; 64 x 8 of up to 6200 tokens, pages of 32, 9.2 and 2.7 us, 0.8 MB in all).

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
  int32_t* counts;            // [R * blocks] pages that a block's columns release
  int32_t* gone;              // [R * blocks][256 B] the pages
  int R, B, W, F, Q, page_log2, blocks;
  int each, parts;            // blocks of a workgroup; workgroups of a request
  int release_each, release;  // blocks of a workgroup of the second kernel; its workgroups
};

struct ReorderBeams {
  int len[kBeamMaxB], have[kBeamMaxB];                   // old rows: tokens, and pages (within the table)
  int parent[kBeamMaxB], fresh[kBeamMaxB];               // new rows: old row or -1; place in the request's free pages or -1
  int4 row[kBeamMaxB];                                   // new rows: old row or 0; the column of a fresh page or -1, and the page;
                                                         // whether there is an old row
  unsigned long long live, childless;                    // old rows that have children; that have pages and none
  int taken;                                             // new rows with a fresh page
  int wave[kReorderThreads / 64];
};

// The request's beams; returns how many pages the requests before it take from the free list.
__device__ __forceinline__ int reorder_beams(const ReorderArgs& a, int r, ReorderBeams& s) {
  const int tid = threadIdx.x, lane = tid & 63, B = a.B, mask = (1 << a.page_log2) - 1;
  // a request to a thread: the rows that are not their parent's first child, of parents with a last page filled in part
  int mine = 0;
  for (int q = tid; q < r; q += kReorderThreads) {
    const int32_t *len = a.kv_len + (size_t)q * B, *of = a.parents + (size_t)q * B;
    unsigned long long part = 0, seen = 0;
    int n[8], p[8];
    auto load = [&](int b0) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        n[i] = len[min(b0 + i, B - 1)];
        p[i] = of[min(b0 + i, B - 1)];
      }
    };
    auto parts = [&](int b0) {
#pragma unroll
      for (int i = 0; i < 8; ++i) part |= (unsigned long long)((max(n[i], 0) & mask) != 0) << min(b0 + i, B - 1);
    };
    auto count = [&](int b0) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const unsigned long long bit = b0 + i < B && (unsigned)p[i] < (unsigned)B ? 1ull << p[i] : 0ull;
        mine += (seen & part & bit) != 0;
        seen |= bit;
      }
    };
    for (int b0 = 8; b0 < B; b0 += 8) {          // (a parent may stand behind)
      load(b0);
      parts(b0);
    }
    load(0);
    parts(0);
    count(0);
    for (int b0 = 8; b0 < B; b0 += 8) {
      load(b0);
      count(b0);
    }
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) mine += __shfl_xor(mine, d);
  if (lane == 0) s.wave[tid >> 6] = mine;
  if (tid < 64) {            // B <= 64: a lane of the first wave to a beam
    const bool in = tid < B;
    const int n = in ? max(a.kv_len[(size_t)r * B + tid], 0) : 0;
    const int have = (int)min(((long)n + mask) >> a.page_log2, (long)a.W);
    const int of = in ? a.parents[(size_t)r * B + tid] : -1;
    const int p = (unsigned)of < (unsigned)B ? of : -1;
    // the first row of the same parent, and that parent's length, from the other lanes
    bool again = false;
    for (int i = 0; i < B; ++i) {
      const int other = __shfl(p, i);
      again |= i < tid && other == p;
    }
    const int of_parent = __shfl(n, max(p, 0));
    const bool part = (of_parent & mask) != 0;
    const unsigned long long fresh = __ballot(in && p >= 0 && again && part);
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

// SEVERAL: whether workgroups take several blocks (the loop that then goes over them costs 0.5 us, with one block too).
template <bool SEVERAL>
__global__ __launch_bounds__(kReorderThreads) void kv_reorder_kernel(ReorderArgs a) {
  extern __shared__ int32_t old_lds[];         // [B][256] the columns' old entries, each thread its own; -1 behind a row's pages
  __shared__ ReorderBeams s;
  __shared__ int gone_n[kReorderThreads / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, B = a.B;
  const int parts = SEVERAL ? a.parts : a.blocks;
  const int r = blockIdx.x / parts, part = blockIdx.x - r * parts;
  int block = SEVERAL ? part * a.each : part;
  const int block_end = SEVERAL ? min(a.blocks, block + a.each) : block + 1;
  const int32_t* old = a.table + (size_t)r * B * a.W;
  int j = block * kReorderThreads + tid;
  // the first eight rows' entries are on their way while the request's beams are looked up
  int32_t x[8];
  auto load = [&](int b0) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = b0 + i < B && j < a.W ? old[(size_t)(b0 + i) * a.W + j] : -1;
  };
  load(0);
  const int first = a.keep ? max(a.keep[r], 0) : 0;
  const int before = reorder_beams(a, r, s);
  if (tid < B) {
    const int p = s.parent[tid], fresh = s.fresh[tid], last = p < 0 ? 0 : s.len[p] >> a.page_log2;
    const bool can = fresh >= 0 && last < a.W && (long)before + fresh < a.F;
    const int page = can ? a.free_pages[(size_t)before + fresh] : -1;
    s.row[tid] = make_int4(max(p, 0), fresh >= 0 ? last : -1, page, p >= 0);
    if (part == 0) {
      const size_t row = (size_t)r * B + tid;
      a.new_len[row] = p < 0 ? 0 : s.len[p];
      a.src[row] = can ? old[(size_t)p * a.W + last] : -1;
      a.dst[row] = page;
    }
  }
  if (r == a.R - 1 && part == 0 && tid == 0) a.used[0] = before + s.taken;
  __syncthreads();
  auto entry = [&](int b) -> int32_t& { return old_lds[b * kReorderThreads + tid]; };
  for (;;) {
    for (int b0 = 0; b0 < B; b0 += 8) {
      if (b0) load(b0);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (b0 + i < B) entry(b0 + i) = j < s.have[b0 + i] ? x[i] : -1;
    }
    unsigned long long gone = 0;
    if (j < a.W) {
      int32_t* out = a.new_table + (size_t)r * B * a.W + j;
#pragma unroll 4
      for (int k = 0; k < B; ++k, out += a.W) {
        const int4 row = s.row[k];
        *out = !row.w ? -1 : j == row.y ? row.z : entry(row.x);
      }
      // Of the column's old entries, those that no new row holds any more. A page stands in the same column of all rows that
      // share it, and a row's children hold all of its pages, so only rows without children can lose one.
      if (j >= first)
        for (unsigned long long m = s.childless; m; m &= m - 1) {
          const int b = __builtin_ctzll(m), id = entry(b);
          const unsigned long long others = s.live | (s.childless & ((1ull << b) - 1));      // (the lower ones list a page that they share)
          bool stays = id < 0;
#pragma unroll 8
          for (int p = 0; p < B; ++p) stays |= entry(p) == id && (others >> p & 1);
          if (!stays) gone |= 1ull << b;
        }
    }
    // the pages, by column and row
    const int n = __builtin_popcountll(gone);
    int inc = n;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int up = __shfl_up(inc, d);
      if (lane >= d) inc += up;
    }
    if (lane == 63) gone_n[wave] = inc;
    __syncthreads();
    int at = inc - n, all = 0;
#pragma unroll
    for (int i = 0; i < kReorderThreads / 64; ++i) {
      at += i < wave ? gone_n[i] : 0;
      all += gone_n[i];
    }
    const size_t at_block = SEVERAL ? (size_t)r * a.blocks + block : blockIdx.x;
    if (tid == 0) a.counts[at_block] = all;
    for (int32_t* out = a.gone + at_block * kReorderThreads * B; gone; gone &= gone - 1) out[at++] = entry(__builtin_ctzll(gone));
    if (!SEVERAL || ++block >= block_end) return;
    j = block * kReorderThreads + tid;
    load(0);
    __syncthreads();            // gone_n has been read
  }
}

// The released pages to their places, -1 behind the last.
template <bool SEVERAL>
__global__ __launch_bounds__(kReorderThreads) void kv_release_kernel(ReorderArgs a) {
  __shared__ int sums[kReorderThreads / 64][2];
  const int tid = threadIdx.x, lane = tid & 63, nblk = a.R * a.blocks;
  const int begin = (int)blockIdx.x * (SEVERAL ? a.release_each : 1), end = min(nblk, begin + a.release_each);
  int mine = a.counts[begin];
  int before = 0, all = 0;
  for (int i = tid; i < nblk; i += kReorderThreads) {
    const int c = a.counts[i];
    all += c;
    if (i < begin) before += c;
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) before += __shfl_xor(before, d), all += __shfl_xor(all, d);
  if (lane == 0) sums[tid >> 6][0] = before, sums[tid >> 6][1] = all;
  __syncthreads();
  before = all = 0;
#pragma unroll
  for (int i = 0; i < kReorderThreads / 64; ++i) before += sums[i][0], all += sums[i][1];
  if (begin == 0 && tid == 0) a.n_released[0] = all;
  const long step = (long)(SEVERAL ? a.release : nblk) * kReorderThreads;
  for (long i = (long)all + (long)blockIdx.x * kReorderThreads + tid; i < a.Q; i += step) a.released[i] = -1;
  for (int block = begin;;) {
    const int32_t* from = a.gone + (size_t)block * kReorderThreads * a.B;
    for (int i = tid; i < mine && before + i < a.Q; i += kReorderThreads) a.released[before + i] = from[i];
    if (!SEVERAL || ++block >= end) return;
    before += mine;
    mine = a.counts[block];
  }
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

// Whole pages, one (pair, 16 KiB) to a workgroup; pairs with a page outside the cache are none. Bound by the launch (few pairs 3.0
// us), then by HBM (up to 448 pairs of 34.8 KB 6.3 us).
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
