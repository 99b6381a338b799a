// Low-rank adapters of many requests beside a shared projection: y[m] += gain[a] B_a (A_a x[m]), a the adapter of row m's
// request. Two launches: mid = gain A x in fp32 to a workspace, then y += B mid.
//
// Rows come in the order of the batch. A workgroup takes a tile of them, lists the adapters that occur in it and goes
// through the list: the products of all rows of the tile with one adapter are one MFMA operand's columns, and each row
// keeps its own adapter's. A prompt's tile has one or two adapters; a decode step's has one a row, whose weights have to
// be read once anyway, and the matrix cores that compute 16 columns for one have nothing else to do.
// A row is chosen, never multiplied by zero: an infinity or NaN of one adapter or request reaches no other.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "qgemm_kernels.hpp"

namespace qg {
namespace {

constexpr int kAdThreads = 256;
constexpr int kAdWaves = kAdThreads / 64;
constexpr int kAdMaxRank = 128;

struct AdapterArgs {
  const uint16_t* x;       // bf16 [M][K] at xs
  const uint16_t* a;       // bf16 [n][r][K]
  const uint16_t* b;       // bf16 [n][N][r]
  const int32_t* ids;      // [R]
  const int32_t* cu;       // [R + 1] or null: one row to a request
  const float* gain;       // [n] or null
  float* y;                // [M][N] at ys
  int32_t* row_id;         // [M] adapters of the rows, -1 for none
  float* mid;              // [splits][M][r]
  long xs, ys;
  int M, N, K, r, n, R;
  int splits, k_split;     // parts of K, and their length (a multiple of 32 kAdWaves)
  int lists;               // workgroups that share a tile's adapters
  int vec;                 // y's rows and columns go 16 bytes at a time
};

// The adapter of row m: the last request that begins at or before it, if it has a row there.
__device__ __forceinline__ int adapter_of(const AdapterArgs& a, int m) {
  if (m >= a.M) return -1;
  int r = m;
  if (a.cu) {
    int lo = 0, hi = a.R;                  // the first entry of cu[1 ..] above m
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (a.cu[mid + 1] > m) hi = mid;
      else lo = mid + 1;
    }
    r = lo;
    if (r >= a.R || a.cu[r] > m) return -1;
  }
  const int id = a.ids[r];
  return (unsigned)id < (unsigned)a.n ? id : -1;
}

template <int ROWS>
struct AdapterTile {
  int id[ROWS];            // of the tile's rows
  int list[ROWS];          // distinct ones, by their first rows
  int n;
};

// Lists the distinct adapters of a tile's rows (ROWS <= 64: a lane of the first wave to a row).
template <int ROWS>
__device__ __forceinline__ void adapter_list(AdapterTile<ROWS>& s, int id) {
  const int lane = threadIdx.x;
  if (lane < 64) {
    if (lane < ROWS) s.id[lane] = id;
    bool first = lane < ROWS && id >= 0;
    for (int i = 0; i < ROWS; ++i) {
      const int other = __shfl(id, i);
      first = first && !(i < lane && other == id);
    }
    const unsigned long long firsts = __ballot(first);
    if (first) s.list[__builtin_popcountll(firsts & ((1ull << lane) - 1))] = id;
    if (lane == 0) s.n = __builtin_popcountll(firsts);
  }
  __syncthreads();
}

// mid[m][j] = gain sum_k a[id][j][k] x[m][k] over one part of K, whose runs of 32 the four waves take in turn.
// MT: 16-row tiles of x; JT: 16-row tiles of A.
template <int MT, int JT>
__global__ __launch_bounds__(kAdThreads) void adapter_down_kernel(AdapterArgs a) {
  constexpr int ROWS = 16 * MT;
  __shared__ AdapterTile<ROWS> s;
  __shared__ f32x4 red[kAdWaves][JT * MT][64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 15, g = lane >> 4;
  const int jb = (a.r + 16 * JT - 1) / (16 * JT);
  int w = blockIdx.x;
  const int j0 = w % jb * 16 * JT;
  w /= jb;
  const int split = w % a.splits;
  w /= a.splits;
  const int lane_of_list = w % a.lists;
  const int m0 = w / a.lists * ROWS;
  const int own = tid < ROWS ? adapter_of(a, m0 + tid) : -1;
  if (tid < ROWS && m0 + tid < a.M && split == 0 && lane_of_list == 0 && j0 == 0) a.row_id[m0 + tid] = own;
  adapter_list(s, own);
  const int k_begin = split * a.k_split, k_end = min(a.K, k_begin + a.k_split);
  const uint16_t* xp[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) xp[t] = a.x + (size_t)min(m0 + 16 * t + col, a.M - 1) * a.xs + 8 * g;
  for (int d = lane_of_list; d < s.n; d += a.lists) {
    const int id = s.list[d];
    const uint16_t* ap[JT];
#pragma unroll
    for (int t = 0; t < JT; ++t)       // rows past the rank give products that nobody keeps
      ap[t] = a.a + ((size_t)id * a.r + min(j0 + 16 * t + col, a.r - 1)) * a.K + 8 * g;
    f32x4 acc[JT][MT];
#pragma unroll
    for (int j = 0; j < JT; ++j)
#pragma unroll
      for (int t = 0; t < MT; ++t) acc[j][t] = f32x4{};
    for (int k = k_begin + 32 * wave; k < k_end; k += 32 * kAdWaves) {
      const bool in = k + 8 * g < k_end;              // (K is a multiple of 8)
      bf16x8 xf[MT], af[JT];
#pragma unroll
      for (int t = 0; t < MT; ++t)
        xf[t] = in ? __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(xp[t] + k)) : bf16x8{};
#pragma unroll
      for (int j = 0; j < JT; ++j)
        af[j] = in ? __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(ap[j] + k)) : bf16x8{};
#pragma unroll
      for (int j = 0; j < JT; ++j)
#pragma unroll
        for (int t = 0; t < MT; ++t) acc[j][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(af[j], xf[t], acc[j][t], 0, 0, 0);
    }
#pragma unroll
    for (int j = 0; j < JT; ++j)
#pragma unroll
      for (int t = 0; t < MT; ++t) red[wave][j * MT + t][lane] = acc[j][t];
    __syncthreads();
    const float gain = a.gain ? a.gain[id] : 1.0f;
    for (int p = wave; p < JT * MT; p += kAdWaves) {      // the waves' sums, in their order
      f32x4 sum = red[0][p][lane];
#pragma unroll
      for (int i = 1; i < kAdWaves; ++i) sum += red[i][p][lane];
      const int t = p % MT, j = j0 + 16 * (p / MT) + 4 * g, row = 16 * t + col;
      // (r is a multiple of 8, and 4 g of 4: a lane's four are all in the rank or none)
      if (j < a.r && s.id[row] == id)
        *reinterpret_cast<f32x4*>(a.mid + ((size_t)split * a.M + m0 + row) * a.r + j) = sum * gain;
    }
    __syncthreads();
  }
}

// x = p[0] + p[1] + p[2] with eight bits of its significand in each, cut and not rounded, so that all 24 are there and
// no finite number becomes infinite: as three bf16 numbers mid enters the product whole, and fp32 y sees no bf16 step.
__device__ __forceinline__ void split_bf16(float x, uint32_t (&p)[3]) {
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    const uint32_t u = __builtin_bit_cast(uint32_t, x) & 0xffff0000u;
    p[i] = u >> 16;
    x = (u & 0x7f800000u) == 0x7f800000u ? 0.0f : x - __builtin_bit_cast(float, u);       // (infinity less itself is no 0)
  }
}

// y[m][c] += sum_j b[id][c][j] mid[m][j]. A wave takes 16 MT rows and 16 NT columns. S: runs of 32 of the rank.
template <int MT, int NT, int S>
__global__ __launch_bounds__(kAdThreads) void adapter_up_kernel(AdapterArgs a) {
  constexpr int ROWS = 16 * MT;
  __shared__ AdapterTile<ROWS> s;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 15, g = lane >> 4;
  const int nb = (a.N + 16 * NT * kAdWaves - 1) / (16 * NT * kAdWaves);
  const int m0 = (int)blockIdx.x / nb * ROWS;
  const int n0 = ((int)blockIdx.x % nb * kAdWaves + wave) * 16 * NT;
  adapter_list(s, tid < ROWS && m0 + tid < a.M ? a.row_id[m0 + tid] : -1);
  if (s.n == 0) return;
  int mine[MT];
  bf16x8 mid[MT][S][3];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    const int m = m0 + 16 * t + col;
    mine[t] = s.id[16 * t + col];
#pragma unroll
    for (int k = 0; k < S; ++k) {
      const int j = 32 * k + 8 * g;
      float v[8] = {};
      if (mine[t] >= 0 && j < a.r) {
        for (int p = 0; p < a.splits; ++p) {
          const float* mp = a.mid + ((size_t)p * a.M + m) * a.r + j;
          const f32x4 v0 = *reinterpret_cast<const f32x4*>(mp), v1 = *reinterpret_cast<const f32x4*>(mp + 4);
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] += v0[e], v[4 + e] += v1[e];
        }
      }
      u32x4 w[3];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        uint32_t p0[3], p1[3];
        split_bf16(v[2 * e], p0);
        split_bf16(v[2 * e + 1], p1);
#pragma unroll
        for (int i = 0; i < 3; ++i) w[i][e] = p0[i] | p1[i] << 16;
      }
#pragma unroll
      for (int i = 0; i < 3; ++i) mid[t][k][i] = __builtin_bit_cast(bf16x8, w[i]);
    }
  }
  if (n0 >= a.N) return;
  f32x4 out[MT][NT];
#pragma unroll
  for (int t = 0; t < MT; ++t)
#pragma unroll
    for (int c = 0; c < NT; ++c) out[t][c] = f32x4{};
  for (int d = 0; d < s.n; ++d) {
    const int id = s.list[d];
#pragma unroll
    for (int c = 0; c < NT; ++c) {
      const uint16_t* bp = a.b + ((size_t)id * a.N + min(n0 + 16 * c + col, a.N - 1)) * a.r + 8 * g;
      bf16x8 bf[S];
#pragma unroll
      for (int k = 0; k < S; ++k)
        bf[k] = 32 * k + 8 * g < a.r ? __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(bp + 32 * k)) : bf16x8{};
#pragma unroll
      for (int t = 0; t < MT; ++t) {
        f32x4 acc = f32x4{};
#pragma unroll
        for (int i = 2; i >= 0; --i)       // the smallest first
#pragma unroll
          for (int k = 0; k < S; ++k) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bf[k], mid[t][k][i], acc, 0, 0, 0);
#pragma unroll
        for (int e = 0; e < 4; ++e) out[t][c][e] = mine[t] == id ? acc[e] : out[t][c][e];
      }
    }
  }
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    if (mine[t] < 0) continue;
    float* yp = a.y + (size_t)(m0 + 16 * t + col) * a.ys;
#pragma unroll
    for (int c = 0; c < NT; ++c) {
      const int n = n0 + 16 * c + 4 * g;
      if (a.vec && n + 3 < a.N) {
        f32x4* q = reinterpret_cast<f32x4*>(yp + n);
        *q = *q + out[t][c];
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (n + e < a.N) yp[n + e] += out[t][c][e];
      }
    }
  }
}

}  // namespace
}  // namespace qg
