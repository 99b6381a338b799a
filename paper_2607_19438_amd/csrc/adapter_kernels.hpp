// Low-rank adapters of many requests beside a shared projection: y[m] += gain[a] B_a (A_a x[m]), a the adapter of row m's
// request. Two launches: mid = gain A x in fp32 to a workspace, then y += B mid.
//
// Rows come in the order of the batch. A workgroup takes a tile of them, lists the adapters that occur in it and goes
// through the list: the products of all rows of the tile with one adapter are one MFMA operand's columns, and each row
// keeps its own adapter's. A prompt's tile has one or two adapters; a decode step's has one a row, whose weights have to
// be read once anyway, and the matrix cores that compute 16 columns for one have nothing else to do.
// Bounds: of many rows HBM, which y passes twice (8500 rows of 8192 columns, rank 64, K = 2048: 160 us; each kernel again and
// again by itself 25.5 us, with x in the caches, and 130, 4.3 TB/s; reading and writing y alone by the same tiles 101); of
// a decode step the two launches and their chains of loads (16 rows of 2048 columns 8.1 us), then the adapters' weights (96
// rows with 64 adapters of 8192 columns, 38 MB, 16.2 us).
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
constexpr int kAdRun = 128;         // of K: what a wave loads at once, 256 bytes of each row

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
  int chunks;              // of the columns of a workgroup
};

// The adapter of row m, -1 for none: that of the last request that begins at or before the row. All lanes of a wave take
// part: each loads an edge of 64 parts of the requests, so that up to 64 of them take one load, and a part's search the rest.
__device__ __forceinline__ int adapter_of(const AdapterArgs& a, int m) {
  int id = -1;
  if (!a.cu) {
    if (m < a.M) id = a.ids[m];
  } else {
    const int lane = threadIdx.x & 63, step = (a.R + 63) / 64;
    const int edge = a.cu[min((lane + 1) * step, a.R)], start = a.cu[0];
    const int ids = a.ids[min(lane, a.R - 1)];
    int b = 0;                             // parts that end at or before m
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) b += __shfl(edge, b + d - 1) <= m ? d : 0;
    b += __shfl(edge, b) <= m ? 1 : 0;
    int r = b * step;
    id = __shfl(ids, min(r, 63));
    if (step > 1) {
      for (int hi = min(r + step, a.R); r < hi;) {       // its first request that ends behind m
        const int mid = (r + hi) >> 1;
        if (a.cu[mid + 1] > m) hi = mid;
        else r = mid + 1;
      }
      if (r < a.R) id = a.ids[r];
    }
    if (m < start || m >= a.M || r >= a.R) id = -1;
  }
  return (unsigned)id < (unsigned)a.n ? id : -1;
}

typedef float f32x4_by4 __attribute__((ext_vector_type(4), aligned(4)));       // y's rows need no more than their elements' alignment

// The distinct adapters of a tile's rows, a lane's row each (id -1: none), in the order of their first rows: next() gives one
// after the other, the same in all lanes.
struct AdapterList {
  int id;
  unsigned long long left;
  __device__ __forceinline__ explicit AdapterList(int of) : id(of), left(__ballot(of >= 0)) {}
  __device__ __forceinline__ int next() {
    const int i = __builtin_amdgcn_readlane(id, __builtin_ctzll(left));
    left &= ~__ballot(id == i);
    return i;
  }
};

// mid[m][j] = gain sum_k a[id][j][k] x[m][k] over one part of K, whose runs of 32 the WAVES waves take in turn, four runs'
// loads at once. MT: 16-row tiles of x; JT: 16-row tiles of A.
template <int MT, int JT, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void adapter_down_kernel(AdapterArgs a) {
  constexpr int ROWS = 16 * MT, DEEP = kAdRun / 32;
  __shared__ f32x4 red[WAVES][JT * MT][64];
  const int tid = threadIdx.x, lane = tid & 63, col = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int jb = (a.r + 16 * JT - 1) / (16 * JT);
  int w = blockIdx.x;
  const int j0 = w % jb * 16 * JT;
  w /= jb;
  const int split = w % a.splits;
  w /= a.splits;
  // (a tile's later lists, many of them empty, come last: next to each other they would leave most XCDs nothing else)
  const int tiles = (a.M + ROWS - 1) / ROWS;
  const int lane_of_list = w / tiles;
  const int m0 = (w - lane_of_list * tiles) * ROWS;
  const int looked = adapter_of(a, m0 + lane);
  const int own = lane < ROWS ? looked : -1;
  if (tid < ROWS && m0 + tid < a.M && split == 0 && lane_of_list == 0 && j0 == 0) a.row_id[m0 + tid] = own;
  const int k_begin = split * a.k_split, k_end = min(a.K, k_begin + a.k_split);
  const uint16_t* xp[MT];
  int mine[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    xp[t] = a.x + (size_t)min(m0 + 16 * t + col, a.M - 1) * a.xs;
    mine[t] = __shfl(own, 16 * t + col);
  }
  AdapterList list(own);
  for (int d = 0; list.left; ++d) {
    const int id = list.next();
    if (d % a.lists != lane_of_list) continue;
    const uint16_t* ap[JT];
#pragma unroll
    for (int t = 0; t < JT; ++t)       // rows past the rank give products that nobody keeps
      ap[t] = a.a + ((size_t)id * a.r + min(j0 + 16 * t + col, a.r - 1)) * a.K;
    f32x4 acc[JT][MT];
#pragma unroll
    for (int j = 0; j < JT; ++j)
#pragma unroll
      for (int t = 0; t < MT; ++t) acc[j][t] = f32x4{};
    for (int k0 = k_begin + kAdRun * wave; k0 < k_end; k0 += kAdRun * WAVES) {
      u32x4 xf[DEEP][MT], af[DEEP][JT];
#pragma unroll
      for (int u = 0; u < DEEP; ++u) {          // (past the end the last elements once more, taken as zero below; K is a multiple of 8)
        const int k = min(k0 + 32 * u + 8 * g, a.K - 8);
#pragma unroll
        for (int t = 0; t < MT; ++t) xf[u][t] = *reinterpret_cast<const u32x4*>(xp[t] + k);
#pragma unroll
        for (int j = 0; j < JT; ++j) af[u][j] = *reinterpret_cast<const u32x4*>(ap[j] + k);
      }
#pragma unroll
      for (int u = 0; u < DEEP; ++u) {
        const bool in = k0 + 32 * u + 8 * g < k_end;
#pragma unroll
        for (int t = 0; t < MT; ++t) xf[u][t] = in ? xf[u][t] : u32x4{};
#pragma unroll
        for (int j = 0; j < JT; ++j) {
          af[u][j] = in ? af[u][j] : u32x4{};
#pragma unroll
          for (int t = 0; t < MT; ++t)
            acc[j][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, af[u][j]), __builtin_bit_cast(bf16x8, xf[u][t]), acc[j][t], 0, 0, 0);
        }
      }
    }
#pragma unroll
    for (int j = 0; j < JT; ++j)
#pragma unroll
      for (int t = 0; t < MT; ++t) red[wave][j * MT + t][lane] = acc[j][t];
    __syncthreads();
    const float gain = a.gain ? a.gain[id] : 1.0f;
#pragma unroll
    for (int p0 = 0; p0 < JT * MT; p0 += WAVES) {      // the waves' sums, in their order
      const int p = p0 + wave;
      if (p >= JT * MT) break;
      f32x4 sum = red[0][p][lane];
#pragma unroll
      for (int i = 1; i < WAVES; ++i) sum += red[i][p][lane];
      const int t = p % MT, j = j0 + 16 * (p / MT) + 4 * g, row = 16 * t + col;
      int of = mine[0];
#pragma unroll
      for (int i = 1; i < MT; ++i) of = t == i ? mine[i] : of;
      // (r is a multiple of 8, and 4 g of 4: a lane's four are all in the rank or none)
      if (j < a.r && of == id) *reinterpret_cast<f32x4*>(a.mid + ((size_t)split * a.M + m0 + row) * a.r + j) = sum * gain;
    }
    __syncthreads();
  }
}

// x = p[0] + p[1] + p[2] with eight bits of its significand in each, so that all 24 are there: as three bf16 numbers mid
// enters the product whole, and fp32 y sees no bf16 step. Cut and not rounded, so that no finite number becomes infinite. The
// first two are the largest bf16 numbers below what is left in size, not up to it (1 is 1 - 2^-8 and so on), so that none
// of the three is 0 beside one that is not, and an infinite weight gives an infinity of the product's sign: 0 times it
// would be NaN. What is below, at most a step of the first part (2^-7), is exact in the other two: the second leaves at
// most a step of its own, 2^-15, a multiple of 2^-23. Below 2^-90 the last part would come near bf16's smallest numbers,
// and x is cut as it is. An infinity or NaN is all three parts.
__device__ __forceinline__ void split_bf16(float x, uint32_t (&p)[3]) {
  const uint32_t size = __builtin_bit_cast(uint32_t, x) & 0x7f800000u;
  const bool finite = size != 0x7f800000u;
  const uint32_t below = finite && size >= (127u - 90u) << 23 ? 1u : 0u;
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    const uint32_t u = (__builtin_bit_cast(uint32_t, x) - (i < 2 ? below : 0u)) & 0xffff0000u;
    p[i] = u >> 16;
    x = finite ? x - __builtin_bit_cast(float, u) : x;
  }
}

// y[m][c] += sum_j b[id][c][j] mid[m][j]. A wave takes 16 MT rows and `chunks` times 16 NT columns, the next of which are on
// their way while it computes; its rows' mid stays in registers. S: runs of 32 of the rank. U: adapters whose weights
// are loaded at once; more than one only where `chunks` is 1.
template <int MT, int NT, int S, int U>
__global__ __launch_bounds__(kAdThreads) void adapter_up_kernel(AdapterArgs a) {
  constexpr int ROWS = 16 * MT, COLS = 16 * NT * kAdWaves;
  const int tid = threadIdx.x, lane = tid & 63, col = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int nb = (a.N + COLS * a.chunks - 1) / (COLS * a.chunks);
  const int m0 = (int)blockIdx.x / nb * ROWS;
  int n0 = (int)blockIdx.x % nb * a.chunks * COLS + wave * 16 * NT;
  const int n_end = min(a.N, ((int)blockIdx.x % nb + 1) * a.chunks * COLS);
  const int own = lane < ROWS && m0 + lane < a.M ? a.row_id[m0 + lane] : -1;
  auto load = [&](int at, f32x4 (&y)[MT][NT]) {
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      const float* yp = a.y + (size_t)min(m0 + 16 * t + col, a.M - 1) * a.ys + at + 4 * g;
#pragma unroll
      for (int c = 0; c < NT; ++c) {
        if (at + 16 * NT <= a.N) {
          y[t][c] = *reinterpret_cast<const f32x4_by4*>(yp + 16 * c);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) y[t][c][e] = at + 16 * c + 4 * g + e < a.N ? yp[16 * c + e] : 0.0f;
        }
      }
    }
  };
  // the weights of adapters id[] for the columns from `at` on
  auto weights = [&](int at, const int (&id)[U], u32x4 (&bf)[U][NT][S]) {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int c = 0; c < NT; ++c) {
        const uint16_t* bp = a.b + ((size_t)id[u] * a.N + min(at + 16 * c + col, a.N - 1)) * a.r;
#pragma unroll
        for (int k = 0; k < S; ++k) bf[u][c][k] = *reinterpret_cast<const u32x4*>(bp + min(32 * k + 8 * g, a.r - 8));
      }
  };
  auto take = [](AdapterList& list, int (&id)[U]) {
#pragma unroll
    for (int u = 0; u < U; ++u) id[u] = u == 0 || list.left ? list.next() : id[0];       // (one of them again changes nothing)
  };
  f32x4 out[MT][NT];
  load(n0, out);
  AdapterList rest(own);
  if (!rest.left) return;
  int first[U];
  take(rest, first);
  u32x4 bf[U][NT][S];
  weights(n0, first, bf);
  int mine[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) mine[t] = __shfl(own, 16 * t + col);
  // mid of 16 rows and a run of the rank as matrix operands
  auto operands = [&](int t, int k, int of, u32x4 (&w)[3]) {
    const int m = m0 + 16 * t + col, j = 32 * k + 8 * g;
    float v[8] = {};
    if (of >= 0 && j < a.r) {
      for (int p = 0; p < a.splits; ++p) {
        const float* mp = a.mid + ((size_t)p * a.M + m) * a.r + j;
        const f32x4 v0 = *reinterpret_cast<const f32x4*>(mp), v1 = *reinterpret_cast<const f32x4*>(mp + 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += v0[e], v[4 + e] += v1[e];
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      uint32_t p0[3], p1[3];
      split_bf16(v[2 * e], p0);
      split_bf16(v[2 * e + 1], p1);
#pragma unroll
      for (int i = 0; i < 3; ++i) w[i][e] = p0[i] | p1[i] << 16;
    }
  };
  bf16x8 mid[MT][S][3];
  // (each wave for itself, 8500 rows of rank 64 took 12% longer)
  if constexpr (MT == 1) {
#pragma unroll
    for (int k = 0; k < S; ++k) {
      u32x4 w[3];
      operands(0, k, mine[0], w);
#pragma unroll
      for (int i = 0; i < 3; ++i) mid[0][k][i] = __builtin_bit_cast(bf16x8, w[i]);
    }
  } else {                 // each wave some of them for all
    __shared__ u32x4 shared_mid[MT * S][3][64];
    for (int p = wave; p < MT * S; p += kAdWaves) {
      u32x4 w[3];
      operands(p / S, p % S, __shfl(own, 16 * (p / S) + col), w);
#pragma unroll
      for (int i = 0; i < 3; ++i) shared_mid[p][i][lane] = w[i];
    }
    __syncthreads();
#pragma unroll
    for (int p = 0; p < MT * S; ++p)
#pragma unroll
      for (int i = 0; i < 3; ++i) mid[p / S][p % S][i] = __builtin_bit_cast(bf16x8, shared_mid[p][i][lane]);
  }
  if (n0 >= n_end) return;
  auto multiply = [&](const int (&id)[U], const u32x4 (&bf)[U][NT][S]) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int c = 0; c < NT; ++c) {
        u32x4 w[S];
#pragma unroll
        for (int k = 0; k < S; ++k) w[k] = 32 * k + 8 * g < a.r ? bf[u][c][k] : u32x4{};
#pragma unroll
        for (int t = 0; t < MT; ++t) {
          f32x4 acc = f32x4{};
#pragma unroll
          for (int i = 2; i >= 0; --i)       // the smallest first
#pragma unroll
            for (int k = 0; k < S; ++k)
              acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w[k]), mid[t][k][i], acc, 0, 0, 0);
          const bool keep = mine[t] == id[u] && (u == 0 || id[u] != id[0]);
#pragma unroll
          for (int e = 0; e < 4; ++e) out[t][c][e] = keep ? out[t][c][e] + acc[e] : out[t][c][e];
        }
      }
    }
  };
  for (;;) {
    // Loads end in the order in which they begin: what the next columns need goes out here, all of it, so that none of these
    // columns' waits for it.
    f32x4 next[MT][NT];
    u32x4 bn[U][NT][S];
    const bool more = U == 1 && n0 + COLS < n_end;
    if (more) {
      weights(n0 + COLS, first, bn);
      load(n0 + COLS, next);
    }
    multiply(first, bf);
    for (AdapterList list = rest; list.left;) {
      int id[U];
      take(list, id);
      weights(n0, id, bf);
      multiply(id, bf);
    }
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      if (mine[t] < 0) continue;
      float* yp = a.y + (size_t)(m0 + 16 * t + col) * a.ys + n0 + 4 * g;
#pragma unroll
      for (int c = 0; c < NT; ++c) {
        if (n0 + 16 * NT <= a.N) {
          *reinterpret_cast<f32x4_by4*>(yp + 16 * c) = out[t][c];
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (n0 + 16 * c + 4 * g + e < a.N) yp[16 * c + e] = out[t][c][e];
        }
      }
    }
    if (!more) break;
    n0 += COLS;
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
      for (int c = 0; c < NT; ++c) out[t][c] = next[t][c];
#pragma unroll
    for (int c = 0; c < NT; ++c)
#pragma unroll
      for (int k = 0; k < S; ++k) bf[0][c][k] = bn[0][c][k];
  }
}

}  // namespace
}  // namespace qg
