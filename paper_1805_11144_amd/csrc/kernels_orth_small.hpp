// Orthogonalised updates of small matrices: one workgroup per matrix, which
// stays in LDS from its first read to its last write.
//
// X [n][m] (n <= 64 rows padded to 16 NT) is float32 in LDS, products run on
// v_mfma_f32_16x16x4f32 (lane l of a wavefront holds row or column l % 16 and
// one k of four; of the result, column l % 16 and rows 4 (l / 16) + q).  Rows
// lie 4 banks apart modulo the 64 banks, so 16 lanes' 16-byte reads come from 64
// different ones.  An iteration:
//   A = X X'    the sum over m split over the wavefronts where A has few tiles,
//               added up in their order; else a wavefront takes whole tiles
//   Q           = c0 I + c1 A + c2 A A
//   X <- Q X    column tiles of 16: each depends on nothing but itself, so they
//               are replaced in place
// Only the launch, the read and the write touch the rest of the chip.  Bound by
// latency: barriers, LDS and dependent products.  200 matrices of 500 x 16 take
// 19 us, and 238 on the tiled kernels (17 launches).  Taken wherever a matrix
// fits, since one workgroup is the faster even for a single one: 64 x 64 29 us and
// 72 tiled, 32 x 400 34 and 90, 48 x 600 83 and 97, 16 x 2000 50 and 115; 64 of 64 x
// 300 76 and 120.  At the largest that fit, 64 x 400, up to eight matrices take
// 94 and 90: even, so the number of matrices plays no part.
#pragma once

#include "kernels_orth.hpp"

typedef float floatx4 __attribute__((ext_vector_type(4)));

constexpr int kOrthWaves = 8;

struct OrthSmall {
  OrthSrc src;
  void* out;               // out, or the weight of an update
  int64_t omat, orow;
  int32_t n, m, stride;    // m padded to 16 is within the stride
  int32_t steps;
  float c0, c1, c2, keep, rate;
  double eps;
};

constexpr int orth_tiles(int nt) { return nt * (nt + 1) / 2; }

// LDS of one workgroup in floats: X, A, Q and the wavefronts' shares of A.
constexpr int64_t orth_small_floats(int nt, int64_t stride) {
  return 16 * nt * stride + 2 * 16 * nt * (16 * nt + 4) + (nt <= 2 ? kOrthWaves * orth_tiles(nt) * 256 : 0);
}

template <class T, bool UPDATE, int NT>
__global__ void __launch_bounds__(64 * kOrthWaves) k_orth_small(OrthSmall p) {
  constexpr int N = 16 * NT, AS = N + 4, TILES = orth_tiles(NT), THREADS = 64 * kOrthWaves;
  extern __shared__ __attribute__((aligned(16))) float orth_lds[];
  __shared__ double red[kOrthWaves];
  float* X = orth_lds;                 // [N][stride]
  float* A = X + N * p.stride;         // [N][AS]
  float* Q = A + N * AS;               // [N][AS]
  float* share = Q + N * AS;           // NT <= 2: [kOrthWaves][TILES][256]
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64, l16 = lane % 16, l4 = lane / 16;
  const int64_t mat = blockIdx.x;
  const int rows = (int)p.src.rows, cols = (int)p.src.cols;
  const bool tall = rows > cols;
  const T* x = (const T*)p.src.x + mat * p.src.mat;
  float* mom = UPDATE ? p.src.momentum + mat * rows * cols : nullptr;
  for (int i = tid; i < N * p.stride; i += THREADS) X[i] = 0.0f;
  __syncthreads();
  double sum = 0.0;
  const int n = rows * cols;
  // value i = (r, c), and the step to value i + THREADS without a division
  struct Place {
    int r, c;
  };
  const int dr = THREADS / cols, dc = THREADS - dr * cols;
  const auto onward = [&](Place& a) {
    a.r += dr, a.c += dc;
    if (a.c >= cols) a.c -= cols, ++a.r;
  };
  const Place begin{tid / cols, tid % cols};
  const auto within = [&](const Place& a) { return tall ? a.c * p.stride + a.r : a.r * p.stride + a.c; };
  Place at = begin;
  for (int i0 = tid; i0 < n; i0 += 8 * THREADS) {
    float in[8], mo[8];   // eight values on their way at once; past the end: the first one, not used
    int to[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      const bool live = i0 + q * THREADS < n;
      in[q] = as_f32(x[live ? at.r * p.src.row + at.c : 0]);
      if (UPDATE) mo[q] = mom[live ? i0 + q * THREADS : 0];
      to[q] = within(at);
      onward(at);
    }
#pragma unroll
    for (int q = 0; q < 8; ++q)
      if (i0 + q * THREADS < n) {
        float v = in[q];
        if constexpr (UPDATE) {
          const float m = fmaf(p.src.decay, mo[q], v);
          mom[i0 + q * THREADS] = m;
          v = p.src.nesterov ? fmaf(p.src.decay, m, v) : m;
        }
        X[to[q]] = v;
        sum += (double)v * v;
      }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_down(sum, o, 64);
  if (lane == 0) red[wave] = sum;
  __syncthreads();
  double total = 0.0;
#pragma unroll
  for (int w = 0; w < kOrthWaves; ++w) total += red[w];
  const double inv = 1.0 / (sqrt(total) + p.eps);
  for (int i = tid; i < p.n * p.stride; i += THREADS) X[i] = (float)(X[i] * inv);
  __syncthreads();
  // one product takes 4 values of k, one from each quarter of the wavefront; a lane's four values of 16 lie side by
  // side, so its part of a fragment of four products is one 16-byte read
  const auto quad = [&](const float* row, int k16) { return *(const floatx4*)(row + 16 * k16 + 4 * l4); };
  const int k16s = (p.m + 15) / 16, ctiles = k16s;
  for (int step = 0; step < p.steps; ++step) {
    if constexpr (NT <= 2) {
      floatx4 acc[TILES] = {};
#pragma unroll 2
      for (int k = wave; k < k16s; k += kOrthWaves) {
        floatx4 f[NT];
#pragma unroll
        for (int i = 0; i < NT; ++i) f[i] = quad(X + (16 * i + l16) * p.stride, k);
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int j = 0, t = 0; j < NT; ++j)
#pragma unroll
            for (int i = 0; i <= j; ++i, ++t)
              acc[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(f[i][e], f[j][e], acc[t], 0, 0, 0);
      }
#pragma unroll
      for (int t = 0; t < TILES; ++t)
#pragma unroll
        for (int q = 0; q < 4; ++q) share[(wave * TILES + t) * 256 + q * 64 + lane] = acc[t][q];
      __syncthreads();
      for (int i = tid; i < TILES * 256; i += THREADS) {
        float s = 0.0f;
#pragma unroll
        for (int w = 0; w < kOrthWaves; ++w) s += share[w * TILES * 256 + i];
        const int t = i / 256, q = i / 64 % 4, l = i % 64;
        const int tj = t == 0 ? 0 : 1, ti = t == 2 ? 1 : 0;   // tiles (0, 0), (0, 1), (1, 1)
        const int r = 16 * ti + 4 * (l / 16) + q, c = 16 * tj + l % 16;
        A[r * AS + c] = s;
        if (ti != tj) A[c * AS + r] = s;
      }
    } else {
      for (int t = wave; t < TILES; t += kOrthWaves) {
        int tj = 0;
        while ((tj + 1) * (tj + 2) / 2 <= t) ++tj;
        const int ti = t - tj * (tj + 1) / 2;
        floatx4 acc[4] = {};   // four sums, so that one product does not wait for the one before it
#pragma unroll 4
        for (int k = 0; k < k16s; ++k) {
          const floatx4 a = quad(X + (16 * ti + l16) * p.stride, k), b = quad(X + (16 * tj + l16) * p.stride, k);
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], acc[e], 0, 0, 0);
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int r = 16 * ti + 4 * l4 + q, c = 16 * tj + l16;
          const float s = (acc[0][q] + acc[1][q]) + (acc[2][q] + acc[3][q]);
          A[r * AS + c] = s;
          if (ti != tj) A[c * AS + r] = s;
        }
      }
    }
    __syncthreads();
    for (int t = wave; t < NT * NT; t += kOrthWaves) {
      const int ti = t / NT, tj = t % NT;
      floatx4 sum4[4] = {};
#pragma unroll
      for (int k = 0; k < NT; ++k) {   // A is symmetric
        const floatx4 a = quad(A + (16 * ti + l16) * AS, k), b = quad(A + (16 * tj + l16) * AS, k);
#pragma unroll
        for (int e = 0; e < 4; ++e) sum4[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], sum4[e], 0, 0, 0);
      }
      const floatx4 acc = (sum4[0] + sum4[1]) + (sum4[2] + sum4[3]);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int r = 16 * ti + 4 * l4 + q, c = 16 * tj + l16;
        Q[r * AS + c] = p.c2 * acc[q] + p.c1 * A[r * AS + c] + (r == c ? p.c0 : 0.0f);
      }
    }
    __syncthreads();
    floatx4 f[NT][NT];
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
      for (int k = 0; k < NT; ++k) f[i][k] = quad(Q + (16 * i + l16) * AS, k);
    for (int u = wave; u < ctiles; u += kOrthWaves) {
      floatx4 acc[NT] = {};
      float b[NT][4];
#pragma unroll
      for (int k = 0; k < NT; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) b[k][e] = X[(16 * k + 4 * l4 + e) * p.stride + 16 * u + l16];
#pragma unroll
      for (int k = 0; k < NT; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int i = 0; i < NT; ++i)
            acc[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(f[i][k][e], b[k][e], acc[i], 0, 0, 0);
#pragma unroll
      for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) X[(16 * i + 4 * l4 + q) * p.stride + 16 * u + l16] = acc[i][q];
    }
    __syncthreads();
  }
  using R = std::conditional_t<UPDATE, float, T>;
  R* out = (R*)p.out + mat * p.omat;
  at = begin;
  for (int i0 = tid; i0 < n; i0 += 8 * THREADS) {
    float old[8], v[8];
    R* o[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      const bool live = i0 + q * THREADS < n;
      o[q] = out + (live ? at.r * p.orow + at.c : 0);
      if (UPDATE) old[q] = (float)*o[q];
      v[q] = X[live ? within(at) : 0];
      onward(at);
    }
#pragma unroll
    for (int q = 0; q < 8; ++q)
      if (i0 + q * THREADS < n) *o[q] = UPDATE ? (R)(p.keep * old[q] - p.rate * v[q]) : (R)v[q];
  }
}
