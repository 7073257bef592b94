// Orthogonalised updates: X <- (c0 I + c1 A + c2 A A) X with A = X X', from
// X / (|X| + eps), `steps` times.
//
// Arithmetic: float32 products on the matrix cores run at a sixteenth of the
// rate of 16-bit ones.  A float32 value scaled into fp16's range is held as
// hi + lo, two fp16 numbers (22 bits), and a product of two matrices is
// hi hi' + hi lo' + lo hi' in float32 sums; the missing lo lo' is 2^-22 of the
// result, the size of a float32 sum's own rounding.  Where the result is
// rounded to bf16 one part is enough (11 bits against the result's 8).
// Matrices are scaled by powers of two that their bounds allow, so the parts
// stay clear of fp16's ends.
//
// Layout: n = min(rows, cols) <= m = the other; X [n][m] and its transpose
// [m][n] in fp16 parts, A and Q = c0 I + c1 A + c2 A A as [n][n], every side
// padded with zeros to whole tiles.  So each product is C = L R' with both
// operands contiguous along the sum: X X', A A (A is symmetric) and Q X.
// A and Q are symmetric: tiles below the diagonal are the others' mirror
// images.
#pragma once

#include "kernels_embed.hpp"

typedef _Float16 half_t;
typedef half_t halfx8 __attribute__((ext_vector_type(8)));
typedef float floatx16 __attribute__((ext_vector_type(16)));

constexpr int kOrthParts = 64;   // partial sums of a matrix's norm

// A matrix as the caller holds it.
struct OrthSrc {
  const void* x;          // x, or the gradient of an update
  float* momentum;        // updates only
  int64_t mat, row;       // strides
  int64_t rows, cols;
  float decay;            // momentum decay
  int32_t nesterov;
};

// Partial sums of squares in 64 bits: no float32 input overflows or loses
// them.  An update also advances its momentum.
template <class T, bool UPDATE>
__global__ void __launch_bounds__(256) k_orth_norm(OrthSrc s, double* parts) {
  __shared__ double red[4];
  const int64_t mat = blockIdx.x / kOrthParts, part = blockIdx.x % kOrthParts;
  const T* x = (const T*)s.x + mat * s.mat;
  float* mom = UPDATE ? s.momentum + mat * s.rows * s.cols : nullptr;
  double sum = 0.0;
  for (int64_t r = part; r < s.rows; r += kOrthParts)
    for (int64_t c = threadIdx.x; c < s.cols; c += 256) {
      float v = as_f32(x[r * s.row + c]);
      if constexpr (UPDATE) {
        const float m = fmaf(s.decay, mom[r * s.cols + c], v);
        mom[r * s.cols + c] = m;
        v = s.nesterov ? fmaf(s.decay, m, v) : m;
      }
      sum += (double)v * v;
    }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_down(sum, o, 64);
  if (threadIdx.x % 64 == 0) red[threadIdx.x / 64] = sum;
  __syncthreads();
  if (threadIdx.x == 0) parts[blockIdx.x] = (red[0] + red[1]) + (red[2] + red[3]);
}

__device__ __forceinline__ void split(float x, half_t& hi, half_t& lo) {
  hi = (half_t)x;
  lo = (half_t)(x - (float)hi);
}

// The first iterate, scale X / (|X| + eps), and its transpose.  grid: batch x
// (mp / 64) x (np / 64) tiles of 64 x 64.
template <class T, bool UPDATE, int PL>
__global__ void __launch_bounds__(256) k_orth_first(OrthSrc s, const double* parts, double eps, double scale, half_t* X,
                                                    half_t* XT, int32_t np, int32_t mp) {
  __shared__ float tile[64][65];
  __shared__ double inv_s;
  const int tid = threadIdx.x;
  const int32_t tn = np / 64, tm = mp / 64;
  const int64_t mat = blockIdx.x / (tn * tm);
  const int32_t u = blockIdx.x % (tn * tm), i0 = u / tm * 64, j0 = u % tm * 64;
  if (tid < 64) {
    double p = parts[mat * kOrthParts + tid];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) p += __shfl_down(p, o, 64);
    if (tid == 0) inv_s = scale / (sqrt(p) + eps);
  }
  __syncthreads();
  const double inv = inv_s;
  const bool tall = s.rows > s.cols;
  const T* x = (const T*)s.x + mat * s.mat;
  const float* mom = UPDATE ? s.momentum + mat * s.rows * s.cols : nullptr;
  // source rows r0.. and columns c0.. of the tile
  const int64_t r0 = tall ? j0 : i0, c0 = tall ? i0 : j0;
  for (int k = tid; k < 64 * 64; k += 256) {
    const int dr = k / 64, dc = k % 64;
    const int64_t r = r0 + dr, c = c0 + dc;
    float v = 0.0f;
    if (r < s.rows && c < s.cols) {
      v = as_f32(x[r * s.row + c]);
      if constexpr (UPDATE) {
        const float m = mom[r * s.cols + c];
        v = s.nesterov ? fmaf(s.decay, m, v) : m;
      }
      v = (float)(v * inv);
    }
    if (tall) tile[dc][dr] = v;
    else tile[dr][dc] = v;
  }
  __syncthreads();
  half_t* x0 = X + mat * PL * np * (int64_t)mp;
  half_t* t0 = XT + mat * PL * np * (int64_t)mp;
  const int64_t plane = (int64_t)np * mp;
  for (int k = tid; k < 64 * 64; k += 256) {
    const int p = k / 64, q = k % 64;
    half_t hi, lo;
    split(tile[p][q], hi, lo);
    x0[(int64_t)(i0 + p) * mp + j0 + q] = hi;
    if (PL == 2) x0[plane + (int64_t)(i0 + p) * mp + j0 + q] = lo;
    split(tile[q][p], hi, lo);
    t0[(int64_t)(j0 + p) * np + i0 + q] = hi;
    if (PL == 2) t0[plane + (int64_t)(j0 + p) * np + i0 + q] = lo;
  }
}

enum OrthEnd { kEndGram, kEndPoly, kEndNext, kEndOut, kEndUpdate };

struct OrthGemm {
  const half_t *l, *r;        // L [M][K], R [N][K]
  int32_t M, N, K;            // padded
  half_t* c;                  // C [M][N], or null
  half_t* ct;                 // its transpose (kEndNext)
  const half_t* a;            // A (kEndPoly)
  float f;                    // sums to C's scale
  float c0, c1;               // kEndPoly, in C's scale (c1 times A's stored value)
  // kEndOut, kEndUpdate
  void* out;
  int64_t mat, row, rows, cols;
  float keep, rate;           // weight <- keep weight - rate X
};

// C = L R' on TILE x TILE tiles, a workgroup of four wavefronts each; K in
// slices of 32, fetched into registers while the one before is multiplied, two
// buffers in LDS (rows padded to 40 numbers, so that the 16-byte reads of a
// fragment spread over the banks).
template <int PL, int TILE, int END, class T>
__global__ void __launch_bounds__(256) k_orth_gemm(OrthGemm g) {
  constexpr int KS = 32, P = 40, W = TILE / 2, B = W / 32, U = PL * TILE * KS / 8 / 256;
  constexpr bool SYM = END == kEndGram || END == kEndPoly;
  static_assert(U >= 1, "every thread fetches");
  extern __shared__ __attribute__((aligned(16))) half_t lds[];
  typedef half_t Slab[2][PL][TILE][P];
  Slab& Ls = *(Slab*)lds;
  Slab& Rs = *(Slab*)(lds + sizeof(Slab) / sizeof(half_t));
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64, wm = wave / 2, wn = wave % 2;
  const int32_t tm = g.M / TILE, tn = g.N / TILE;
  const int32_t per = SYM ? tm * (tm + 1) / 2 : tm * tn;
  const int64_t mat = blockIdx.x / per;
  int32_t u = blockIdx.x % per, ti, tj;
  if (SYM) {   // tiles ti <= tj, by columns
    tj = (int32_t)((sqrtf(8.0f * u + 1.0f) - 1.0f) * 0.5f);
    while (tj * (tj + 1) / 2 > u) --tj;
    while ((tj + 1) * (tj + 2) / 2 <= u) ++tj;
    ti = u - tj * (tj + 1) / 2;
  } else {
    ti = u % tm, tj = u / tm;
  }
  const int64_t lplane = (int64_t)g.M * g.K, rplane = (int64_t)g.N * g.K;
  const half_t* L = g.l + mat * PL * lplane + (int64_t)ti * TILE * g.K;
  const half_t* R = g.r + mat * PL * rplane + (int64_t)tj * TILE * g.K;
  halfx8 fl[U], fr[U];
  auto fetch = [&](int32_t k0) {
#pragma unroll
    for (int q = 0; q < U; ++q) {
      const int i = q * 256 + tid, p = i / (TILE * KS / 8), row = i / (KS / 8) % TILE, k = 8 * (i % (KS / 8));
      fl[q] = *(const halfx8*)(L + p * lplane + (int64_t)row * g.K + k0 + k);
      fr[q] = *(const halfx8*)(R + p * rplane + (int64_t)row * g.K + k0 + k);
    }
  };
  auto store = [&](int buf) {
#pragma unroll
    for (int q = 0; q < U; ++q) {
      const int i = q * 256 + tid, p = i / (TILE * KS / 8), row = i / (KS / 8) % TILE, k = 8 * (i % (KS / 8));
      *(halfx8*)&Ls[buf][p][row][k] = fl[q];
      *(halfx8*)&Rs[buf][p][row][k] = fr[q];
    }
  };
  floatx16 acc[B][B];
#pragma unroll
  for (int i = 0; i < B; ++i)
#pragma unroll
    for (int j = 0; j < B; ++j) acc[i][j] = floatx16{};
  fetch(0);
  store(0);
  __syncthreads();
  int buf = 0;
  for (int32_t k0 = 0; k0 < g.K; k0 += KS) {
    const bool more = k0 + KS < g.K;
    if (more) fetch(k0 + KS);
#pragma unroll
    for (int ks = 0; ks < KS; ks += 16) {
      halfx8 a[PL][B], b[PL][B];
#pragma unroll
      for (int p = 0; p < PL; ++p)
#pragma unroll
        for (int i = 0; i < B; ++i) {
          a[p][i] = *(const halfx8*)&Ls[buf][p][wm * W + i * 32 + lane % 32][ks + 8 * (lane / 32)];
          b[p][i] = *(const halfx8*)&Rs[buf][p][wn * W + i * 32 + lane % 32][ks + 8 * (lane / 32)];
        }
#pragma unroll
      for (int i = 0; i < B; ++i)
#pragma unroll
        for (int j = 0; j < B; ++j) {
          if constexpr (PL == 2) {
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[1][i], b[0][j], acc[i][j], 0, 0, 0);
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[0][i], b[1][j], acc[i][j], 0, 0, 0);
          }
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[0][i], b[0][j], acc[i][j], 0, 0, 0);
        }
    }
    if (more) store(buf ^ 1);
    __syncthreads();
    buf ^= 1;
  }
  // a lane holds column lane % 32 and rows 8 (q / 4) + 4 (lane / 32) + q % 4 of each 32 x 32 block
  const int64_t cplane = (int64_t)g.M * g.N;
  half_t* C = g.c + mat * PL * cplane;
  half_t* CT = END == kEndNext ? g.ct + mat * PL * cplane : nullptr;
  const half_t* A = END == kEndPoly ? g.a + mat * PL * cplane : nullptr;
#pragma unroll
  for (int i = 0; i < B; ++i)
#pragma unroll
    for (int j = 0; j < B; ++j) {
      const int64_t col = (int64_t)tj * TILE + wn * W + j * 32 + lane % 32;
#pragma unroll
      for (int q = 0; q < 16; ++q) {
        const int64_t row = (int64_t)ti * TILE + wm * W + i * 32 + 8 * (q / 4) + 4 * (lane / 32) + q % 4;
        float v = g.f * acc[i][j][q];
        if constexpr (END == kEndOut || END == kEndUpdate) {
          const bool tall = g.rows > g.cols;
          const int64_t r = tall ? col : row, c = tall ? row : col;
          if (r < g.rows && c < g.cols) {
            T* o = (T*)g.out + mat * g.mat + r * g.row + c;
            if constexpr (END == kEndOut) *o = (T)v;
            else *o = (T)(g.keep * (float)*o - g.rate * v);
          }
        } else {
          if constexpr (END == kEndPoly) {
            float av = (float)A[row * g.N + col];
            if (PL == 2) av += (float)A[cplane + row * g.N + col];
            v += g.c1 * av + (row == col ? g.c0 : 0.0f);
          }
          half_t hi, lo;
          split(v, hi, lo);
          C[row * g.N + col] = hi;
          if (PL == 2) C[cplane + row * g.N + col] = lo;
          if (SYM ? ti != tj : END == kEndNext) {
            half_t* D = SYM ? C : CT;
            D[col * g.M + row] = hi;
            if (PL == 2) D[cplane + col * g.M + row] = lo;
          }
        }
      }
    }
}
