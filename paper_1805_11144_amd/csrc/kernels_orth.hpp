// Orthogonalised updates: X <- (c0 I + c1 A + c2 A A) X with A = X X', from
// X / (|X| + eps), `steps` times.
//
// Arithmetic: float32 products on the matrix cores run at a sixteenth of the
// rate of 16-bit ones.  A float32 value scaled into fp16's range is held as
// hi + lo, two fp16 numbers (22 bits), and a product of two matrices is
// hi hi' + hi lo' + lo hi' in float32 sums; the missing lo lo' is 2^-22 of the
// result, the size of a float32 sum's own rounding.  (Against 64 bits the result
// is about half as far off as five iterations of float32 products are.)  A bf16
// result takes the same two parts: an iteration lets the rounding of small
// singular values grow with them, by 3.4445^5 = 485 in all, and with one part
// (11 bits) a matrix of 16 strong directions came out 4e-2 off, 25 times its own
// rounding.  Matrices are scaled by powers of two that their bounds allow, so
// the parts stay clear of fp16's ends.  A matrix whose norm is below eps, or that
// the coefficients shrink, is also lifted: its norm is at most 2^-E from the
// start, and at most 2^(g - E) after steps that let it grow by 2^g, so it is held
// 2^max(0, E - g) times as large and stays below one.
//
// Layout: n = min(rows, cols) <= m = the other; X [n][m] and its transpose
// [m][n] in fp16 parts, A and Q = c0 I + c1 A + c2 A A as [n][n], every side
// padded with zeros to whole tiles.  So each product is C = L R' with both
// operands contiguous along the sum: X X', A A (A is symmetric) and Q X.
// A and Q are symmetric: blocks below the diagonal are the others' mirror
// images and are not computed.
//
// What bounds it: large matrices the matrix cores (4096 x 4096: Q X 335 to 350
// us, 1.2 PFLOP/s of 16-bit products, as a large library product in bf16, the
// cores busy 60% of the cycles; X X' and A A 250, half the blocks at 0.85: 528
// tiles on 256 CUs), small ones a launch's latency (1024 x 784: 12 to 15 us for
// each of 15 products that take 2 at full rate, the matrix cores busy 2200 to 4100
// of some 25000 cycles).  Step by step at 4096 x 4096: 5.0 ms with tiles straight
// from memory to LDS; 4.4 with slices of k behind each other and 256 x 256 tiles
// for Q X; 4.2 with results in 16-byte words.
#pragma once

#include "kernels_embed.hpp"
#include "operators_rules.hpp"

using ms::kOrthSlice;

typedef _Float16 half_t;
typedef half_t halfx8 __attribute__((ext_vector_type(8)));
typedef half_t halfx4 __attribute__((ext_vector_type(4)));
typedef float floatx16 __attribute__((ext_vector_type(16)));

constexpr int kPair = 2;          // fp16 parts of a value: hi, lo
constexpr int kOrthParts = 256;   // partial sums of a matrix's norm

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
// them.  An update also advances its momentum.  A workgroup takes every
// kOrthParts-th run of 4096 values of a packed matrix, V at a time, or (V = 0)
// every kOrthParts-th row.
template <class T, bool UPDATE, int V>
__global__ void __launch_bounds__(256) k_orth_norm(OrthSrc s, double* parts) {
  __shared__ double red[4];
  const int64_t mat = blockIdx.x / kOrthParts, part = blockIdx.x % kOrthParts;
  const T* x = (const T*)s.x + mat * s.mat;
  float* mom = UPDATE ? s.momentum + mat * s.rows * s.cols : nullptr;
  double sum = 0.0;
  const auto take = [&](float v, float* m) {
    if constexpr (UPDATE) {
      *m = fmaf(s.decay, *m, v);
      v = s.nesterov ? fmaf(s.decay, *m, v) : *m;
    }
    sum += (double)v * v;
  };
  if constexpr (V > 0) {
    constexpr int A = 16 / V;
    const int64_t n = s.rows * s.cols;
    for (int64_t i0 = part * 4096 + threadIdx.x * V; i0 < n; i0 += kOrthParts * 4096) {
      Words<T, V> v[A];
      Words<float, V> m[A];
#pragma unroll
      for (int q = 0; q < A; ++q) {
        const int64_t i = min(i0 + q * 256 * V, n - V);   // past the end: read, and not used
        v[q] = *(const Words<T, V>*)(x + i);
        if (UPDATE) m[q] = *(const Words<float, V>*)(mom + i);
      }
#pragma unroll
      for (int q = 0; q < A; ++q)
        if (i0 + q * 256 * V < n) {
#pragma unroll
          for (int e = 0; e < V; ++e) take(as_f32(v[q].v[e]), &m[q].v[e]);
          if (UPDATE) *(Words<float, V>*)(mom + i0 + q * 256 * V) = m[q];
        }
    }
  } else {
    for (int64_t r = part; r < s.rows; r += kOrthParts)
      for (int64_t c = threadIdx.x; c < s.cols; c += 256) {
        float m = UPDATE ? mom[r * s.cols + c] : 0.0f;
        take(as_f32(x[r * s.row + c]), &m);
        if (UPDATE) mom[r * s.cols + c] = m;
      }
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

// Where value (row, k) of a matrix with `rows` rows is: slices of KS values of k
// lie one after the other, so a tile's part of a slice is one contiguous piece.
// With rows of whole k behind each other, the rows of a tile of a 4096 x 4096
// matrix are 8 KB apart and load a few of the L2's channels only.
template <int KS>
__device__ __forceinline__ int64_t orth_at(int64_t rows, int64_t row, int64_t k) {
  return (k / KS * rows + row) * KS + k % KS;
}

// The first iterate, scale X / (|X| + eps) lifted by 2^E, and its transpose; E to
// lift[].  grid: batch x (mp / 64) x (np / 64) tiles of 64 x 64.
template <class T, bool UPDATE, int KS>
__global__ void __launch_bounds__(256) k_orth_first(OrthSrc s, const double* parts, double eps, double scale, half_t* X,
                                                    half_t* XT, int32_t* lift, int32_t np, int32_t mp) {
  __shared__ float tile[64][65];
  __shared__ double inv_s;
  const int tid = threadIdx.x;
  const int32_t tn = np / 64, tm = mp / 64;
  const int64_t mat = blockIdx.x / (tn * tm);
  const int32_t u = blockIdx.x % (tn * tm), i0 = u / tm * 64, j0 = u % tm * 64;
  if (tid < 64) {
    double p = 0.0;
#pragma unroll
    for (int q = 0; q < kOrthParts / 64; ++q) p += parts[mat * kOrthParts + q * 64 + tid];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) p += __shfl_down(p, o, 64);
    if (tid == 0) {
      const double norm = sqrt(p), ratio = (norm + eps) / norm;   // not finite for zeros
      const int e = ratio < 1e300 ? ilogb(ratio) : 0;
      inv_s = ldexp(scale / (norm + eps), e);
      if (u == 0) lift[mat] = e;
    }
  }
  __syncthreads();
  const double inv = inv_s;
  const bool tall = s.rows > s.cols;
  const T* x = (const T*)s.x + mat * s.mat;
  const float* mom = UPDATE ? s.momentum + mat * s.rows * s.cols : nullptr;
  // source rows r0.. and columns c0.. of the tile
  const int64_t r0 = tall ? j0 : i0, c0 = tall ? i0 : j0;
  float in[16], mo[16];   // all on their way at once; past the matrix's end: read at its last value, and not used
  const int dc = tid % 64;
  const int64_t c = c0 + dc, cc = min(c, s.cols - 1);
#pragma unroll
  for (int k = 0; k < 16; ++k) {
    const int64_t r = min(r0 + tid / 64 + 4 * k, s.rows - 1);
    in[k] = as_f32(x[r * s.row + cc]);
    if (UPDATE) mo[k] = mom[r * s.cols + cc];
  }
#pragma unroll
  for (int k = 0; k < 16; ++k) {
    const int dr = tid / 64 + 4 * k;
    float v = in[k];
    if constexpr (UPDATE) v = s.nesterov ? fmaf(s.decay, mo[k], v) : mo[k];
    v = r0 + dr < s.rows && c < s.cols ? (float)(v * inv) : 0.0f;
    if (tall) tile[dc][dr] = v;
    else tile[dr][dc] = v;
  }
  __syncthreads();
  half_t* x0 = X + mat * kPair * np * (int64_t)mp;
  half_t* t0 = XT + mat * kPair * np * (int64_t)mp;
  const int64_t plane = (int64_t)np * mp;
  for (int k = tid; k < 64 * 64; k += 256) {
    const int p = k / 64, q = k % 64;
    half_t hi, lo;
    split(tile[p][q], hi, lo);
    const int64_t xa = orth_at<KS>(np, i0 + p, j0 + q), ta = orth_at<KS>(mp, j0 + p, i0 + q);
    x0[xa] = hi;
    x0[plane + xa] = lo;
    split(tile[q][p], hi, lo);
    t0[ta] = hi;
    t0[plane + ta] = lo;
  }
}

enum OrthEnd { kEndGram, kEndPoly, kEndNext, kEndOut, kEndUpdate, kEndPart };

struct OrthGemm {
  const half_t *l, *r;        // L [M][K], R [N][K]
  int32_t M, N, K;            // padded
  uint32_t batch, per, whole; // tiles of a matrix; tiles of all that are computed whole
  half_t* c;                  // C [M][N], or null
  half_t* ct;                 // its transpose (kEndNext)
  const half_t* a;            // A (kEndPoly)
  float f;                    // sums to C's scale
  float c0, c1;               // kEndPoly, in C's scale (c1 times A's stored value)
  const int32_t* lift;        // E of each matrix
  int32_t grown, grows;       // g before and after this step
  // kEndPart: the sum over slices [part * slices, ..) alone, unscaled, to sums[part][matrix][M][M]
  float* sums;
  int32_t slices, parts;      // slices of a part (all of them, and 1, for other ends)
  // kEndOut, kEndUpdate
  void* out;
  int64_t mat, row, rows, cols;
  float keep, rate;           // weight <- keep weight - rate X
};

// 16 bytes per lane from memory straight to LDS: lane i's to dst + 16 i (dst
// uniform over the wavefront).
__device__ __forceinline__ void fetch_lds(const half_t* src, half_t* dst) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src,
                                   (__attribute__((address_space(3))) void*)dst, 16, 0, 0);
}

// A barrier that leaves this wavefront's last N loads to LDS on their way.
// __syncthreads waits for all of them.
template <int N>
__device__ __forceinline__ void barrier_but() {
  static_assert(N < 64, "six bits");
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// C = L R' on the TILE x TILE tile at (row, col) of matrix `mat`.  2 x WC
// wavefronts share a tile; K runs in slices of KS through ST buffers in LDS,
// ST - 1 slices on their way while one is multiplied.  KG = 2: a second group
// of wavefronts takes every other slice, and the two sums are added at the end;
// where tiles are fewer than the CUs, that is what shortens a call.
// A slice's rows are KS / 8 chunks of 16 bytes without padding (memory goes to
// LDS in lane order); chunk c of row r sits at c ^ (r / (128 / KS)), so the
// rows of a fragment read different banks.
template <int TILE, int WC, int KS, int ST, int KG, int END, class T>
__device__ __forceinline__ void orth_tile(const OrthGemm& g, half_t* lds, int64_t mat, int32_t part, int32_t trow,
                                          int32_t tcol) {
  constexpr int NW = 2 * WC, WM = TILE / 2, WN = TILE / WC, BI = WM / 32, BJ = WN / 32;
  constexpr int CH = KS / 8, U = kPair * TILE * CH / (64 * NW);
  static_assert(BI >= 1 && BJ >= 1 && U >= 1, "work for every wavefront");
  constexpr bool SYM = END == kEndGram || END == kEndPoly || END == kEndPart;
  constexpr int LEFT = kPair * TILE * KS, SLAB = 2 * LEFT;   // of one slice; lds: [KG][ST][SLAB]
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64 % NW);
  const int group = KG == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / (64 * NW));
  const int wm = wave / WC, wn = wave % WC;
  const auto swizzle = [](int row) { return row / (128 / KS) % CH; };
  const int64_t lplane = (int64_t)g.M * g.K, rplane = (int64_t)g.N * g.K;
  const half_t* L = g.l + mat * kPair * lplane + (int64_t)trow * KS;
  const half_t* R = g.r + mat * kPair * rplane + (int64_t)tcol * KS;
  half_t* own = lds + group * ST * SLAB;
  // the lane's chunks of a slice, in values within a plane
  uint32_t off[U];
#pragma unroll
  for (int q = 0; q < U; ++q) {
    const int i = (q * NW + wave) * 64 + lane, row = i / CH % TILE;
    off[q] = (uint32_t)(row * KS + 8 * (i % CH ^ swizzle(row)));
  }
  const auto fetch = [&](int64_t slice, int buf) {
#pragma unroll
    for (int q = 0; q < U; ++q) {
      const int i0 = (q * NW + wave) * 64, p = i0 / (TILE * CH);
      fetch_lds(L + p * lplane + slice * g.M * KS + off[q], own + buf * SLAB + 8 * i0);
      fetch_lds(R + p * rplane + slice * g.N * KS + off[q], own + buf * SLAB + LEFT + 8 * i0);
    }
  };
  // where a wavefront has a single block, several sums for it, so that a product does not wait for the one before
  constexpr int NA = BI * BJ > 1 ? 1 : 3;
  floatx16 acc[BI][BJ], more[NA > 1 ? NA - 1 : 1];
#pragma unroll
  for (int i = 0; i < BI; ++i)
#pragma unroll
    for (int j = 0; j < BJ; ++j) acc[i][j] = floatx16{};
#pragma unroll
  for (int n = 0; n < NA - 1; ++n) more[n] = floatx16{};
  // what the iterates are lifted by, and what that makes of the sums
  float f = g.f, c1 = g.c1;
  int32_t shift = 0;
  if constexpr (END != kEndGram && END != kEndPart) {
    const int32_t now = max(0, g.lift[mat] - g.grown);
    if constexpr (END == kEndPoly) f = ldexpf(f, -4 * now), c1 = ldexpf(c1, -2 * now);
    else shift = END == kEndNext ? max(0, g.lift[mat] - g.grows) - now : -now;
  }
  // A's values for the polynomial, on their way while the product is made
  [[maybe_unused]] half_t early[kPair][16];
  constexpr bool EARLY = END == kEndPoly && BI * BJ == 1;
  if constexpr (EARLY) {
    const half_t* A = g.a + mat * kPair * lplane;   // A has the product's shape and K its side
#pragma unroll
    for (int p = 0; p < kPair; ++p)
#pragma unroll
      for (int q = 0; q < 16; ++q)
        early[p][q] = A[p * lplane + orth_at<KS>(g.M, trow + wm * WM + 8 * (q / 4) + 4 * (lane / 32) + q % 4,
                                                 tcol + wn * WN + lane % 32)];
  }
  const int32_t slices = min(g.slices, g.K / KS - part * g.slices);
  L += (int64_t)part * g.slices * g.M * KS, R += (int64_t)part * g.slices * g.N * KS;
#pragma unroll
  for (int q = 0; q < ST - 1; ++q)
    if (q * KG + group < slices) fetch(q * KG + group, q);
  int buf = 0;
  for (int32_t s0 = 0; s0 < slices; s0 += KG) {
    const int32_t s = s0 + group;
    // everyone's part of slice s is in LDS (the later ones may be on their way), and the buffer of the slice
    // before is read
    if (s0 + (ST - 1) * KG <= slices) barrier_but<(ST - 2) * 2 * U>();
    else barrier_but<0>();
    const half_t *Ls = own + buf * SLAB, *Rs = Ls + LEFT;
    halfx8 a[KS / 16][kPair][BI], b[KS / 16][kPair][BJ];
    if (s < slices) {
#pragma unroll
      for (int ks = 0; ks < KS / 16; ++ks)
#pragma unroll
        for (int p = 0; p < kPair; ++p) {
          const int c = 2 * ks + lane / 32;
#pragma unroll
          for (int i = 0; i < BI; ++i) {
            const int r = wm * WM + i * 32 + lane % 32;
            a[ks][p][i] = *(const halfx8*)(Ls + (p * TILE + r) * KS + 8 * (c ^ swizzle(r)));
          }
#pragma unroll
          for (int j = 0; j < BJ; ++j) {
            const int r = wn * WN + j * 32 + lane % 32;
            b[ks][p][j] = *(const halfx8*)(Rs + (p * TILE + r) * KS + 8 * (c ^ swizzle(r)));
          }
        }
    }
    const int32_t next = s + (ST - 1) * KG;
    if (next < slices) fetch(next, buf == 0 ? ST - 1 : buf - 1);
    if (s < slices) {
#pragma unroll
      for (int ks = 0; ks < KS / 16; ++ks)
#pragma unroll
        for (int i = 0; i < BI; ++i)
#pragma unroll
          for (int j = 0; j < BJ; ++j) {
            floatx16& s0 = acc[i][j];
            floatx16& s1 = NA > 1 ? more[0] : s0;
            floatx16& s2 = NA > 2 ? more[NA > 2 ? 1 : 0] : s0;
            s1 = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[ks][1][i], b[ks][0][j], s1, 0, 0, 0);
            s2 = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[ks][0][i], b[ks][1][j], s2, 0, 0, 0);
            s0 = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[ks][0][i], b[ks][0][j], s0, 0, 0, 0);
          }
    }
    buf = buf + 1 == ST ? 0 : buf + 1;
  }
#pragma unroll
  for (int n = 0; n < NA - 1; ++n) acc[0][0] += more[n];
  if constexpr (KG == 2) {   // the second group's sums through LDS
    __syncthreads();
    float* sums = (float*)lds + wave * BI * BJ * 16 * 64 + lane;
    if (group == 1) {
#pragma unroll
      for (int i = 0; i < BI; ++i)
#pragma unroll
        for (int j = 0; j < BJ; ++j)
#pragma unroll
          for (int q = 0; q < 16; ++q) sums[((i * BJ + j) * 16 + q) * 64] = acc[i][j][q];
    }
    __syncthreads();
    if (group == 1) return;
#pragma unroll
    for (int i = 0; i < BI; ++i)
#pragma unroll
      for (int j = 0; j < BJ; ++j)
#pragma unroll
        for (int q = 0; q < 16; ++q) acc[i][j][q] += sums[((i * BJ + j) * 16 + q) * 64];
  }
  // Results in fp16 parts: a block of 32 x 32 is one piece of memory.  Where a wavefront has several, it writes them
  // in 16-byte words, through its own 32 rows of 40 in LDS (4096 x 4096 4.4 -> 4.2 ms); a single one
  // goes out as it lies in the registers (1024 x 784: 187 us, through LDS 204).
  constexpr bool PARTS = END == kEndGram || END == kEndPoly || END == kEndNext, STAGED = PARTS && BI * BJ > 1;
  half_t* block = lds + wave * 32 * 40;
  if (STAGED) __syncthreads();   // the buffers are read
  const int64_t cplane = (int64_t)g.M * g.N;
  half_t* C = g.c + mat * kPair * cplane;
  half_t* CT = END == kEndNext ? g.ct + mat * kPair * cplane : nullptr;
  const half_t* A = END == kEndPoly ? g.a + mat * kPair * cplane : nullptr;
#pragma unroll
  for (int i = 0; i < BI; ++i)
#pragma unroll
    for (int j = 0; j < BJ; ++j) {
      // a lane holds column lane % 32 and rows 8 (q / 4) + 4 (lane / 32) + q % 4 of each 32 x 32 block
      const int32_t brow = trow + wm * WM + i * 32, bcol = tcol + wn * WN + j * 32;
      if (SYM && brow > bcol) continue;   // the mirror image of another block
      const int64_t col = bcol + lane % 32;
      halfx4 low[4];
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) {
        const int64_t row0 = brow + 8 * q4 + 4 * (lane / 32);
        halfx4 hi, lo;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int64_t row = row0 + q;
          float v = f * acc[i][j][4 * q4 + q];
          if (END == kEndNext || END == kEndOut || END == kEndUpdate) v = ldexpf(v, shift);
          if constexpr (END == kEndPart) {
            g.sums[((part * (int64_t)g.batch + mat) * g.M + row) * g.M + col] = acc[i][j][4 * q4 + q];
          } else if constexpr (END == kEndOut || END == kEndUpdate) {
            const bool tall = g.rows > g.cols;
            const int64_t r = tall ? col : row, c = tall ? row : col;
            if (r < g.rows && c < g.cols) {
              T* o = (T*)g.out + mat * g.mat + r * g.row + c;
              if constexpr (END == kEndOut) *o = (T)v;
              else *o = (T)(g.keep * (float)*o - g.rate * v);
            }
          } else {
            if constexpr (END == kEndPoly) {
              float av;
              if constexpr (EARLY) {
                av = (float)early[0][4 * q4 + q] + (float)early[1][4 * q4 + q];
              } else {
                av = (float)A[orth_at<KS>(g.M, row, col)] + (float)A[cplane + orth_at<KS>(g.M, row, col)];
              }
              v += c1 * av + (row == col ? g.c0 : 0.0f);
            }
            half_t h, l;
            split(v, h, l);
            hi[q] = h, lo[q] = l;
            if constexpr (STAGED) {
              block[(8 * q4 + 4 * (lane / 32) + q) * 40 + lane % 32] = h;
            } else {
              C[orth_at<KS>(g.M, row, col)] = h;
              C[cplane + orth_at<KS>(g.M, row, col)] = l;
            }
          }
        }
        low[q4] = lo;
        if constexpr (END == kEndGram || END == kEndPoly || END == kEndNext) {
          if (END == kEndNext || brow != bcol) {
            half_t* D = (SYM ? C : CT) + orth_at<KS>(g.N, col, row0);
            *(halfx4*)D = hi;
            *(halfx4*)(D + cplane) = lo;
          }
        }
      }
      if constexpr (STAGED) {   // two lanes to a row
        static_assert(KS == 32, "a block's rows lie behind each other");
        half_t* D = C + orth_at<KS>(g.M, brow, bcol) + lane * 16;
        const half_t* mine = block + lane / 2 * 40 + lane % 2 * 16;
#pragma unroll
        for (int p = 0; p < kPair; ++p) {
          if (p == 1) {
            wave_order();
#pragma unroll
            for (int q = 0; q < 16; ++q) block[(8 * (q / 4) + 4 * (lane / 32) + q % 4) * 40 + lane % 32] = low[q / 4][q % 4];
          }
          wave_order();
          *(halfx8*)(D + p * cplane) = *(const halfx8*)mine;
          *(halfx8*)(D + p * cplane + 8) = *(const halfx8*)(mine + 8);
        }
        wave_order();
      }
    }
}

// Tile number u of a matrix: all tiles by columns, or (SYM) those on and above
// the diagonal.
template <bool SYM>
__device__ __forceinline__ void orth_place(uint32_t u, uint32_t tm, uint32_t& ti, uint32_t& tj) {
  ti = u % tm, tj = u / tm;
  if constexpr (SYM) {
    tj = (uint32_t)((sqrtf(8.0f * u + 1.0f) - 1.0f) * 0.5f);
    while (tj * (tj + 1) / 2 > u) --tj;
    while ((tj + 1) * (tj + 2) / 2 <= u) ++tj;
    ti = u - tj * (tj + 1) / 2;
  }
}

// `whole` tiles, and the others in quarters.
template <int TILE, int WC, int KS, int ST, int KG, int END, class T>
__global__ void __launch_bounds__(128 * WC * KG) k_orth_gemm(OrthGemm g) {
  constexpr bool SYM = END == kEndGram || END == kEndPoly || END == kEndPart;
  extern __shared__ __attribute__((aligned(16))) half_t orth_gemm_lds[];
  // workgroups i, i + 8.. run on one XCD: it gets a contiguous part of the
  // tiles, whose columns and rows it then finds in its L2
  const uint32_t share = (g.whole + 7) / 8;
  uint32_t ti, tj;
  if (blockIdx.x < share * 8) {
    const uint32_t tile = blockIdx.x % 8 * share + blockIdx.x / 8;
    if (tile >= g.whole) return;
    orth_place<SYM>(tile % g.per, g.M / TILE, ti, tj);
    const uint32_t mat = tile / g.per;   // of the batch, once for each part
    orth_tile<TILE, WC, KS, ST, KG, END, T>(g, orth_gemm_lds, mat % g.batch, mat / g.batch, ti * TILE, tj * TILE);
  } else if constexpr (TILE > 64) {
    constexpr uint32_t HALF = TILE / 2;
    const uint32_t part = blockIdx.x - share * 8, tile = g.whole + part / 4;
    orth_place<SYM>(tile % g.per, g.M / TILE, ti, tj);
    ti = 2 * ti + part % 2, tj = 2 * tj + part / 2 % 2;
    if (SYM && ti > tj) return;
    orth_tile<HALF, WC, KS, ST, 1, END, T>(g, orth_gemm_lds, tile / g.per, 0, ti * HALF, tj * HALF);
  }
}

// A from the parts of its sum, added in their order.  A thread takes a value of
// the blocks on and above the diagonal, and its mirror image.
template <int KS>
__global__ void __launch_bounds__(256) k_orth_join(OrthGemm g) {
  const int64_t size = (int64_t)g.M * g.M, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= g.batch * size) return;
  const int64_t mat = i / size, row = i % size / g.M, col = i % g.M;
  if (row / 32 > col / 32) return;
  float v = 0.0f;
#pragma unroll 8
  for (int p = 0; p < g.parts; ++p) v += g.sums[p * (int64_t)g.batch * size + i];
  half_t hi, lo;
  split(g.f * v, hi, lo);
  half_t* C = g.c + mat * kPair * size;
  const int64_t at = orth_at<KS>(g.M, row, col), mirror = orth_at<KS>(g.M, col, row);
  C[at] = hi;
  C[size + at] = lo;
  if (row / 32 < col / 32) {
    C[mirror] = hi;
    C[size + mirror] = lo;
  }
}
