// The gated delta rule: a head's memory S [keys][values] forgets by a = exp(decay)
// and learns, with rate b, the error z between a value and what is read at its key:
//     P = a S,  z = v - P'k,  S <- P + b k z',  y = scale S'q.
//
// Chunks of C steps.  With G the sums of decays from the chunk's start, e = exp(G),
// D[i][j] = exp(G[i] - G[j]) for i >= j and 0 above, o = D's last row:
//     M = D o (K K') below the diagonal,  T = (I + M diag(b))^-1
//     Z = T (V - diag(e) K S)
//     Y = scale (diag(e) Q S + (D o (Q K')) diag(b) Z)
//     S <- e[C-1] S + K' diag(o b) Z
// k_delta_chunk computes T and the lower triangle of scale D o (Q K') diag(b) of
// every chunk, all at once; k_delta_scan goes through the chunks in order.  The
// columns of S (the values) never meet: a wavefront carries 16 of them through the
// whole sequence in registers, and the rows of one product's result, four to a
// lane, are the next product's operand as they are: an operand's lane wants eight
// values along the sum, which are its rows of two 16-row results, if the other
// operand's columns are dealt to lanes in the same order (order_of).  Only K, Q and
// the two triangles pass through LDS, for all wavefronts of a workgroup, laid out as
// the matrix instructions take them; K' is read from K's rows by LDS's transposing
// reads.  Four wavefronts of a workgroup compute and four feed them: they bring the
// next chunk's operands from memory to the other half of LDS and take results out.
//
// Arithmetic: 16-bit matrix instructions, 16 times as fast as 32-bit ones.  A
// 32-bit value is the sum of three bf16 parts (24 bits, and bf16 has float32's
// range), bf16 inputs are one part, and products of parts below 2^-24 of the result
// are left out: 3 products with an input, 6 between two 32-bit values.  So it is also for
// what passes into a bf16 result only (the second term of Y, and the state read by Q):
// with two parts, a read that cancels lost more than the result's own rounding.  The
// sums of decays are 64-bit: a difference of two of them is good where each is large.
//
// What bounds it.  The scan: a chunk's chain of dependent products.  2 x 16384 steps of
// 16 heads of 128 x 128 bf16, 32 heads on 64 workgroups: 890 us, 256 chunks of 3.5 us or
// 8400 cycles, of which matrix instructions take 3450 and the splitting of results
// into parts, which the wavefront cannot do beside them, most of the rest.  A chunk
// took 20 us with everything between two barriers, 6.7 with the next one's operands
// on their way, 5.4 with operands read ahead of their use, 3.0 with wavefronts that
// only feed and two parts of what only y sees, 3.5 with three.  Sums of two tiles in turn,
// splitting placed between matrix instructions, and orders of instructions given to the
// compiler changed nothing.  The chunks at once: memory, 8192 of them 165 us for 268 MB
// read and 308 MB of triangles written (250 us at two workgroups to a CU, with 254 MB).
#pragma once

#include <type_traits>
#include <utility>

#include "kernels_words.hpp"

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// Strides in values: between batch rows, steps, heads.
struct Walk {
  int64_t b, t, h;
};

struct DeltaArgs {
  int64_t batch, nchunk;
  int32_t steps, heads, group, dk, dv;   // group: heads that share a key head
  Walk q, k, v, y, decay, rate;
  const int32_t* lengths;
  float scale;
};

// A chunk's steps.  Products with the state take the same time for any length, those
// within a chunk grow with it, and the chain of chunks shrinks; the operands of two
// chunks of 64 steps in one part take 154 KB of LDS, of 32 steps in three parts 155.
template <class T>
constexpr int kChunk = sizeof(T) == 2 ? 64 : 32;
template <class T>
constexpr int kIn = sizeof(T) == 2 ? 1 : 3;    // parts of an input
constexpr int kState = 3;                      // of what is computed

// Eight values of an operand's row, as P parts.
template <int P>
struct Op {
  bf16x8 p[P];
};

template <int P>
__device__ __forceinline__ Op<P> op_of(const float (&x)[8]) {
  Op<P> o;
  float r[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) r[j] = x[j];
#pragma unroll
  for (int p = 0; p < P; ++p)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      o.p[p][j] = (__bf16)r[j];
      if (p + 1 < P) r[j] -= (float)o.p[p][j];
    }
  return o;
}

template <int P>
__device__ __forceinline__ Op<P> op_of(f32x4 a, f32x4 b) {
  const float x[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
  return op_of<P>(x);
}

// c + a b over the parts whose product is at least 2^(-8 (MAX - 1)) of the whole,
// the smallest first.
template <int MAX, int PA, int PB>
__device__ __forceinline__ f32x4 op_mul(const Op<PA>& a, const Op<PB>& b, f32x4 c) {
#pragma unroll
  for (int s = MAX - 1; s >= 0; --s)
#pragma unroll
    for (int i = 0; i < PA; ++i)
      if (s - i >= 0 && s - i < PB) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.p[i], b.p[s - i], c, 0, 0, 0);
  return c;
}

__device__ __forceinline__ f32x4 zero4() { return f32x4{0.0f, 0.0f, 0.0f, 0.0f}; }

// a x, and nothing of x where a is 0.
__device__ __forceinline__ float share_of(float a, float x) { return a == 0.0f ? 0.0f : a * x; }

// Eight values from p, n of them there (below 0: none), the others zeros.
template <class T, bool VEC>
__device__ __forceinline__ void load8(const T* p, int n, float (&x)[8]) {
  if constexpr (VEC) {
    if (n > 0) {
      constexpr int W = 16 / sizeof(T);
#pragma unroll
      for (int q = 0; q < 8; q += W) {
        const Words<T, W> w = *(const Words<T, W>*)(p + q);
#pragma unroll
        for (int j = 0; j < W; ++j) x[q + j] = as_f32(w.v[j]);
      }
      return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = 0.0f;
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = j < n ? as_f32(p[j]) : 0.0f;
  }
}

template <class T, bool VEC>
__device__ __forceinline__ Op<kIn<T>> op_load(const T* p, int n) {
  float x[8];
  load8<T, VEC>(p, n, x);
  return op_of<kIn<T>>(x);
}

// ---------------------------------------------------------------- triangles
// A triangle's 16 x 32 pieces that are not all zeros, by rows: of a lower one piece
// (mt, ks) with ks <= mt / 2, of an upper one its mirror image.
__host__ __device__ constexpr int tri_pieces(int C) { return C / 32 * (C / 32 + 1); }
template <int C, bool UPPER>
__device__ __forceinline__ constexpr int tri_piece(int mt, int ks) {
  const int m = UPPER ? C / 16 - 1 - mt : mt, k = UPPER ? C / 32 - 1 - ks : ks;
  return m / 2 * (m / 2 + 1) + m % 2 * (m / 2 + 1) + k;
}
template <int C, bool UPPER>
__device__ __forceinline__ constexpr bool tri_has(int mt, int ks) {
  return UPPER ? ks >= mt / 2 : ks <= mt / 2;
}

// What k_delta_chunk leaves of a chunk: T and the reads' triangle in three parts, each
// piece 64 x 16 bytes, then e, o and b.
template <int C>
struct ChunkWork {
  static constexpr int solve = 0, reads = kState * tri_pieces(C) * 1024, scales = 2 * reads, bytes = scales + 3 * C * 4;
};

// The pieces of a triangle in LDS (rows LD apart), as operands, to memory.
template <int C, int LD, bool UPPER, int P>
__device__ __forceinline__ void tri_store(const float* m, char* out, int tid, int threads) {
  for (int u = tid; u < C / 16 * (C / 32) * 64; u += threads) {
    const int lane = u % 64, ks = u / 64 % (C / 32), mt = u / 64 / (C / 32);
    if (!tri_has<C, UPPER>(mt, ks)) continue;
    const int i = mt * 16 + lane % 16, j = ks * 32 + lane / 16 * 4;
    float x[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      const int c = j + q % 4 + q / 4 * 16;
      x[q] = UPPER ? m[c * LD + i] : m[i * LD + c];
    }
    const Op<P> o = op_of<P>(x);
#pragma unroll
    for (int p = 0; p < P; ++p)
      *(bf16x8*)(out + ((p * tri_pieces(C) + tri_piece<C, UPPER>(mt, ks)) * 64 + lane) * 16) = o.p[p];
  }
}

// ------------------------------------------------------------------ operands
// Rows of 32 k values as operands in LDS, part by part: piece (rows / 16, k / 32) is
// 64 x 16 bytes, and lane m + 16 g's eight values, row m, k = 8 g .., lie at
// (m ^ 4 g) + 16 g: rows that are written or read together are in different banks.
__device__ __forceinline__ constexpr int lane_place(int m, int g) { return (m ^ 4 * g) + 16 * g; }

// A piece of `pieces`, at this lane's place `at`.
template <int P>
__device__ __forceinline__ Op<P> op_take(const char* lds, int pieces, int piece, int at) {
  Op<P> o;
#pragma unroll
  for (int p = 0; p < P; ++p) o.p[p] = *(const bf16x8*)(lds + ((p * pieces + piece) * 64 + at) * 16);
  return o;
}

// The transpose of such rows as an operand: 16 of the columns against 32 rows.  A
// transposing read takes 4 rows x 16 columns from 16 lanes, 8 bytes each (lane s: row
// s / 4, columns 4 (s % 4) ..), and gives lane i column i of them; the lanes of group
// g take rows 4 g .. and, by a second read, 16 + 4 g ...  Columns of a tile are either
// 16 in a row or (SPREAD) order_of: 4 of each of the four groups of 8.
template <bool SPREAD>
__device__ __forceinline__ int turn_place(int lane) {
  const int s = lane % 16, g = lane / 16, row = 4 * g + s / 4;
  return SPREAD ? lane_place(row, s % 4) * 16 : lane_place(row, s % 4 / 2) * 16 + s % 2 * 8;
}

// The two places above differ in the odd tile's: 8 bytes on, or two groups on.
template <bool SPREAD>
__device__ __forceinline__ int turn_odd(int lane) {
  if (SPREAD) return turn_place<true>(lane) + 8;
  const int s = lane % 16, g = lane / 16, row = 4 * g + s / 4;
  return lane_place(row, 2 + s % 4 / 2) * 16 + s % 2 * 8;
}

// KS: pieces to a row of pieces; tile: of 16 columns; step: 32 rows; even, odd: this
// lane's turn_place and turn_odd.
template <int P, int KS>
__device__ __forceinline__ Op<P> op_turn(const char* lds, int pieces, int tile, int step, int even, int odd) {
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) s16x4* From;
  Op<P> o;
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const char* at = lds + (p * pieces + 2 * step * KS + tile / 2) * 1024 + (tile % 2 ? odd : even);
    const bf16x4 a = __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((From)at)),
                 b = __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((From)(at + KS * 1024)));
    o.p[p] = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
  }
  return o;
}

// Row 4 g + r of the 16-row result m of a product over rows of SPREAD columns.
__device__ __forceinline__ int order_of(int m, int g, int r) { return m / 2 * 32 + g * 8 + m % 2 * 4 + r; }

// A chunk's rows of K or Q on their way from memory to LDS: in registers.  Four threads
// take 32 values of a row, the next four the next row: 16 of them write to all banks.
template <class T, bool VEC, int ROWS, int COLS, int THREADS>
struct RowsInFlight {
  static constexpr int N = ROWS * COLS / 8, U = (N + THREADS - 1) / THREADS, KS = COLS / 32;
  Words<T, 8> v[U];

  // n rows and dk columns are there, the others zeros.
  __device__ __forceinline__ void load(const T* x, int64_t stride, int n, int dk, int tid) {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int u = tid + i * THREADS, row = u / 4 % ROWS, d = u / (4 * ROWS) * 32 + u % 4 * 8;
      const bool there = row < n && d < dk;
      const T* from = x + (there ? row * stride + d : 0);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i].v[j] = (T)0.0f;
      if constexpr (VEC) {
        constexpr int W = 16 / sizeof(T);
        if (there)
#pragma unroll
          for (int q = 0; q < 8; q += W) *(Words<T, W>*)(v[i].v + q) = *(const Words<T, W>*)(from + q);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (there && d + j < dk) v[i].v[j] = from[j];
      }
    }
  }

  __device__ __forceinline__ void store(char* lds, int tid) const {
    constexpr int P = kIn<T>;
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int u = tid + i * THREADS, row = u / 4 % ROWS, c = u / (4 * ROWS) * 4 + u % 4;
      if (N % THREADS != 0 && u >= N) continue;
      float x[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = as_f32(v[i].v[j]);
      const Op<P> o = op_of<P>(x);
#pragma unroll
      for (int p = 0; p < P; ++p)
        *(bf16x8*)(lds + ((p * (ROWS / 16) * KS + row / 16 * KS + c / 4) * 64 + lane_place(row % 16, c % 4)) * 16) = o.p[p];
    }
  }
};

// A chunk's triangles and scales on their way, the same way.  (Loads straight to LDS
// make the compiler wait for them before any read of LDS: a chunk then took 6.5 us.)
template <int BYTES, int THREADS>
struct WorkInFlight {
  static constexpr int U = (BYTES / 16 + THREADS - 1) / THREADS;
  typedef uint32_t Raw __attribute__((ext_vector_type(4)));
  Raw v[U];

  __device__ __forceinline__ void load(const char* from, int tid) {
#pragma unroll
    for (int i = 0; i < U; ++i) v[i] = *(const Raw*)(from + min((tid + i * THREADS) * 16, BYTES - 16));
  }

  __device__ __forceinline__ void store(char* to, int tid) const {
#pragma unroll
    for (int i = 0; i < U; ++i)
      if (tid + i * THREADS < BYTES / 16) *(Raw*)(to + (tid + i * THREADS) * 16) = v[i];
  }
};

// Operands 0 .. N - 1, read from LDS D ahead of their use: a read takes as long as
// eight matrix instructions, and left to itself the compiler waits for each.
template <int N, int D, class B, class F>
struct Ahead {
  B b[D + 1];
  F load;

  __device__ __forceinline__ explicit Ahead(F f) : load(f) {
#pragma unroll
    for (int i = 0; i < D && i < N; ++i) b[i] = load(i);
    __builtin_amdgcn_sched_barrier(0);
  }

  __device__ __forceinline__ const B& operator()(int i) {
    if (i + D < N) b[(i + D) % (D + 1)] = load(i + D);
    __builtin_amdgcn_sched_barrier(0);
    return b[i % (D + 1)];
  }
};

template <int N, int D, class F>
__device__ __forceinline__ auto ahead_of(F f) {
  return Ahead<N, D, decltype(f(0)), F>(f);
}

// The triangle's piece i of those that are there, by rows.
template <int C, bool UPPER>
__device__ __forceinline__ constexpr int tri_row(int i) {
  int m = 0;
  for (int n = 0; m < C / 16; ++m) {
    const int here = UPPER ? C / 32 - m / 2 : m / 2 + 1;
    if (i < n + here) break;
    n += here;
  }
  return m;
}
template <int C, bool UPPER>
__device__ __forceinline__ constexpr int tri_column(int i) {
  int n = 0;
  for (int m = 0; m < C / 16; ++m) {
    const int here = UPPER ? C / 32 - m / 2 : m / 2 + 1;
    if (i < n + here) break;
    n += here;
  }
  return i - n + (UPPER ? tri_row<C, UPPER>(i) / 2 : 0);
}

// Where the upper triangle's piece i, by rows, lies: as the mirror image's, from the end.
template <int C>
__device__ __forceinline__ constexpr int tri_upper(int i) {
  return tri_pieces(C) - 1 - i;
}

// f(0) .. f(N - 1), each with its number as a compile-time value.
template <class F, int... I>
__device__ __forceinline__ void each_of(F&& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class F>
__device__ __forceinline__ void each(F&& f) {
  each_of(f, std::make_integer_sequence<int, N>{});
}

template <int A, int B>
struct OpPair {
  Op<A> a;
  Op<B> b;
};

// ----------------------------------------------------------- chunks, all at once
// T and the reads' triangle of every chunk.  GRAD: their transposes, the second one
// without b.  A wavefront computes 16 rows of K K' and Q K'; the inverse of the
// diagonal blocks of 16 goes column by column, a lane each, and blocks double by
// [[A, 0], [B, C]]^-1 = [[A', 0], [-C' B A', C']] on 32-bit matrix instructions.
template <class T, bool VEC, int DK, bool GRAD>
__global__ void __launch_bounds__(kChunk<T> * 4, sizeof(T) == 2 ? 4 : 3)
    k_delta_chunk(DeltaArgs p, const T* q, const T* k, const float* decay, const float* rate, char* work) {
  constexpr int C = kChunk<T>, LD = C + 4, KS = DK / 32, PI = kIn<T>, RP = C / 16 * KS;
  using Work = ChunkWork<C>;
  constexpr int ROWS = PI * C * DK * 2, BOTH = 2 * C * LD * 4;
  __shared__ __align__(16) char lds[ROWS > BOTH ? ROWS : BOTH];   // K's rows; then the two triangles
  float *const m = (float*)lds, *const t = m + C * LD;
  __shared__ double sum[C];
  __shared__ float rates[C];
  const int tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64), g = lane / 16;
  const int at = lane_place(lane % 16, g);
  const int64_t all = p.batch * p.heads * p.nchunk;
  for (int64_t u = blockIdx.x; u < all; u += gridDim.x) {
    const int64_t chunk = u % p.nchunk, b = u / p.nchunk / p.heads;
    const int head = (int)(u / p.nchunk % p.heads), kh = head / p.group;
    const int64_t t0 = chunk * C;
    const int len = p.lengths ? min(max(p.lengths[b], 0), p.steps) : p.steps;
    const int n = (int)min((int64_t)C, len - t0);   // steps of this chunk that count
    if (n <= 0) continue;                           // nothing reads it
    char* out = work + u * Work::bytes;
    RowsInFlight<T, VEC, C, DK, C * 4> kr;
    kr.load(k + b * p.k.b + t0 * p.k.t + kh * p.k.h, p.k.t, n, p.dk, tid);
    Op<PI> qa[KS];
    {
      const int i = wave * 16 + lane % 16;
      const T* qb = q + b * p.q.b + t0 * p.q.t + kh * p.q.h;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const int d = ks * 32 + g * 8, there = i < n ? p.dk - d : 0;
        qa[ks] = op_load<T, VEC>(qb + (there > 0 ? i * p.q.t + d : 0), there);
      }
    }
    if (tid < C) {
      double d = 0.0;
      float r = 0.0f;
      if (tid < n) {
        const float x = decay[b * p.decay.b + (t0 + tid) * p.decay.t + head * p.decay.h];
        d = x < -200.0f ? -200.0 : (double)x;   // exp is 0 in 32 bits long before
        r = rate[b * p.rate.b + (t0 + tid) * p.rate.t + head * p.rate.h];
      }
#pragma unroll
      for (int o = 1; o < C; o *= 2) {
        const double x = __shfl_up(d, o, 64);
        if (tid >= o) d += x;
      }
      d *= 1.4426950408889634;
      const double end = __shfl(d, C - 1, 64);
      sum[tid] = d;
      rates[tid] = r;
      float* s = (float*)(out + Work::scales);
      s[tid] = __builtin_amdgcn_exp2f((float)d);
      s[C + tid] = __builtin_amdgcn_exp2f((float)(end - d));
      s[2 * C + tid] = r;
    }
    kr.store(lds, tid);
    __syncthreads();
    // rows 16 wave .. of K K' and Q K'
    f32x4 kk[C / 16], qk[C / 16];
    {
      Op<PI> ka[KS];
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) ka[ks] = op_take<PI>(lds, RP, wave * KS + ks, at);
#pragma unroll
      for (int ct = 0; ct < C / 16; ++ct) {
        kk[ct] = qk[ct] = zero4();
        if (ct > wave) continue;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const Op<PI> kb = op_take<PI>(lds, RP, ct * KS + ks, at);
          kk[ct] = op_mul<PI>(ka[ks], kb, kk[ct]);
          qk[ct] = op_mul<PI>(qa[ks], kb, qk[ct]);
        }
      }
    }
    __syncthreads();
#pragma unroll
    for (int ct = 0; ct < C / 16; ++ct)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int i = wave * 16 + g * 4 + r, j = ct * 16 + lane % 16;
        float d = 0.0f, x = 0.0f;
        if (ct <= wave) {
          d = i >= j ? __builtin_amdgcn_exp2f((float)(sum[i] - sum[j])) : 0.0f;
          x = i > j ? kk[ct][r] * d * rates[j] : 0.0f;
          qk[ct][r] *= d * p.scale * (GRAD ? 1.0f : rates[j]);
        }
        m[i * LD + j] = x;
        t[i * LD + j] = 0.0f;
      }
    __syncthreads();
    if (tid < C) {
      const int d0 = tid / 16 * 16, c = tid % 16;
      float x[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        float s = i == c ? 1.0f : 0.0f;
#pragma unroll
        for (int j = 0; j < i; ++j) s = fmaf(-m[(d0 + i) * LD + d0 + j], x[j], s);
        x[i] = s;
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) t[(d0 + i) * LD + d0 + c] = x[i];
    }
    __syncthreads();
#pragma unroll
    for (int size = 16; size < C; size *= 2) {
      // B A', in the place of B, and then -C' of it; a tile of 16 x 16 to a wavefront
      const int side = size / 16, per = side * side, tiles = C / (2 * size) * per;
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        f32x4 c = zero4();
        int r0 = 0, c0 = 0;
        if (wave < tiles) {
          const int pair = wave / per * 2 * size;
          r0 = pair + size + wave % per / side * 16, c0 = pair + wave % side * 16;
          for (int x = 0; x < size; x += 4) {
            const float a = half ? t[(r0 + lane % 16) * LD + pair + size + x + g] : m[(r0 + lane % 16) * LD + pair + x + g];
            const float v = half ? m[(pair + size + x + g) * LD + c0 + lane % 16] : t[(pair + x + g) * LD + c0 + lane % 16];
            c = __builtin_amdgcn_mfma_f32_16x16x4f32(a, v, c, 0, 0, 0);
          }
        }
        __syncthreads();
        if (wave < tiles)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            if (half) t[(r0 + g * 4 + r) * LD + c0 + lane % 16] = -c[r];
            else m[(r0 + g * 4 + r) * LD + c0 + lane % 16] = c[r];
          }
        __syncthreads();
      }
    }
    tri_store<C, LD, GRAD, kState>(t, out + Work::solve, tid, C * 4);
#pragma unroll
    for (int ct = 0; ct < C / 16; ++ct)
#pragma unroll
      for (int r = 0; r < 4; ++r) m[(wave * 16 + g * 4 + r) * LD + ct * 16 + lane % 16] = qk[ct][r];
    __syncthreads();
    tri_store<C, LD, GRAD, kState>(m, out + Work::reads, tid, C * 4);
    __syncthreads();
  }
}

// ---------------------------------------------------------------- chunks in order
// 64 columns of a chunk of V, Y or dY in LDS.  16 bits: V and dY by steps, Y by
// columns, 128 bytes a row, its 16-byte words mixed by the row so that transposing
// reads and writes of columns meet different banks; 32 bits: by steps, 68 values apart.
template <class T>
struct Panel {
  static constexpr int C = kChunk<T>, bytes = sizeof(T) == 2 ? 64 * 128 : C * 68 * 4;
  static __device__ __forceinline__ int at(int row, int i) {   // 16 bits: value i of a row
    return row * 128 + (i / 8 ^ row % 8) * 16 + i % 8 * 2;
  }
};

// 64 columns of V or dY on their way there, by 256 threads; n steps and `there`
// columns are there, the others zeros.
template <class T, bool VEC>
struct PanelInFlight {
  static constexpr int C = kChunk<T>, U = C * 8 / 256;
  Words<T, 8> v[U];

  __device__ __forceinline__ void load(const T* x, int32_t stride, int n, int there, int tid) {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int row = tid / 8 + i * 32, c = tid % 8 * 8;
      const bool some = row < n && c < there;
      const T* from = x + (some ? (int64_t)(uint32_t)(row * stride) + c : 0);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i].v[j] = (T)0.0f;
      if constexpr (VEC) {
        constexpr int W = 16 / sizeof(T);
        if (some)
#pragma unroll
          for (int q = 0; q < 8; q += W) *(Words<T, W>*)(v[i].v + q) = *(const Words<T, W>*)(from + q);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (some && c + j < there) v[i].v[j] = from[j];
      }
    }
  }

  __device__ __forceinline__ void store(char* lds, int tid) const {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int row = tid / 8 + i * 32, c = tid % 8 * 8;
      if constexpr (sizeof(T) == 2) {
        *(Words<T, 8>*)(lds + Panel<T>::at(row, c)) = v[i];
      } else {
        *(Words<T, 4>*)(lds + (row * 68 + c) * 4) = *(const Words<T, 4>*)v[i].v;
        *(Words<T, 4>*)(lds + (row * 68 + c + 4) * 4) = *(const Words<T, 4>*)(v[i].v + 4);
      }
    }
  }
};

// This wavefront's 16 columns (of tile `wave`) as results' registers: row 4 g + r of
// result m is step 16 m + 4 g + r.
template <class T>
__device__ __forceinline__ void panel_take(const char* lds, int wave, int lane, f32x4 (&z)[kChunk<T> / 16]) {
  const int g = lane / 16;
#pragma unroll
  for (int m = 0; m < kChunk<T> / 16; ++m) {
    if constexpr (sizeof(T) == 2) {
      typedef short s16x4 __attribute__((ext_vector_type(4)));
      typedef __attribute__((address_space(3))) s16x4* From;
      const char* from = lds + Panel<T>::at(m * 16 + g * 4 + lane % 16 / 4, wave * 16 + lane % 4 * 4);
      const bf16x4 h = __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((From)from));
#pragma unroll
      for (int r = 0; r < 4; ++r) z[m][r] = (float)h[r];
    } else {
#pragma unroll
      for (int r = 0; r < 4; ++r) z[m][r] = *(const float*)(lds + ((m * 16 + g * 4 + r) * 68 + wave * 16 + lane % 16) * 4);
    }
  }
}

template <class T>
__device__ __forceinline__ void panel_put(char* lds, int wave, int lane, const f32x4 (&o)[kChunk<T> / 16]) {
  const int g = lane / 16;
#pragma unroll
  for (int m = 0; m < kChunk<T> / 16; ++m) {
    if constexpr (sizeof(T) == 2) {
      *(bf16x4*)(lds + Panel<T>::at(wave * 16 + lane % 16, m * 16 + g * 4)) =
          bf16x4{(__bf16)o[m][0], (__bf16)o[m][1], (__bf16)o[m][2], (__bf16)o[m][3]};
    } else {
#pragma unroll
      for (int r = 0; r < 4; ++r) *(float*)(lds + ((m * 16 + g * 4 + r) * 68 + wave * 16 + lane % 16) * 4) = o[m][r];
    }
  }
}

// What panel_put left, to memory, by 256 threads.
template <class T, bool VEC>
__device__ __forceinline__ void panel_out(const char* lds, T* y, int32_t stride, int n, int there, int tid) {
  constexpr int C = kChunk<T>;
#pragma unroll
  for (int i = 0; i < C * 8 / 256; ++i) {
    Words<T, 8> w;
    int t, c;
    if constexpr (sizeof(T) == 2) {
      typedef short s16x4 __attribute__((ext_vector_type(4)));
      typedef __attribute__((address_space(3))) s16x4* From;
      const int group = tid / 16 + i * 16, s = tid % 16;
      c = group % 8 * 8, t = group / 8 * 16;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const char* from = lds + Panel<T>::at(c + h * 4 + s / 4, t + s % 4 * 4);
        *(s16x4*)(w.v + h * 4) = __builtin_amdgcn_ds_read_tr16_b64_v4i16((From)from);
      }
      t += s;
    } else {
      t = tid / 8 + i * 32, c = tid % 8 * 8;
      *(Words<T, 4>*)w.v = *(const Words<T, 4>*)(lds + (t * 68 + c) * 4);
      *(Words<T, 4>*)(w.v + 4) = *(const Words<T, 4>*)(lds + (t * 68 + c + 4) * 4);
    }
    if (t >= n || c >= there) continue;
    T* to = y + (int64_t)(uint32_t)(t * stride) + c;
    if constexpr (VEC) {
      constexpr int W = 16 / sizeof(T);
#pragma unroll
      for (int q = 0; q < 8; q += W) *(Words<T, W>*)(to + q) = *(const Words<T, W>*)(w.v + q);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (c + j < there) to[j] = w.v[j];
    }
  }
}

// One of the two halves of a scan's LDS: rows of K and of Q, the chunk's triangles and
// scales; behind them panels of V or dY, and of Y.  PAIRS: two of each panel, one for
// each half; chunks of 64 steps of 128 keys leave room for one, and pay for it with a
// barrier more.
template <class T, int DK, bool GRAD>
struct ScanLds {
  static constexpr int C = kChunk<T>, each = Panel<T>::bytes;
  static constexpr int k = 0, q = kIn<T> * C * DK * 2, work = 2 * q, bytes = work + ChunkWork<C>::bytes, panel = 2 * bytes;
  static constexpr bool PAIRS = GRAD || panel + 4 * each <= 160 * 1024;
  static constexpr int out = panel + (PAIRS ? 2 : 1) * each, all = out + (GRAD ? 0 : out - panel);
  static __device__ __forceinline__ int panel_of(int chunk) { return PAIRS ? panel + (chunk & 1) * each : panel; }
  static __device__ __forceinline__ int out_of(int chunk) { return PAIRS ? out + (chunk & 1) * each : out; }
};

// A chunk's operands on their way from memory to one half, by 256 threads.
template <class T, bool VEC, int DK, bool GRAD>
struct ChunkInFlight {
  using Lds = ScanLds<T, DK, GRAD>;
  static constexpr int C = Lds::C, BYTES = ChunkWork<C>::bytes;
  RowsInFlight<T, VEC, C, DK, 256> k, q;
  WorkInFlight<BYTES, 256> w;
  PanelInFlight<T, VEC> x;

  // all but the panel
  __device__ __forceinline__ void load(const DeltaArgs& p, const T* kp, const T* qp, const char* wp, int64_t chunk, int n,
                                       int tid) {
    const int64_t t0 = chunk * C;
    w.load(wp + chunk * BYTES, tid);
    k.load(kp + t0 * p.k.t, p.k.t, n, p.dk, tid);
    q.load(qp + t0 * p.q.t, p.q.t, n, p.dk, tid);
  }

  __device__ __forceinline__ void store(char* half, int tid) const {
    w.store(half + Lds::work, tid);
    k.store(half + Lds::k, tid);
    q.store(half + Lds::q, tid);
  }
};

// Batch row, head and block of columns of a workgroup: the blocks of a head are 8
// apart, on one of the 8 dies, whose L2 then reads the head's K, Q and triangles once.
__device__ __forceinline__ bool scan_place(const DeltaArgs& p, int blocks, int64_t& bh, int& block) {
  const int64_t x = blockIdx.x;
  bh = x / (8 * blocks) * 8 + x % 8;
  block = (int)(x / 8 % blocks);
  return bh < p.batch * p.heads;
}

// What the passes leave for k_delta_grad of a chunk: its state, or the state's
// gradient, [columns][keys], and Z or X, [columns][C]: a column's values side by side,
// as a lane has them, columns padded to 32 (zeros) and keys to 8.
__host__ __device__ constexpr int pad_keys(int dk) { return (dk + 7) / 8 * 8; }
__host__ __device__ constexpr int pad_columns(int dv) { return (dv + 31) / 32 * 32; }

template <int DK>
__device__ __forceinline__ void put_state(float* x, int dk, int col, int g, const f32x4 (&s)[DK / 16]) {
  const int kp = pad_keys(dk);
  float* const at = x + (uint32_t)(col * kp + g * 8);
#pragma unroll
  for (int m = 0; m < DK / 16; ++m)
    if (order_of(m, g, 0) < kp) *(f32x4*)(at + order_of(m, 0, 0)) = s[m];
}

template <int C>
__device__ __forceinline__ void put_rows(float* x, int col, int g, const f32x4 (&z)[C / 16]) {
  float* const at = x + (uint32_t)(col * C + g * 4);
#pragma unroll
  for (int m = 0; m < C / 16; ++m) *(f32x4*)(at + m * 16) = z[m];
}

// The chunks of a head in order, 64 columns to a workgroup (grid: see scan_place) and
// 16 to a computing wavefront.
// KEEP: S before each chunk to `states` and Z to `errors`, for the gradient.
template <class T, bool VEC, int DK, bool KEEP>
__global__ void __launch_bounds__(512, 1)
    k_delta_scan(DeltaArgs p, int blocks, const T* q, const T* k, const T* v, const float* decay, const float* s0,
                 const char* work, T* y, float* last, float* states, float* errors) {
  using Lds = ScanLds<T, DK, false>;
  constexpr int C = Lds::C, KS = DK / 32, PI = kIn<T>, RP = C / 16 * KS;
  using Work = ChunkWork<C>;
  extern __shared__ __align__(16) char lds[];
  int64_t bh;
  int block;
  if (!scan_place(p, blocks, bh, block)) return;
  const int64_t b = bh / p.heads;
  const int head = (int)(bh % p.heads), kh = head / p.group, first = block * 64;
  const int len = p.lengths ? min(max(p.lengths[b], 0), p.steps) : p.steps;
  const int chunks = len / C + (len % C != 0);
  if (threadIdx.x >= 256) {   // feeds
    const int tid = threadIdx.x - 256, there = p.dv - first;
    const T *kp = k + b * p.k.b + kh * p.k.h, *qp = q + b * p.q.b + kh * p.q.h, *vp = v + b * p.v.b + head * p.v.h + first;
    T* const yp = y + b * p.y.b + head * p.y.h + first;
    const char* wp = work + bh * p.nchunk * Work::bytes;
    ChunkInFlight<T, VEC, DK, false> f;
    const auto load = [&](int chunk) { f.load(p, kp, qp, wp, chunk, min(C, len - chunk * C), tid); };
    const auto load_panel = [&](int chunk) {
      f.x.load(vp + (int64_t)chunk * C * p.v.t, (int32_t)p.v.t, min(C, len - chunk * C), there, tid);
    };
    const auto store = [&](int chunk) { f.store(lds + (chunk & 1) * Lds::bytes, tid); };
    const auto store_panel = [&](int chunk) { f.x.store(lds + Lds::panel_of(chunk), tid); };
    const auto out = [&](int chunk) {
      panel_out<T, VEC>(lds + Lds::out_of(chunk), yp + (int64_t)chunk * C * p.y.t, (int32_t)p.y.t, min(C, len - chunk * C),
                        there, tid);
    };
    if (chunks > 0) load(0), load_panel(0), store(0), store_panel(0);
    if (chunks > 1) load(1), load_panel(1);
    for (int64_t t = len + tid / 64; t < p.steps; t += 4)
      if (tid % 64 < there) yp[t * p.y.t + tid % 64] = (T)0.0f;
    for (int chunk = 0; chunk < chunks; ++chunk) {
      const bool next = chunk + 1 < chunks, after = chunk + 2 < chunks;
      __syncthreads();   // this chunk's operands are there, the other half is read and the last results are written
      if constexpr (Lds::PAIRS) {
        if (next) store(chunk + 1), store_panel(chunk + 1);
        if (after) load(chunk + 2), load_panel(chunk + 2);
        if (chunk > 0) out(chunk - 1);
      } else {
        if (chunk > 0) out(chunk - 1);
        if (next) store(chunk + 1);
        if (after) load(chunk + 2);
        __syncthreads();   // V is read, and the last results are out
        if (next) store_panel(chunk + 1);
        if (after) load_panel(chunk + 2);
      }
    }
    __syncthreads();
    if (chunks > 0) out(chunks - 1);
    return;
  }
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, g = lane / 16, at = lane_place(lane % 16, g);
  const int even = turn_place<true>(lane), odd = turn_odd<true>(lane);
  const int tile = first + wave * 16, col = tile + lane % 16;
  const bool mine = col < p.dv, some = tile < (KEEP ? pad_columns(p.dv) : p.dv);
  f32x4 s[DK / 16];
  // where the first step forgets, what s0 holds does not count
  const bool fresh = !s0 || (len > 0 && decay[b * p.decay.b + head * p.decay.h] < -200.0f);
#pragma unroll
  for (int m = 0; m < DK / 16; ++m)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int d = order_of(m, g, r);
      s[m][r] = !fresh && mine && d < p.dk ? s0[(bh * p.dk + d) * p.dv + col] : 0.0f;
    }
  for (int chunk = 0; chunk < chunks; ++chunk) {
    const char* const here = lds + (chunk & 1) * Lds::bytes;
    __syncthreads();
    if (!some) {
      if (!Lds::PAIRS) __syncthreads();
      continue;
    }
    if (KEEP) put_state<DK>(states + (bh * p.nchunk + chunk) * pad_keys(p.dk) * pad_columns(p.dv), p.dk, col, g, s);
    constexpr int TRI = tri_pieces(C), NEAR = sizeof(T) == 2 ? 3 : 1;   // 5 products to a pair, or 12
    const char* const tri = here + Lds::work;
    const float* e = (const float*)(tri + Work::scales);
    auto kq = ahead_of<RP, NEAR>([&](int i) {
      return OpPair<PI, PI>{op_take<PI>(here + Lds::k, RP, i, at), op_take<PI>(here + Lds::q, RP, i, at)};
    });
    f32x4 z[C / 16], o[C / 16];
    panel_take<T>(lds + Lds::panel_of(chunk), wave, lane, z);
    Op<kState> sp[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) sp[ks] = op_of<kState>(s[2 * ks], s[2 * ks + 1]);
#pragma unroll
    for (int m = 0; m < C / 16; ++m) {
      f32x4 c = zero4(), w = zero4();
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const auto& x = kq(m * KS + ks);
        c = op_mul<kState>(x.a, sp[ks], c);
        w = op_mul<kState>(x.b, sp[ks], w);
      }
      const f32x4 em = *(const f32x4*)(e + m * 16 + g * 4);
#pragma unroll
      for (int r = 0; r < 4; ++r) z[m][r] = fmaf(-em[r], c[r], z[m][r]), o[m][r] = em[r] * p.scale * w[r];
    }
    auto solve = ahead_of<TRI, 2>([&](int i) { return op_take<kState>(tri + Work::solve, TRI, i, lane); });
    Op<kState> zp[C / 32];
#pragma unroll
    for (int ks = 0; ks < C / 32; ++ks) zp[ks] = op_of<kState>(z[2 * ks], z[2 * ks + 1]);
#pragma unroll
    for (int m = 0; m < C / 16; ++m) z[m] = zero4();
    each<TRI>([&](auto i) {
      constexpr int m = tri_row<C, false>(i), ks = tri_column<C, false>(i);
      z[m] = op_mul<kState>(solve(i), zp[ks], z[m]);
    });
    if (KEEP) put_rows<C>(errors + (bh * p.nchunk + chunk) * C * pad_columns(p.dv), col, g, z);
    auto reads = ahead_of<TRI, 3>([&](int i) { return op_take<kState>(tri + Work::reads, TRI, i, lane); });
#pragma unroll
    for (int ks = 0; ks < C / 32; ++ks) zp[ks] = op_of<kState>(z[2 * ks], z[2 * ks + 1]);
    each<TRI>([&](auto i) {
      constexpr int m = tri_row<C, false>(i), ks = tri_column<C, false>(i);
      o[m] = op_mul<kState>(reads(i), zp[ks], o[m]);
    });
    if (!Lds::PAIRS) __syncthreads();   // V is read, and the last results are out
    auto turned = ahead_of<RP, NEAR + 1>(
        [&](int i) { return op_turn<PI, KS>(here + Lds::k, RP, i / (C / 32), i % (C / 32), even, odd); });
    panel_put<T>(lds + Lds::out_of(chunk), wave, lane, o);
#pragma unroll
    for (int m = 0; m < C / 16; ++m) {
      const f32x4 om = *(const f32x4*)(e + C + m * 16 + g * 4), bm = *(const f32x4*)(e + 2 * C + m * 16 + g * 4);
#pragma unroll
      for (int r = 0; r < 4; ++r) z[m][r] *= om[r] * bm[r];
    }
#pragma unroll
    for (int ks = 0; ks < C / 32; ++ks) zp[ks] = op_of<kState>(z[2 * ks], z[2 * ks + 1]);
    const float keep = e[C - 1];
#pragma unroll
    for (int m = 0; m < DK / 16; ++m) {
      s[m] *= keep;
#pragma unroll
      for (int ks = 0; ks < C / 32; ++ks) s[m] = op_mul<kState>(turned(m * (C / 32) + ks), zp[ks], s[m]);
    }
  }
  __syncthreads();
  if (last && mine)
#pragma unroll
    for (int m = 0; m < DK / 16; ++m)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int d = order_of(m, g, r);
        if (d < p.dk) last[(bh * p.dk + d) * p.dv + col] = s[m][r];
      }
}

// ---------------------------------------------------------------- single step
struct DeltaStepArgs {
  int64_t rows, slots, state;   // state: between slots
  int32_t heads, group, dk, dv;
  int64_t q[2], k[2], v[2], y[2], decay[2], rate[2];   // between rows, between heads
  float scale;
};

constexpr int kStepRows = 16;   // of a matrix to a thread, at most

// One step of a row's head: P'k and P'q are sums over the keys of one read of the
// matrix, which stays in registers, y = scale (P'q + b z (k'q)).  `nl` threads (a
// power of two, at most 32) take V columns each, the others of 256 further keys.
// Memory bounds it: 112 served rows of 32 heads of 128 x 128, 470 MB read and written,
// 86 us, 5.5 TB/s (v read ahead of the barriers instead of y written behind them: 3 us
// more).  8 rows of 4 heads of 64 x 64: 7 us; the call's 14 us are the host's time.
template <class T, int V>
__global__ void __launch_bounds__(256) k_delta_step(DeltaStepArgs p, int32_t nl, int32_t tiles, const T* q, const T* k,
                                                    const T* v, const float* decay, const float* rate, float* state,
                                                    const int32_t* slots, T* y) {
  __shared__ float kq[2][128];
  __shared__ float red[2][256 / 4 * 4][V];   // sums of up to 64 groups of columns and 4 wavefronts
  __shared__ float dots[4];
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64, groups = 256 / nl, rg = tid / nl;
  const int64_t all = p.rows * p.heads * tiles;
  for (int64_t u = blockIdx.x; u < all; u += gridDim.x) {
    const int64_t i = u / tiles / p.heads;
    const int head = (int)(u / tiles % p.heads), kh = head / p.group;
    const int c = ((int)(u % tiles) * nl + tid % nl) * V;
    const bool mine = c < p.dv;
    const int64_t slot = slots ? (int64_t)slots[i] : i;
    if (slot < 0 || slot >= p.slots) {   // idle
      if (mine && rg == 0)
#pragma unroll
        for (int e = 0; e < V; ++e) y[i * p.y[0] + head * p.y[1] + c + e] = (T)0.0f;
      continue;
    }
    float* s = state + slot * p.state + (int64_t)head * p.dk * p.dv + c;
    Words<float, V> m[kStepRows];
#pragma unroll
    for (int r = 0; r < kStepRows; ++r) {
      const int d = rg + r * groups;
#pragma unroll
      for (int e = 0; e < V; ++e) m[r].v[e] = 0.0f;
      if (mine && d < p.dk) m[r] = *(const Words<float, V>*)(s + (int64_t)d * p.dv);
    }
    float kd = 0.0f, qd = 0.0f;
    if (tid < 128 && tid < p.dk) {
      kd = as_f32(k[i * p.k[0] + kh * p.k[1] + tid]);
      qd = as_f32(q[i * p.q[0] + kh * p.q[1] + tid]);
    }
    if (tid < 128) kq[0][tid] = kd, kq[1][tid] = qd;
    float dot = kd * qd;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) dot += __shfl_xor(dot, o, 64);
    if (lane == 0) dots[wave] = dot;
    const float a = expf(decay[i * p.decay[0] + head * p.decay[1]]);
    const float b = rate[i * p.rate[0] + head * p.rate[1]];
    __syncthreads();
    dot = dots[0] + dots[1];
    float w[V], o[V];
#pragma unroll
    for (int e = 0; e < V; ++e) w[e] = o[e] = 0.0f;
#pragma unroll
    for (int r = 0; r < kStepRows; ++r) {
      const int d = rg + r * groups;
      const float kr = d < 128 ? kq[0][d] : 0.0f, qr = d < 128 ? kq[1][d] : 0.0f;
#pragma unroll
      for (int e = 0; e < V; ++e) {
        m[r].v[e] = share_of(a, m[r].v[e]);
        w[e] = fmaf(m[r].v[e], kr, w[e]);
        o[e] = fmaf(m[r].v[e], qr, o[e]);
      }
    }
    for (int x = nl; x < 64; x *= 2)
#pragma unroll
      for (int e = 0; e < V; ++e) w[e] += __shfl_xor(w[e], x, 64), o[e] += __shfl_xor(o[e], x, 64);
    if (lane < nl)
#pragma unroll
      for (int e = 0; e < V; ++e) red[0][wave * nl + lane][e] = w[e], red[1][wave * nl + lane][e] = o[e];
    __syncthreads();
#pragma unroll
    for (int e = 0; e < V; ++e) {
      w[e] = o[e] = 0.0f;
#pragma unroll
      for (int x = 0; x < 4; ++x) w[e] += red[0][x * nl + tid % nl][e], o[e] += red[1][x * nl + tid % nl][e];
    }
    if (mine) {
      float z[V];
#pragma unroll
      for (int e = 0; e < V; ++e) {
        z[e] = b * (as_f32(v[i * p.v[0] + head * p.v[1] + c + e]) - w[e]);
        o[e] = p.scale * fmaf(z[e], dot, o[e]);
      }
#pragma unroll
      for (int r = 0; r < kStepRows; ++r) {
        const int d = rg + r * groups;
        if (d >= p.dk) continue;
        const float kr = kq[0][d];
#pragma unroll
        for (int e = 0; e < V; ++e) m[r].v[e] = fmaf(kr, z[e], m[r].v[e]);
        *(Words<float, V>*)(s + (int64_t)d * p.dv) = m[r];
      }
    }
    __syncthreads();   // kq, red and dots are free again, and all have read v, in whose place y may lie
    if (mine && rg == 0)
#pragma unroll
      for (int e = 0; e < V; ++e) y[i * p.y[0] + head * p.y[1] + c + e] = (T)o[e];
  }
}
