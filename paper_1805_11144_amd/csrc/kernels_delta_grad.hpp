// The gradient of the gated delta rule (kernels_delta.hpp has the rule, the chunks
// and the operands).
//
// From the states S before each chunk and the errors Z that the forward pass left.
// With H[t] the gradient of the state after step t, x = b H'k is the gradient of v
// and the state before step t gets a (H - k x').  In a chunk, with dS the gradient of
// the state behind it:
//     X = T' diag(b) (diag(o) K dS + scale (D o (Q K'))' dY)
//     dS <- e[C-1] dS + Q' diag(scale e) dY - K' diag(e) X
// k_delta_back goes through the chunks in reverse order like k_delta_scan, 16 columns
// to a wavefront, and leaves X and each chunk's dS.  k_delta_grad computes the rest
// for all chunks at once, sums over the values, and writes X out as dV:
//     dQ[s] = scale (e[s] S dy[s] + sum_{t <= s} D[s][t] b[t] k[t] (z[t] dy[s]))
//     W[t]  = o[t] dS z[t] + sum_{s >= t} D[s][t] scale q[s] (dy[s] z[t])
//                          - sum_{s > t} D[s][t] k[s] (x[s] z[t])                (H z)
//     R[t]  = e[t] S x[t] + sum_{s < t} D[t][s] b[s] k[s] (z[s] x[t])            (P x)
//     dK = b W - R,   drate = k W
// The decays: G[t] scales what t reads and undoes what it writes, so that
//     dG[t] = q dQ - k R - b (k W),  and behind the last step <dS, S behind the chunk>,
// and decay[t] is in all G from t on: a sum from the chunk's end, or from the next step
// whose a is 0 in 32 bits.  What lies from there on cancels in it, but only to the
// rounding of its own size, which may be any number of times what is before.
//
// Everything here takes three parts, also for bf16 results: the gates' gradients are 32
// bits and differences of the same products.
//
// Measured, 8 x 2048 steps of 16 heads of 128 x 128 bf16, 4096 chunks: k_delta_back 190
// to 206 us (the scan 215 to 230); k_delta_grad 430 to 490.  It has to read 980 MB (states and
// their gradients, 32 bits each, are most), 210 us at a copy's rate; the matrix
// instructions take 12900 cycles of a chunk, 90 us.  Of a chunk's 62000 cycles (before
// the last step) a computing wavefront spent 24000 on sums over the values, 11200 on the
// products' scaling and 5400 on the last products, while nothing is fed, and 14600 in
// waiting for values.  Step by step: 1290 us with everything in one group of
// wavefronts, 880 with the four products computed once a workgroup, 500 with
// wavefronts that feed and go on to the next chunk, 440 with the decays between steps
// without branches.  Two sets of values on their way need more registers than there
// are: 590 to 650.
#pragma once

#include "kernels_delta.hpp"

// Columns of the state's gradient through the chunks in reverse order.
template <class T, bool VEC, int DK>
__global__ void __launch_bounds__(512, 1)
    k_delta_back(DeltaArgs p, int blocks, const T* q, const T* k, const T* dy, const float* dlast, const char* work,
                 float* ds0, float* dstates, float* xs) {
  using Lds = ScanLds<T, DK, true>;
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
    const T *kp = k + b * p.k.b + kh * p.k.h, *qp = q + b * p.q.b + kh * p.q.h, *yp = dy + b * p.y.b + head * p.y.h + first;
    const char* wp = work + bh * p.nchunk * Work::bytes;
    ChunkInFlight<T, VEC, DK, true> f;
    const auto load = [&](int chunk) {
      const int n = min(C, len - chunk * C);
      f.load(p, kp, qp, wp, chunk, n, tid);
      f.x.load(yp + (int64_t)chunk * C * p.y.t, (int32_t)p.y.t, n, there, tid);
    };
    const auto store = [&](int chunk) {
      f.store(lds + (chunk & 1) * Lds::bytes, tid);
      f.x.store(lds + Lds::panel_of(chunk), tid);
    };
    if (chunks > 0) load(chunks - 1), store(chunks - 1);
    if (chunks > 1) load(chunks - 2);
    for (int chunk = chunks - 1; chunk >= 0; --chunk) {
      __syncthreads();   // this chunk's operands are there, and the other half is read
      if (chunk > 0) store(chunk - 1);
      if (chunk > 1) load(chunk - 2);
    }
    return;
  }
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, g = lane / 16, at = lane_place(lane % 16, g);
  const int even = turn_place<true>(lane), odd = turn_odd<true>(lane);
  const int tile = first + wave * 16, col = tile + lane % 16;
  const bool mine = col < p.dv, some = tile < pad_columns(p.dv);
  f32x4 s[DK / 16];
#pragma unroll
  for (int m = 0; m < DK / 16; ++m)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int d = order_of(m, g, r);
      s[m][r] = dlast && mine && d < p.dk ? dlast[(bh * p.dk + d) * p.dv + col] : 0.0f;
    }
  for (int chunk = chunks - 1; chunk >= 0; --chunk) {
    const char* const here = lds + (chunk & 1) * Lds::bytes;
    __syncthreads();
    if (!some) continue;
    put_state<DK>(dstates + (bh * p.nchunk + chunk) * pad_keys(p.dk) * pad_columns(p.dv), p.dk, col, g, s);
    constexpr int TRI = tri_pieces(C), NEAR = sizeof(T) == 2 ? 4 : 1;
    const char* const tri = here + Lds::work;
    const float* e = (const float*)(tri + Work::scales);
    f32x4 dyr[C / 16], x[C / 16];
    {
      auto rows = ahead_of<RP, NEAR>([&](int i) { return op_take<PI>(here + Lds::k, RP, i, at); });
      Op<kState> sp[KS];
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) sp[ks] = op_of<kState>(s[2 * ks], s[2 * ks + 1]);
#pragma unroll
      for (int m = 0; m < C / 16; ++m) {
        x[m] = zero4();
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) x[m] = op_mul<kState>(rows(m * KS + ks), sp[ks], x[m]);
        x[m] *= *(const f32x4*)(e + C + m * 16 + g * 4);
      }
    }
    {
      auto reads = ahead_of<TRI, 2>([&](int i) { return op_take<kState>(tri + Work::reads, TRI, tri_upper<C>(i), lane); });
      panel_take<T>(lds + Lds::panel_of(chunk), wave, lane, dyr);
      Op<PI> dp[C / 32];
#pragma unroll
      for (int ks = 0; ks < C / 32; ++ks) dp[ks] = op_of<PI>(dyr[2 * ks], dyr[2 * ks + 1]);
      each<TRI>([&](auto i) {
        constexpr int m = tri_row<C, true>(i), ks = tri_column<C, true>(i);
        x[m] = op_mul<kState>(reads(i), dp[ks], x[m]);
      });
    }
    auto solve = ahead_of<TRI, 2>([&](int i) { return op_take<kState>(tri + Work::solve, TRI, tri_upper<C>(i), lane); });
    Op<kState> xp[C / 32], dp[C / 32];
#pragma unroll
    for (int m = 0; m < C / 16; ++m) x[m] *= *(const f32x4*)(e + 2 * C + m * 16 + g * 4);
#pragma unroll
    for (int ks = 0; ks < C / 32; ++ks) xp[ks] = op_of<kState>(x[2 * ks], x[2 * ks + 1]);
#pragma unroll
    for (int m = 0; m < C / 16; ++m) x[m] = zero4();
    each<TRI>([&](auto i) {
      constexpr int m = tri_row<C, true>(i), ks = tri_column<C, true>(i);
      x[m] = op_mul<kState>(solve(i), xp[ks], x[m]);
    });
    put_rows<C>(xs + (bh * p.nchunk + chunk) * C * pad_columns(p.dv), col, g, x);
    auto turned = ahead_of<RP, NEAR / 2 + 1>([&](int i) {
      return OpPair<PI, PI>{op_turn<PI, KS>(here + Lds::q, RP, i / (C / 32), i % (C / 32), even, odd),
                            op_turn<PI, KS>(here + Lds::k, RP, i / (C / 32), i % (C / 32), even, odd)};
    });
#pragma unroll
    for (int m = 0; m < C / 16; ++m) {
      const f32x4 em = *(const f32x4*)(e + m * 16 + g * 4);
      x[m] *= -em;
      dyr[m] *= p.scale * em;
    }
#pragma unroll
    for (int ks = 0; ks < C / 32; ++ks) {
      xp[ks] = op_of<kState>(x[2 * ks], x[2 * ks + 1]);
      dp[ks] = op_of<kState>(dyr[2 * ks], dyr[2 * ks + 1]);
    }
    const float keep = e[C - 1];
#pragma unroll
    for (int m = 0; m < DK / 16; ++m) {
      s[m] *= keep;
#pragma unroll
      for (int ks = 0; ks < C / 32; ++ks) {
        const auto& o = turned(m * (C / 32) + ks);
        s[m] = op_mul<kState>(o.a, dp[ks], s[m]);
        s[m] = op_mul<kState>(o.b, xp[ks], s[m]);
      }
    }
  }
  if (ds0 && mine)
#pragma unroll
    for (int m = 0; m < DK / 16; ++m)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int d = order_of(m, g, r);
        if (d < p.dk) ds0[(bh * p.dk + d) * p.dv + col] = s[m][r];
      }
}

// Four computing wavefronts: C / 16 tiles of steps, and the keys dealt to so many of each.
template <class T>
constexpr int kGradParts = 64 / kChunk<T>;

// 32 columns of a chunk at a time: rows of S, dS (a column's keys), Z, X (a column's
// steps) and dY (a step's columns), two of these beside each other.  Behind the last
// ones the rows of K and Q come, and then the four products in the place of the last
// ones, as operands, 16 steps x 32 steps a piece.
template <class T, int DK>
struct GradLds {
  static constexpr int C = kChunk<T>, PI = kIn<T>, NP = kGradParts<T>, product = kState * tri_pieces(C) * 1024;
  static constexpr int s = 0, ds = kState * DK * 64, z = 2 * ds, x = z + kState * C * 64, dy = x + kState * C * 64,
                       slabs = dy + PI * C * 64, k = 0, q = PI * C * DK * 2, rows = 2 * q;
  static constexpr int most(int a, int b) { return a > b ? a : b; }
  static constexpr int half = most(slabs, most(rows, 4 * product)), sums = 2 * half,
                       bytes = sums + (3 * C + 2 * NP * C + 16) * 4 + C * 8;
};

struct DeltaGradOut {
  void *dq, *dk, *dv;   // packed
  float *ddecay, *drate;
};

// The row in LDS of column j of 32: a transposing operand's lanes of group g take rows
// 4 g .. and 16 + 4 g .., and get columns 8 g .. 8 g + 7, as rows' operands do.
__device__ __forceinline__ int column_row(int j) { return j / 8 * 4 + j % 4 + j % 8 / 4 * 16; }

// 32 columns of COLS values side by side (`there` of them in memory), on their way to LDS.
template <int COLS, int THREADS>
struct SlabInFlight {
  static constexpr int N = 32 * COLS / 8, U = (N + THREADS - 1) / THREADS, KS = COLS / 32;
  f32x4 v[U][2];

  __device__ __forceinline__ void load(const float* x, int there, int tid) {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int u = tid + i * THREADS, row = u / 4 % 32, c = u / 128 * 32 + u % 4 * 8;
      v[i][0] = v[i][1] = zero4();
      if ((N % THREADS == 0 || u < N) && c < there) {
        const f32x4* from = (const f32x4*)(x + (uint32_t)(row * there + c));
        v[i][0] = from[0], v[i][1] = from[1];
      }
    }
  }

  __device__ __forceinline__ void store(char* lds, int tid) const {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int u = tid + i * THREADS, row = column_row(u / 4 % 32), c = u / 128 * 4 + u % 4;
      if (N % THREADS != 0 && u >= N) continue;
      const Op<kState> o = op_of<kState>(v[i][0], v[i][1]);
#pragma unroll
      for (int p = 0; p < kState; ++p)
        *(bf16x8*)(lds + ((p * 2 * KS + row / 16 * KS + c / 4) * 64 + lane_place(row % 16, c % 4)) * 16) = o.p[p];
    }
  }
};

// 32 columns of dY, rows of steps, the same way.
template <class T, bool VEC, int C, int THREADS>
struct StepsInFlight {
  static constexpr int N = C * 4, U = (N + THREADS - 1) / THREADS;
  float v[U][8];

  __device__ __forceinline__ void load(const T* x, int64_t stride, int there, int width, int tid) {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int u = tid + i * THREADS, row = u / 4, c = u % 4 * 8;
      const bool some = row < there && c < width;
      load8<T, VEC>(x + (some ? row * stride + c : 0), some ? width - c : 0, v[i]);
    }
  }

  __device__ __forceinline__ void store(char* lds, int tid) const {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int u = tid + i * THREADS, row = u / 4;
      if (N % THREADS != 0 && u >= N) continue;
      const Op<kIn<T>> o = op_of<kIn<T>>(v[i]);
#pragma unroll
      for (int p = 0; p < kIn<T>; ++p)
        *(bf16x8*)(lds + ((p * (C / 16) + row / 16) * 64 + lane_place(row % 16, u % 4)) * 16) = o.p[p];
    }
  }
};

// Chunk u of all key heads and rows: n steps count, `in` are in the arrays.
struct GradPlace {
  int64_t chunk, b, t0, step;
  int kh, n, in;
  __device__ __forceinline__ GradPlace(const DeltaArgs& p, int key_heads, int64_t u, int C) {
    const uint32_t nchunk = (uint32_t)p.nchunk, of = (uint32_t)u / nchunk;   // fewer than 2^31 chunks
    chunk = (uint32_t)u % nchunk, b = of / key_heads, kh = (int)(of % key_heads);
    t0 = chunk * C, step = b * p.steps + t0;
    const int len = p.lengths ? min(max(p.lengths[b], 0), p.steps) : p.steps;
    n = (int)max((int64_t)0, min((int64_t)C, len - t0)), in = (int)min((int64_t)C, p.steps - t0);
  }
};

// dQ, dK and the gates of a chunk of one key head, its heads one after the other, and
// dV.  A workgroup to a CU goes from chunk to chunk.  Four wavefronts feed (256 threads): the next columns' values to the other half
// of LDS as operands, X out as dV, the gates' sums.  Of the four that compute each
// has 16 steps and a part of the keys.  The four products over the values z dy', z x'
// (of earlier steps with later ones), dy z', x z' (of later with earlier) are computed
// beside, in tiles dealt to all of them, and then are the operands that multiply K, Q.
// GROUP: heads share key heads, and dQ and dK stay in registers from head to head.
template <class T, bool VEC, int DK, bool GROUP>
__global__ void __launch_bounds__(512, 1)
    k_delta_grad(DeltaArgs p, const T* q, const T* k, const T* dy, const float* decay, const float* rate,
                 const float* states, const float* errors, const float* dstates, const float* xs, DeltaGradOut out) {
  using Lds = GradLds<T, DK>;
  constexpr int C = kChunk<T>, PI = kIn<T>, NP = kGradParts<T>;
  constexpr int RT = C / 16, KC = C / 32, NT = DK / 16, MT = NT / NP, KS = DK / 32, RP = RT * KS;
  constexpr int JOBS = RT * (RT + 1), MINE = (JOBS + 3) / 4;
  extern __shared__ __align__(16) char lds[];
  float* const sc = (float*)(lds + Lds::sums);   // e, o, b
  float* const dg = sc + 3 * C;                  // gradients of G, and k W, by parts
  float* const kw = dg + NP * C;
  float* const red = kw + NP * C;                // <dS, S>: of the feeding wavefronts, then the others' part
  double* const sum = (double*)(red + 16);
  const int key_heads = p.heads / p.group, kp = pad_keys(p.dk), cols = pad_columns(p.dv), rounds = cols / 32;
  const int64_t all = p.batch * key_heads * p.nchunk;
  if (threadIdx.x >= 256) {   // feeds
    const int tid = threadIdx.x - 256;
    // the next chunk from u on that has steps; dQ, dK, dV and the gates of those without are zeros
    const auto some_from = [&](int64_t u) {
      for (; u < all; u += gridDim.x) {
        const GradPlace w(p, key_heads, u, C);
        if (w.n > 0) break;
        for (int i = tid; i < w.in * p.dk; i += 256) {
          const int64_t to = ((w.step + i / p.dk) * key_heads + w.kh) * p.dk + i % p.dk;
          ((T*)out.dq)[to] = ((T*)out.dk)[to] = (T)0.0f;
        }
        for (int h = w.kh * p.group; h < (w.kh + 1) * p.group; ++h) {
          for (int i = tid; i < w.in * p.dv; i += 256)
            ((T*)out.dv)[((w.step + i / p.dv) * p.heads + h) * p.dv + i % p.dv] = (T)0.0f;
          for (int t = tid; t < w.in; t += 256) out.ddecay[(w.step + t) * p.heads + h] = out.drate[(w.step + t) * p.heads + h] = 0.0f;
        }
      }
      return u;
    };
    RowsInFlight<T, VEC, C, DK, 256> kr, qr;
    SlabInFlight<DK, 256> sr, dsr;
    SlabInFlight<C, 256> zr, xr;
    StepsInFlight<T, VEC, C, 256> yr;
    float dx = 0.0f, rx = 0.0f;   // this thread's step's gates
    const auto load = [&](const GradPlace& w, int h, int c) {
      const int64_t cell = (w.b * p.heads + w.kh * p.group + h) * p.nchunk + w.chunk;
      sr.load(states + cell * kp * cols + c * kp, kp, tid);
      dsr.load(dstates + cell * kp * cols + c * kp, kp, tid);
      zr.load(errors + cell * C * cols + c * C, C, tid);
      xr.load(xs + cell * C * cols + c * C, C, tid);
      yr.load(dy + w.b * p.y.b + w.t0 * p.y.t + (w.kh * p.group + h) * p.y.h + c, p.y.t, w.n, p.dv - c, tid);
    };
    const auto begin = [&](const GradPlace& w, int h) {
      if (tid < w.n && tid < C) {
        const int head = w.kh * p.group + h;
        dx = decay[w.b * p.decay.b + (w.t0 + tid) * p.decay.t + head * p.decay.h];
        rx = rate[w.b * p.rate.b + (w.t0 + tid) * p.rate.t + head * p.rate.h];
      }
      load(w, h, 0);
      if (h == 0) {
        kr.load(k + w.b * p.k.b + w.t0 * p.k.t + w.kh * p.k.h, p.k.t, w.n, p.dk, tid);
        qr.load(q + w.b * p.q.b + w.t0 * p.q.t + w.kh * p.q.h, p.q.t, w.n, p.dk, tid);
      }
    };
    int64_t u = some_from(blockIdx.x);
    int h = 0;
    if (u < all) begin(GradPlace(p, key_heads, u, C), 0);
    while (u < all) {
      const GradPlace w(p, key_heads, u, C);
      const int64_t gate = w.step * p.heads + w.kh * p.group + h;
      const bool counts = tid < C && tid < w.n,
                 forgets = counts && __builtin_amdgcn_exp2f((float)((double)dx * 1.4426950408889634)) == 0.0f;
      float inner = 0.0f, all_kept = 0.0f;   // <dS, S>, this thread's part
      const auto store = [&](char* half) {
        sr.store(half + Lds::s, tid);
        dsr.store(half + Lds::ds, tid);
        zr.store(half + Lds::z, tid);
        xr.store(half + Lds::x, tid);
        yr.store(half + Lds::dy, tid);
#pragma unroll
        for (int i = 0; i < decltype(sr)::U; ++i)
#pragma unroll
          for (int j = 0; j < 8; ++j) inner = fmaf(sr.v[i][j / 4][j % 4], dsr.v[i][j / 4][j % 4], inner);
      };
      if (tid < C) {
        double d = counts ? dx < -200.0f ? -200.0 : (double)dx : 0.0;
#pragma unroll
        for (int o = 1; o < C; o *= 2) {
          const double x = __shfl_up(d, o, 64);
          if (tid >= o) d += x;
        }
        d *= 1.4426950408889634;
        const double end = __shfl(d, C - 1, 64);
        all_kept = __builtin_amdgcn_exp2f((float)end);
        sum[tid] = d;
        sc[tid] = __builtin_amdgcn_exp2f((float)d);
        sc[C + tid] = __builtin_amdgcn_exp2f((float)(end - d));
        sc[2 * C + tid] = counts ? rx : 0.0f;
      }
      store(lds);
      if (rounds > 1) load(w, h, 32);
      for (int round = 0; round < rounds; ++round) {
        __syncthreads();   // these columns' values are there, and the other half is read
        char* const next = lds + (~round & 1) * Lds::half;
        if (round + 1 < rounds) {
          store(next);
          if (round + 2 < rounds) load(w, h, (round + 2) * 32);
        } else {
          kr.store(next + Lds::k, tid);
          qr.store(next + Lds::q, tid);
        }
        // X's four columns of a step, as dV
#pragma unroll
        for (int j0 = 0; j0 < C * 8; j0 += 256) {
          typedef short s16x4 __attribute__((ext_vector_type(4)));
          typedef __attribute__((address_space(3))) s16x4* From;
          const int i = j0 + tid, s = i % 16, j = i / 16 % 8, tile = i / 128, t = tile * 16 + s, c = round * 32 + j * 4;
          const int r0 = column_row(j * 4) + s / 4;   // columns of one transposing read, in order
          f32x4 x = zero4();
#pragma unroll
          for (int o = PI - 1; o >= 0; --o) {
            const char* from = lds + (round & 1) * Lds::half + Lds::x + (o * 2 * KC + r0 / 16 * KC + tile / 2) * 1024 +
                               lane_place(r0 % 16, tile % 2 * 2 + s % 4 / 2) * 16 + s % 2 * 8;
            const bf16x4 v = __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((From)from));
#pragma unroll
            for (int r = 0; r < 4; ++r) x[r] += (float)v[r];
          }
          if (t >= w.in || c >= p.dv) continue;
          Words<T, 4> o;
#pragma unroll
          for (int r = 0; r < 4; ++r) o.v[r] = (T)x[r];
          T* const to = (T*)out.dv + (gate + (int64_t)t * p.heads) * p.dv + c;
          if constexpr (VEC) {
            *(Words<T, 4>*)to = o;
          } else {
#pragma unroll
            for (int r = 0; r < 4; ++r)
              if (c + r < p.dv) to[r] = o.v[r];
          }
        }
      }
      // the next head's or chunk's first values, while this one's last products are computed
      if (++h == p.group) h = 0, u = some_from(u + gridDim.x);
      if (u < all) begin(GradPlace(p, key_heads, u, C), h);
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) inner += __shfl_xor(inner, o, 64);
      if (tid % 64 == 0) red[tid / 64] = inner;
      __syncthreads();   // K and Q are there, and the last values are read
      __syncthreads();   // the products are there
      __syncthreads();   // and read: the sums are there
      if (tid < C) {
        double s = 0.0;   // what lies behind a step cancels in its sum
        float v = 0.0f;
#pragma unroll
        for (int i = 0; i < NP; ++i) s += dg[i * C + tid], v += kw[i * C + tid];
        if (tid == C - 1) s += (double)all_kept * ((red[0] + red[1]) + (red[2] + red[3])) + ((red[4] + red[5]) + (red[6] + red[7]));
        int ends = __shfl_down((int)forgets, 1, 64);   // the sum of this step and those behind it stops within
        if (tid == C - 1) ends = 1;
#pragma unroll
        for (int o = 1; o < C; o *= 2) {
          const double x = __shfl_down(s, o, 64);
          const int there = __shfl_down(ends, o, 64);
          if (!ends) s += x, ends = there;
        }
        if (tid < w.in) {
          out.ddecay[gate + (int64_t)tid * p.heads] = counts && !forgets ? (float)s : 0.0f;
          out.drate[gate + (int64_t)tid * p.heads] = counts ? v : 0.0f;
        }
      }
    }
    return;
  }
  for (int64_t u = blockIdx.x; u < all; u += gridDim.x) {
    const GradPlace w(p, key_heads, u, C);
    if (w.n == 0) continue;
    T* const dqb = (T*)out.dq + (w.step * key_heads + w.kh) * p.dk;
    T* const dkb = (T*)out.dk + (w.step * key_heads + w.kh) * p.dk;
    const int in = w.in;
    const int lane = threadIdx.x % 64, g = lane / 16, all_waves = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int wave = all_waves % RT, part = all_waves / RT;
    const int at = lane_place(lane % 16, g), even = turn_place<false>(lane), odd = turn_odd<false>(lane);
    f32x4 dq[MT], dk[MT];
    if (GROUP)
#pragma unroll
      for (int m = 0; m < MT; ++m) dq[m] = dk[m] = zero4();
    for (int h = 0; h < p.group; ++h) {
      // sums over the values, 32 at a time
      f32x4 eq[MT], er[MT], ew[MT], py[MINE], px[MINE];
#pragma unroll
      for (int m = 0; m < MT; ++m) eq[m] = er[m] = ew[m] = zero4();
#pragma unroll
      for (int i = 0; i < MINE; ++i) py[i] = px[i] = zero4();
      for (int round = 0; round < rounds; ++round) {
        __syncthreads();
        const char* const here = lds + (round & 1) * Lds::half;
        {
          const Op<kState> zo = op_turn<kState, KC>(here + Lds::z, 2 * KC, wave, 0, even, odd),
                           xo = op_turn<kState, KC>(here + Lds::x, 2 * KC, wave, 0, even, odd);
          const Op<PI> yo = op_take<PI>(here + Lds::dy, RT, wave, at);
          auto states_of = ahead_of<2 * MT, 1>([&](int i) {
            return op_turn<kState, KS>(here + (i % 2 ? Lds::ds : Lds::s), 2 * KS, part * MT + i / 2, 0, even, odd);
          });
#pragma unroll
          for (int m = 0; m < MT; ++m) {
            const Op<kState>& o = states_of(2 * m);
            eq[m] = op_mul<kState>(yo, o, eq[m]);
            er[m] = op_mul<kState>(xo, o, er[m]);
            ew[m] = op_mul<kState>(zo, states_of(2 * m + 1), ew[m]);
          }
        }
        // tile i of the first half: steps 16 a .. of Z against 16 c .. of dY and X, a <= c;
        // of the second: 16 c .. of dY and X against 16 a .. of Z
#pragma unroll
        for (int i = 0; i < MINE; ++i) {
          int job = all_waves + i * 4;
          asm volatile("" : "+s"(job));   // what follows from it is computed here, not kept in registers from round to round
          if (JOBS % 4 != 0 && job >= JOBS) continue;
          const int half = job < JOBS / 2 ? job : job - JOBS / 2;
          const int c = half < 1 ? 0 : half < 3 ? 1 : half < 6 ? 2 : 3, a = half - c * (c + 1) / 2;
          const Op<kState> zo = op_turn<kState, KC>(here + Lds::z, 2 * KC, a, 0, even, odd),
                           xo = op_turn<kState, KC>(here + Lds::x, 2 * KC, c, 0, even, odd);
          const Op<PI> yo = op_take<PI>(here + Lds::dy, RT, c, at);
          if (job < JOBS / 2) {
            py[i] = op_mul<kState>(zo, yo, py[i]);
            px[i] = op_mul<kState>(zo, xo, px[i]);
          } else {
            py[i] = op_mul<kState>(yo, zo, py[i]);
            px[i] = op_mul<kState>(xo, zo, px[i]);
          }
        }
      }
      __syncthreads();   // K and Q are there, and the last values are read
      const char* const rows = lds + (rounds & 1) * Lds::half;
      char* const products = lds + (~rounds & 1) * Lds::half;
#pragma unroll
      for (int i = 0; i < MINE; ++i) {
        int job = all_waves + i * 4;
        asm volatile("" : "+s"(job));
        if (JOBS % 4 != 0 && job >= JOBS) continue;
        const bool first = job < JOBS / 2;
        const int half = first ? job : job - JOBS / 2;
        const int c = half < 1 ? 0 : half < 3 ? 1 : half < 6 ? 2 : 3, a = half - c * (c + 1) / 2;
        // the operand's row is the lane's column, its 32 columns rows of this result and the next
        const int mt = first ? c : a, kt = first ? a : c, step = mt * 16 + lane % 16;
        const int piece = (first ? tri_piece<C, false>(mt, kt / 2) : tri_piece<C, true>(mt, kt / 2)) * 64 + lane;
        const double mine = sum[step];
        f32x4 y = py[i], x = px[i];
        const int t0 = kt * 16 + g * 4;
        const f32x4 bt = first ? *(const f32x4*)(sc + 2 * C + t0) : f32x4{1.0f, 1.0f, 1.0f, 1.0f};
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float apart = (float)(first ? mine - sum[t0 + r] : sum[t0 + r] - mine);
          const float d = __builtin_amdgcn_exp2f(apart) * bt[r];
          const int before = first ? step - (t0 + r) : t0 + r - step;   // below 0: on the wrong side, where d may be infinite
          y[r] = before >= 0 ? y[r] * d * p.scale : 0.0f;
          x[r] = before > 0 ? x[r] * (first ? d : -d) : 0.0f;
        }
        char* const to = products + (first ? 0 : 2 * Lds::product) + piece * 16 + kt % 2 * 8;
#pragma unroll
        for (int o = 0; o < kState; ++o) {
          bf16x4 hy, hx;
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            hy[r] = (__bf16)y[r], hx[r] = (__bf16)x[r];
            y[r] -= (float)hy[r], x[r] -= (float)hx[r];
          }
          *(bf16x4*)(to + o * tri_pieces(C) * 1024) = hy;
          *(bf16x4*)(to + Lds::product + o * tri_pieces(C) * 1024) = hx;
        }
      }
      // the halves of a piece on the diagonal that no tile fills: rows of an even tile have
      // nothing from the next one, and of an odd one nothing after
      if (all_waves < RT) {
        const bool first = wave % 2 == 0;
        const int piece = (first ? tri_piece<C, false>(wave, wave / 2) : tri_piece<C, true>(wave, wave / 2)) * 64 + lane;
        char* const to = products + (first ? 0 : 2 * Lds::product) + piece * 16 + (first ? 8 : 0);
#pragma unroll
        for (int o = 0; o < kState; ++o)
          *(bf16x4*)(to + o * tri_pieces(C) * 1024) = *(bf16x4*)(to + Lds::product + o * tri_pieces(C) * 1024) = bf16x4{};
      }
      float end = 0.0f;   // o[t] b[t] k[t] dS z[t], this lane's part: <dS, K' diag(o b) Z>
      f32x4 total = zero4(), wk = zero4();
      const f32x4 re = *(const f32x4*)(sc + wave * 16 + g * 4), ro = *(const f32x4*)(sc + C + wave * 16 + g * 4),
                  rb = *(const f32x4*)(sc + 2 * C + wave * 16 + g * 4);
      // K or Q of this tile's steps 4 g + r, key 16 m + lane % 16: a transposing read of 4 rows
      const auto values = [&](const char* from, int m) {
        typedef short s16x4 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) s16x4* From;
        f32x4 x = zero4();
#pragma unroll
        for (int o = PI - 1; o >= 0; --o) {
          const char* a = from + (o * RP + wave * KS + m / 2) * 1024 + (m % 2 ? odd : even);
          const bf16x4 v = __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((From)a));
#pragma unroll
          for (int r = 0; r < 4; ++r) x[r] += (float)v[r];
        }
        return x;
      };
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        const f32x4 kv = values(rows + Lds::k, part * MT + m);
        eq[m] *= re * p.scale, er[m] *= re, ew[m] *= ro;
#pragma unroll
        for (int r = 0; r < 4; ++r) end = fmaf(rb[r] * kv[r], ew[m][r], end);
      }
      __syncthreads();   // the products are there
#pragma unroll
      for (int ks = 0; ks < KC; ++ks) {
        if (ks <= wave / 2) {
          const int piece = tri_piece<C, false>(wave, ks);
          const Op<kState> y = op_take<kState>(products, tri_pieces(C), piece, lane),
                           x = op_take<kState>(products + Lds::product, tri_pieces(C), piece, lane);
          auto keys = ahead_of<MT, 2>(
              [&](int m) { return op_turn<PI, KS>(rows + Lds::k, RP, part * MT + m, ks, even, odd); });
#pragma unroll
          for (int m = 0; m < MT; ++m) {
            const auto& kc = keys(m);
            eq[m] = op_mul<kState>(y, kc, eq[m]);
            er[m] = op_mul<kState>(x, kc, er[m]);
          }
        }
        if (ks >= wave / 2) {
          const int piece = tri_piece<C, true>(wave, ks);
          const Op<kState> y = op_take<kState>(products + 2 * Lds::product, tri_pieces(C), piece, lane),
                           x = op_take<kState>(products + 3 * Lds::product, tri_pieces(C), piece, lane);
          auto both = ahead_of<MT, 1>([&](int m) {
            return OpPair<PI, PI>{op_turn<PI, KS>(rows + Lds::q, RP, part * MT + m, ks, even, odd),
                                  op_turn<PI, KS>(rows + Lds::k, RP, part * MT + m, ks, even, odd)};
          });
#pragma unroll
          for (int m = 0; m < MT; ++m) {
            const auto& o = both(m);
            ew[m] = op_mul<kState>(y, o.a, ew[m]);
            ew[m] = op_mul<kState>(x, o.b, ew[m]);
          }
        }
      }
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        const f32x4 kv = values(rows + Lds::k, part * MT + m), qv = values(rows + Lds::q, part * MT + m);
        wk += kv * ew[m];
        total += qv * eq[m] - kv * er[m];
        er[m] = rb * ew[m] - er[m];
        if (GROUP) dq[m] += eq[m], dk[m] += er[m];
      }
      // sums over the 16 lanes of a row, and over the workgroup
#pragma unroll
      for (int o = 1; o < 16; o *= 2)
#pragma unroll
        for (int r = 0; r < 4; ++r) total[r] += __shfl_xor(total[r], o, 64), wk[r] += __shfl_xor(wk[r], o, 64);
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) end += __shfl_xor(end, o, 64);
      if (lane == 0) red[4 + all_waves] = end;
      if (lane % 16 == 0) {
        *(f32x4*)(dg + part * C + wave * 16 + g * 4) = total - rb * wk;
        *(f32x4*)(kw + part * C + wave * 16 + g * 4) = wk;
      }
      __syncthreads();   // the products are read: the sums are there
      if (GROUP && h + 1 < p.group) continue;
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int t = wave * 16 + g * 4 + r, d = (part * MT + m) * 16 + lane % 16;
          if (t < in && d < p.dk) {
            dqb[(int64_t)t * key_heads * p.dk + d] = (T)(GROUP ? dq[m][r] : eq[m][r]);
            dkb[(int64_t)t * key_heads * p.dk + d] = (T)(GROUP ? dk[m][r] : er[m][r]);
          }
        }
    }
  }
}
