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
// and decay[t] is in all G from t on: a sum from the chunk's end.
#pragma once

#include "kernels_delta.hpp"

// Columns of the state's gradient through the chunks in reverse order.
template <class T, bool VEC, int DK>
__global__ void __launch_bounds__(512, 1)
    k_delta_back(DeltaArgs p, int blocks, const T* q, const T* k, const T* dy, const float* dlast, const char* work,
                 float* ds0, float* dstates, float* xs) {
  using Lds = ScanLds<T, DK, true>;
  constexpr int C = Lds::C, KS = DK / 32, PI = kIn<T>, RP = C / 16 * KS;
  using Work = ChunkWork<C, kState>;
  extern __shared__ __align__(16) char lds[];
  int64_t bh;
  int block;
  if (!scan_place(p, blocks, bh, block)) return;
  const int64_t b = bh / p.heads;
  const int head = (int)(bh % p.heads), kh = head / p.group, first = block * 64;
  const int len = p.lengths ? min(max(p.lengths[b], 0), p.steps) : p.steps;
  const int chunks = (len + C - 1) / C;
  if (threadIdx.x >= 256) {   // feeds
    const int tid = threadIdx.x - 256, there = p.dv - first;
    const T *kp = k + b * p.k.b + kh * p.k.h, *qp = q + b * p.q.b + kh * p.q.h, *yp = dy + b * p.y.b + head * p.y.h + first;
    const char* wp = work + bh * p.nchunk * Work::bytes;
    ChunkInFlight<T, VEC, DK, true> f;
    const auto load = [&](int chunk) { f.load(p, kp, qp, yp, p.y, wp, chunk, min(C, len - chunk * C), there, tid); };
    if (chunks > 0) {
      load(chunks - 1);
      f.store(lds + (~chunks & 1) * Lds::bytes, tid);
    }
    if (chunks > 1) load(chunks - 2);
    for (int chunk = chunks - 1; chunk >= 0; --chunk) {
      __syncthreads();   // this chunk's operands are there, and the other half is read
      if (chunk > 0) f.store(lds + (~chunk & 1) * Lds::bytes, tid);
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
      panel_take<T>(here + Lds::panel, wave, lane, dyr);
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

// Wavefronts of k_delta_grad: C / 16 tiles of steps, and the keys dealt to so many of each.
template <class T, int DK>
constexpr int kGradParts = kChunk<T> == 64 ? 2 : DK >= 64 ? 4 : 2;
template <class T, int DK>
constexpr int kGradThreads = kChunk<T> * 4 * kGradParts<T, DK>;

// 32 columns of a chunk at a time: rows of K and Q, then rows of S, dS (a column's
// keys), Z, X (a column's steps) and dY (a step's columns); then, in their place, the
// four products as operands, 16 steps x 32 steps a piece.
template <class T, int DK>
struct GradLds {
  static constexpr int C = kChunk<T>, PI = kIn<T>, NP = kGradParts<T, DK>, product = kState * tri_pieces(C) * 1024;
  static constexpr int k = 0, q = k + PI * C * DK * 2, s = q + PI * C * DK * 2, ds = s + kState * DK * 64,
                       z = ds + kState * DK * 64, x = z + kState * C * 64, dy = x + kState * C * 64,
                       products = s, after = dy + PI * C * 64 > s + 4 * product ? dy + PI * C * 64 : s + 4 * product,
                       sums = after, bytes = sums + (3 * C + 2 * NP * C + 16) * 4 + C * 8;
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
      const int u = tid + i * THREADS, row = u / (COLS / 8), c = u % (COLS / 8) * 8;
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
      const int u = tid + i * THREADS, row = column_row(u / (COLS / 8)), c = u % (COLS / 8);
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

// dQ, dK and the gates of a chunk of one key head, its heads one after the other.  A
// wavefront has 16 steps and a part of the keys.  The four products over the values
// z dy', z x' (of earlier steps with later ones), dy z', x z' (of later with earlier)
// are computed beside them, in tiles dealt to all wavefronts, and then are the
// operands that multiply K and Q.
template <class T, bool VEC, int DK>
__global__ void __launch_bounds__((kGradThreads<T, DK>), 1)
    k_delta_grad(DeltaArgs p, const T* q, const T* k, const T* dy, const float* decay, const float* rate,
                 const float* states, const float* errors, const float* dstates, const float* xs, DeltaGradOut out) {
  using Lds = GradLds<T, DK>;
  constexpr int C = kChunk<T>, PI = kIn<T>, NP = kGradParts<T, DK>, THREADS = kGradThreads<T, DK>;
  constexpr int RT = C / 16, KC = C / 32, NT = DK / 16, MT = NT / NP, KS = DK / 32, RP = RT * KS;
  constexpr int JOBS = RT * (RT + 1), WAVES = THREADS / 64, MINE = (JOBS + WAVES - 1) / WAVES;
  extern __shared__ __align__(16) char lds[];
  float* const sc = (float*)(lds + Lds::sums);   // e, o, b
  float* const dg = sc + 3 * C;                  // gradients of G, and k W, by parts
  float* const kw = dg + NP * C;
  float* const red = kw + NP * C;
  double* const sum = (double*)(red + 16);
  const int tid = threadIdx.x, lane = tid % 64, g = lane / 16;
  const int all_waves = __builtin_amdgcn_readfirstlane(tid / 64), wave = all_waves % RT, part = all_waves / RT;
  const int at = lane_place(lane % 16, g), even = turn_place<false>(lane), odd = turn_odd<false>(lane);
  const int key_heads = p.heads / p.group, kp = pad_keys(p.dk), cols = pad_columns(p.dv);
  const int64_t all = p.batch * key_heads * p.nchunk;
  for (int64_t u = blockIdx.x; u < all; u += gridDim.x) {
    const int64_t chunk = u % p.nchunk, b = u / p.nchunk / key_heads, t0 = chunk * C;
    const int kh = (int)(u / p.nchunk % key_heads);
    const int len = p.lengths ? min(max(p.lengths[b], 0), p.steps) : p.steps;
    const int n = (int)max((int64_t)0, min((int64_t)C, len - t0)), in = (int)min((int64_t)C, p.steps - t0);
    f32x4 dq[MT], dk[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) dq[m] = dk[m] = zero4();
    for (int h = 0; h < p.group; ++h) {
      const int head = kh * p.group + h;
      const int64_t bh = b * p.heads + head, cell = bh * p.nchunk + chunk, gate = (b * p.steps + t0) * p.heads + head;
      T* const dvp = (T*)out.dv + ((b * p.steps + t0) * p.heads + head) * p.dv;
      if (n == 0) {
        for (int i = tid; i < in * p.dv; i += THREADS) dvp[(int64_t)(i / p.dv) * p.heads * p.dv + i % p.dv] = (T)0.0f;
        for (int t = tid; t < in; t += THREADS)
          out.ddecay[gate + (int64_t)t * p.heads] = out.drate[gate + (int64_t)t * p.heads] = 0.0f;
        continue;
      }
      SlabInFlight<DK, THREADS> sr, dsr;
      SlabInFlight<C, THREADS> zr, xr;
      StepsInFlight<T, VEC, C, THREADS> yr;
      const float *sp = states + cell * kp * cols, *dsp = dstates + cell * kp * cols, *zp = errors + cell * C * cols,
                  *xp = xs + cell * C * cols;
      const T* yp = dy + b * p.y.b + t0 * p.y.t + head * p.y.h;
      const auto ahead = [&](int c) {
        sr.load(sp + c * kp, kp, tid);
        dsr.load(dsp + c * kp, kp, tid);
        zr.load(zp + c * C, C, tid);
        xr.load(xp + c * C, C, tid);
        yr.load(yp + c, p.y.t, n, p.dv - c, tid);
      };
      if (h == 0) {
        RowsInFlight<T, VEC, C, DK, THREADS> kr, qr;
        kr.load(k + b * p.k.b + t0 * p.k.t + kh * p.k.h, p.k.t, n, p.dk, tid);
        qr.load(q + b * p.q.b + t0 * p.q.t + kh * p.q.h, p.q.t, n, p.dk, tid);
        ahead(0);
        __syncthreads();   // what was there is read
        kr.store(lds + Lds::k, tid);
        qr.store(lds + Lds::q, tid);
      } else {
        ahead(0);
      }
      bool forgets = false;
      if (tid < C) {
        double d = 0.0;
        float r = 0.0f;
        if (tid < n) {
          const float x = decay[b * p.decay.b + (t0 + tid) * p.decay.t + head * p.decay.h];
          forgets = x < -200.0f;
          d = forgets ? -200.0 : (double)x;
          r = rate[b * p.rate.b + (t0 + tid) * p.rate.t + head * p.rate.h];
        }
#pragma unroll
        for (int o = 1; o < C; o *= 2) {
          const double x = __shfl_up(d, o, 64);
          if (tid >= o) d += x;
        }
        d *= 1.4426950408889634;
        sum[tid] = d;
        const double end = __shfl(d, C - 1, 64);
        sc[tid] = __builtin_amdgcn_exp2f((float)d);
        sc[C + tid] = __builtin_amdgcn_exp2f((float)(end - d));
        sc[2 * C + tid] = r;
      }
      // sums over the values, 32 at a time
      f32x4 eq[MT], er[MT], ew[MT], py[MINE], px[MINE];
      float inner = 0.0f;   // <dS, S>, this thread's part
#pragma unroll
      for (int m = 0; m < MT; ++m) eq[m] = er[m] = ew[m] = zero4();
#pragma unroll
      for (int i = 0; i < MINE; ++i) py[i] = px[i] = zero4();
      for (int c0 = 0; c0 < cols; c0 += 32) {
        __syncthreads();
        sr.store(lds + Lds::s, tid);
        dsr.store(lds + Lds::ds, tid);
        zr.store(lds + Lds::z, tid);
        xr.store(lds + Lds::x, tid);
        yr.store(lds + Lds::dy, tid);
#pragma unroll
        for (int i = 0; i < decltype(sr)::U; ++i)
#pragma unroll
          for (int j = 0; j < 8; ++j) inner = fmaf(sr.v[i][j / 4][j % 4], dsr.v[i][j / 4][j % 4], inner);
        __syncthreads();
        if (c0 + 32 < cols) ahead(c0 + 32);
        // X's four columns of a step, as dV
        for (int i = tid; i < C * 8; i += THREADS) {
          typedef short s16x4 __attribute__((ext_vector_type(4)));
          typedef __attribute__((address_space(3))) s16x4* From;
          const int s = i % 16, j = i / 16 % 8, tile = i / 128, t = tile * 16 + s, c = c0 + j * 4;
          const int row = column_row(j * 4) + s / 4;   // columns of one transposing read, in order
          Words<T, 4> w;
          f32x4 x = zero4();
#pragma unroll
          for (int o = PI - 1; o >= 0; --o) {
            const char* from = lds + Lds::x + (o * 2 * KC + row / 16 * KC + tile / 2) * 1024 +
                               lane_place(row % 16, tile % 2 * 2 + s % 4 / 2) * 16 + s % 2 * 8;
            const bf16x4 h = __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((From)from));
#pragma unroll
            for (int r = 0; r < 4; ++r) x[r] += (float)h[r];
          }
          if (t >= in || c >= p.dv) continue;
#pragma unroll
          for (int r = 0; r < 4; ++r) w.v[r] = (T)x[r];
          T* const to = dvp + (int64_t)t * p.heads * p.dv + c;
          if constexpr (VEC) {
            *(Words<T, 4>*)to = w;
          } else {
#pragma unroll
            for (int r = 0; r < 4; ++r)
              if (c + r < p.dv) to[r] = w.v[r];
          }
        }
        {
          const Op<kState> zo = op_turn<kState, KC>(lds + Lds::z, 2 * KC, wave, 0, even, odd),
                           xo = op_turn<kState, KC>(lds + Lds::x, 2 * KC, wave, 0, even, odd);
          const Op<PI> yo = op_take<PI>(lds + Lds::dy, RT, wave, at);
#pragma unroll
          for (int m = 0; m < MT; ++m) {
            const Op<kState> so = op_turn<kState, KS>(lds + Lds::s, 2 * KS, part * MT + m, 0, even, odd);
            eq[m] = op_mul<kState>(yo, so, eq[m]);
            er[m] = op_mul<kState>(xo, so, er[m]);
            ew[m] = op_mul<kState>(zo, op_turn<kState, KS>(lds + Lds::ds, 2 * KS, part * MT + m, 0, even, odd), ew[m]);
          }
        }
        // tile i of the first half: steps 16 a .. of Z against 16 c .. of dY and X, a <= c;
        // of the second: 16 c .. of dY and X against 16 a .. of Z
#pragma unroll
        for (int i = 0; i < MINE; ++i) {
          const int job = all_waves + i * WAVES;
          if (job >= JOBS) continue;
          const int half = job < JOBS / 2 ? job : job - JOBS / 2;
          const int c = half < 1 ? 0 : half < 3 ? 1 : half < 6 ? 2 : 3, a = half - c * (c + 1) / 2;
          const Op<kState> zo = op_turn<kState, KC>(lds + Lds::z, 2 * KC, a, 0, even, odd),
                           xo = op_turn<kState, KC>(lds + Lds::x, 2 * KC, c, 0, even, odd);
          const Op<PI> yo = op_take<PI>(lds + Lds::dy, RT, c, at);
          if (job < JOBS / 2) {
            py[i] = op_mul<kState>(zo, yo, py[i]);
            px[i] = op_mul<kState>(zo, xo, px[i]);
          } else {
            py[i] = op_mul<kState>(yo, zo, py[i]);
            px[i] = op_mul<kState>(xo, zo, px[i]);
          }
        }
      }
      __syncthreads();   // the products take the slabs' place
#pragma unroll
      for (int i = 0; i < MINE; ++i) {
        const int job = all_waves + i * WAVES;
        if (job >= JOBS) continue;
        const bool first = job < JOBS / 2;
        const int half = first ? job : job - JOBS / 2;
        const int c = half < 1 ? 0 : half < 3 ? 1 : half < 6 ? 2 : 3, a = half - c * (c + 1) / 2;
        // the operand's row is the lane's column, its 32 columns rows of this result and the next
        const int mt = first ? c : a, kt = first ? a : c, row = mt * 16 + lane % 16;
        const int piece = (first ? tri_piece<C, false>(mt, kt / 2) : tri_piece<C, true>(mt, kt / 2)) * 64 + lane;
        const double mine = sum[row];
        f32x4 y = py[i], x = px[i];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int t = kt * 16 + g * 4 + r;
          const bool there = first ? t <= row : t >= row;
          const float d = there ? __builtin_amdgcn_exp2f((float)(first ? mine - sum[t] : sum[t] - mine)) : 0.0f;
          const float w = first ? d * sc[2 * C + t] : d;
          y[r] = there ? y[r] * w * p.scale : 0.0f;
          x[r] = there && t != row ? (first ? x[r] * w : -x[r] * w) : 0.0f;
        }
        char* const to = lds + Lds::products + (first ? 0 : 2 * Lds::product) + piece * 16 + kt % 2 * 8;
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
      // the halves of a piece on the diagonal that no tile fills
      if (all_waves < RT) {
        const int other = wave ^ 1;
        const bool first = wave % 2 == 0;   // rows of an even tile have nothing from the next one, and of an odd one nothing after
        const int piece = (first ? tri_piece<C, false>(wave, wave / 2) : tri_piece<C, true>(wave, wave / 2)) * 64 + lane;
        char* const to = lds + Lds::products + (first ? 0 : 2 * Lds::product) + piece * 16 + other % 2 * 8;
#pragma unroll
        for (int o = 0; o < kState; ++o)
          *(bf16x4*)(to + o * tri_pieces(C) * 1024) = *(bf16x4*)(to + Lds::product + o * tri_pieces(C) * 1024) = bf16x4{};
      }
      float end = 0.0f;   // o[t] b[t] k[t] dS z[t], this lane's part: <dS, K' diag(o b) Z>
      float rows[4], wk[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) rows[r] = wk[r] = 0.0f;
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
          const bf16x4 h = __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((From)a));
#pragma unroll
          for (int r = 0; r < 4; ++r) x[r] += (float)h[r];
        }
        return x;
      };
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        const f32x4 kv = values(lds + Lds::k, part * MT + m);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          eq[m][r] = share_of(re[r], eq[m][r]) * p.scale;
          er[m][r] = share_of(re[r], er[m][r]);
          ew[m][r] = share_of(ro[r], ew[m][r]);
          end = fmaf(rb[r] * kv[r], ew[m][r], end);
        }
      }
      __syncthreads();
#pragma unroll
      for (int ks = 0; ks < KC; ++ks) {
        const char* const products = lds + Lds::products;
        if (ks <= wave / 2) {
          const int piece = tri_piece<C, false>(wave, ks);
          const Op<kState> y = op_take<kState>(products, tri_pieces(C), piece, lane),
                           x = op_take<kState>(products + Lds::product, tri_pieces(C), piece, lane);
#pragma unroll
          for (int m = 0; m < MT; ++m) {
            const Op<PI> kc = op_turn<PI, KS>(lds + Lds::k, RP, part * MT + m, ks, even, odd);
            eq[m] = op_mul<kState>(y, kc, eq[m]);
            er[m] = op_mul<kState>(x, kc, er[m]);
          }
        }
        if (ks >= wave / 2) {
          const int piece = tri_piece<C, true>(wave, ks);
          const Op<kState> y = op_take<kState>(products + 2 * Lds::product, tri_pieces(C), piece, lane),
                           x = op_take<kState>(products + 3 * Lds::product, tri_pieces(C), piece, lane);
#pragma unroll
          for (int m = 0; m < MT; ++m) {
            ew[m] = op_mul<kState>(y, op_turn<PI, KS>(lds + Lds::q, RP, part * MT + m, ks, even, odd), ew[m]);
            ew[m] = op_mul<kState>(x, op_turn<PI, KS>(lds + Lds::k, RP, part * MT + m, ks, even, odd), ew[m]);
          }
        }
      }
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        const f32x4 kv = values(lds + Lds::k, part * MT + m), qv = values(lds + Lds::q, part * MT + m);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          wk[r] = fmaf(kv[r], ew[m][r], wk[r]);
          rows[r] += qv[r] * eq[m][r] - kv[r] * er[m][r];
          dq[m][r] += eq[m][r];
          dk[m][r] += fmaf(rb[r], ew[m][r], -er[m][r]);
        }
      }
      // sums over the 16 lanes of a row, and over the workgroup
#pragma unroll
      for (int o = 1; o < 16; o *= 2)
#pragma unroll
        for (int r = 0; r < 4; ++r) rows[r] += __shfl_xor(rows[r], o, 64), wk[r] += __shfl_xor(wk[r], o, 64);
      inner = share_of(sc[C - 1], inner) + end;
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) inner += __shfl_xor(inner, o, 64);
      if (lane == 0) red[all_waves] = inner;
      if (lane % 16 == 0)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int t = wave * 16 + g * 4 + r;
          dg[part * C + t] = rows[r] - rb[r] * wk[r];
          kw[part * C + t] = wk[r];
        }
      __syncthreads();
      if (tid < C) {
        float s = 0.0f, w = 0.0f;
#pragma unroll
        for (int i = 0; i < NP; ++i) s += dg[i * C + tid], w += kw[i * C + tid];
        if (tid == C - 1)
#pragma unroll
          for (int i = 0; i < WAVES; ++i) s += red[i];
#pragma unroll
        for (int o = 1; o < C; o *= 2) {
          const float x = __shfl_down(s, o, 64);
          if (tid + o < C) s += x;
        }
        if (tid < in) {
          out.ddecay[gate + (int64_t)tid * p.heads] = tid < n && !forgets ? s : 0.0f;
          out.drate[gate + (int64_t)tid * p.heads] = tid < n ? w : 0.0f;
        }
      }
    }
    T* const dqb = (T*)out.dq + ((b * p.steps + t0) * key_heads + kh) * p.dk;
    T* const dkb = (T*)out.dk + ((b * p.steps + t0) * key_heads + kh) * p.dk;
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int t = wave * 16 + g * 4 + r, d = (part * MT + m) * 16 + lane % 16;
        if (t < in && d < p.dk) {
          dqb[(int64_t)t * key_heads * p.dk + d] = (T)dq[m][r];
          dkb[(int64_t)t * key_heads * p.dk + d] = (T)dk[m][r];
        }
      }
  }
}
