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
// for all chunks at once, sums over the values:
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
__global__ void __launch_bounds__(256)
    k_delta_back(DeltaArgs p, int blocks, const T* q, const T* k, const T* dy, const float* dlast, const char* work, T* dv,
                 float* ds0, float* dstates, float* xs) {
  using Lds = ScanLds<T, DK, true>;
  constexpr int C = Lds::C, KS = DK / 32, PI = kIn<T>, RP = C / 16 * KS, CP = DK / 16 * (C / 32);
  using Work = ChunkWork<C, kState>;
  extern __shared__ __align__(16) char lds[];
  int64_t bh;
  int block;
  if (!scan_place(p, blocks, bh, block)) return;
  const int tid = threadIdx.x, lane = tid % 64, g = lane / 16, at = (lane % 16 ^ g) + 16 * g;
  const int64_t b = bh / p.heads;
  const int head = (int)(bh % p.heads), kh = head / p.group;
  const int col = (block * (int)(blockDim.x / 64) + tid / 64) * 16 + lane % 16;
  const bool mine = col < p.dv;
  const int len = p.lengths ? min(max(p.lengths[b], 0), p.steps) : p.steps;
  const T* yb = dy + b * p.y.b + head * p.y.h + col;
  T* vb = dv + (b * p.steps * p.heads + head) * p.dv + col;
  const int64_t vt = (int64_t)p.heads * p.dv;
  f32x4 s[DK / 16];
#pragma unroll
  for (int m = 0; m < DK / 16; ++m)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int d = m * 16 + g * 4 + r;
      s[m][r] = dlast && mine && d < p.dk ? dlast[(bh * p.dk + d) * p.dv + col] : 0.0f;
    }
  const int64_t chunks = (len + C - 1) / C;
  if (mine)
    for (int64_t t = chunks * C + g; t < p.steps; t += 4) vb[t * vt] = (T)0.0f;
  for (int64_t chunk = chunks - 1; chunk >= 0; --chunk) {
    const int64_t t0 = chunk * C;
    const int n = (int)min((int64_t)C, len - t0);
    __syncthreads();
    stage_operands<T, VEC, C, DK, true, true>(k + b * p.k.b + t0 * p.k.t + kh * p.k.h, p.k.t, n, p.dk, lds + Lds::rows,
                                              lds + Lds::cols, tid, blockDim.x);
    stage_operands<T, VEC, C, DK, false, true>(q + b * p.q.b + t0 * p.q.t + kh * p.q.h, p.q.t, n, p.dk, nullptr,
                                               lds + Lds::q, tid, blockDim.x);
    copy_work(work + (bh * p.nchunk + chunk) * Work::bytes, lds + Lds::work, Work::bytes, tid, blockDim.x);
    f32x4 dyr[C / 16], x[C / 16];
#pragma unroll
    for (int m = 0; m < C / 16; ++m)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int t = m * 16 + g * 4 + r;
        dyr[m][r] = mine && t < n ? as_f32(yb[(t0 + t) * p.y.t]) : 0.0f;
      }
    if (mine)
#pragma unroll
      for (int m = 0; m < DK / 16; ++m)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int d = m * 16 + g * 4 + r;
          if (d < p.dk) dstates[((bh * p.nchunk + chunk) * p.dk + d) * p.dv + col] = s[m][r];
        }
    __syncthreads();
    const float* e = (const float*)(lds + Lds::work + Work::scales);
    {
      Op<kState> sp[KS];
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) sp[ks] = op_of<kState>(s[2 * ks], s[2 * ks + 1]);
#pragma unroll
      for (int m = 0; m < C / 16; ++m) {
        x[m] = zero4();
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) x[m] = op_mul<kState>(op_take<PI>(lds + Lds::rows, RP, m * KS + ks, at), sp[ks], x[m]);
#pragma unroll
        for (int r = 0; r < 4; ++r) x[m][r] = share_of(e[C + m * 16 + g * 4 + r], x[m][r]);
      }
    }
    {
      Op<PI> dp[C / 32];
#pragma unroll
      for (int ks = 0; ks < C / 32; ++ks) dp[ks] = op_of<PI>(dyr[2 * ks], dyr[2 * ks + 1]);
#pragma unroll
      for (int m = 0; m < C / 16; ++m) {
#pragma unroll
        for (int ks = m / 2; ks < C / 32; ++ks)
          x[m] = op_mul<kState>(op_take<kState>(lds + Lds::work + Work::reads, tri_pieces(C), tri_piece<C, true>(m, ks), lane),
                                dp[ks], x[m]);
#pragma unroll
        for (int r = 0; r < 4; ++r) x[m][r] *= e[2 * C + m * 16 + g * 4 + r];
      }
    }
    Op<kState> xp[C / 32];
#pragma unroll
    for (int ks = 0; ks < C / 32; ++ks) xp[ks] = op_of<kState>(x[2 * ks], x[2 * ks + 1]);
#pragma unroll
    for (int m = 0; m < C / 16; ++m) {
      x[m] = zero4();
#pragma unroll
      for (int ks = m / 2; ks < C / 32; ++ks)
        x[m] = op_mul<kState>(op_take<kState>(lds + Lds::work + Work::solve, tri_pieces(C), tri_piece<C, true>(m, ks), lane),
                              xp[ks], x[m]);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int t = m * 16 + g * 4 + r;
        if (mine) xs[((bh * p.nchunk + chunk) * C + t) * p.dv + col] = x[m][r];
        if (mine && t0 + t < p.steps) vb[(t0 + t) * vt] = t < n ? (T)x[m][r] : (T)0.0f;
        x[m][r] *= -e[t];
        dyr[m][r] *= p.scale * e[t];
      }
    }
    Op<kState> dp[C / 32];
#pragma unroll
    for (int ks = 0; ks < C / 32; ++ks) {
      xp[ks] = op_of<kState>(x[2 * ks], x[2 * ks + 1]);
      dp[ks] = op_of<kState>(dyr[2 * ks], dyr[2 * ks + 1]);
    }
    const float keep = e[C - 1];
#pragma unroll
    for (int m = 0; m < DK / 16; ++m) {
#pragma unroll
      for (int r = 0; r < 4; ++r) s[m][r] = share_of(keep, s[m][r]);
#pragma unroll
      for (int ks = 0; ks < C / 32; ++ks) {
        s[m] = op_mul<kState>(op_take<PI>(lds + Lds::q, CP, m * (C / 32) + ks, at), dp[ks], s[m]);
        s[m] = op_mul<kState>(op_take<PI>(lds + Lds::cols, CP, m * (C / 32) + ks, at), xp[ks], s[m]);
      }
    }
  }
  if (ds0 && mine)
#pragma unroll
    for (int m = 0; m < DK / 16; ++m)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int d = m * 16 + g * 4 + r;
        if (d < p.dk) ds0[(bh * p.dk + d) * p.dv + col] = s[m][r];
      }
}

// `rows` rows of 32 values as operands in LDS, part by part, lane m + 16 g of a piece
// at (m ^ 4 g) + 16 g; `there` rows and `width` values of a row are there.
template <int P, class T, bool VEC>
__device__ __forceinline__ void stage_slab(const T* x, int64_t stride, int rows, int there, int width, char* out, int tid,
                                           int threads) {
  for (int u = tid; u < rows * 4; u += threads) {
    const int row = u / 4, g = u % 4;
    float v[8];
    load8<T, VEC>(x + (row < there ? row * stride + g * 8 : 0), row < there ? width - g * 8 : 0, v);
    const Op<P> o = op_of<P>(v);
#pragma unroll
    for (int q = 0; q < P; ++q)
      *(bf16x8*)(out + ((q * (rows / 16) + row / 16) * 64 + (row % 16 ^ 4 * g) + 16 * g) * 16) = o.p[q];
  }
}

template <class T, int DK>
struct GradLds {
  static constexpr int C = kChunk<T>, PI = kIn<T>;
  static constexpr int kc = 0, qc = kc + PI * C * DK * 2, s = qc + PI * C * DK * 2, ds = s + kState * DK * 64,
                       z = ds + kState * DK * 64, x = z + kState * C * 64, dy = x + kState * C * 64,
                       sums = dy + PI * C * 64, bytes = sums + (3 * C + C + 16) * 4 + C * 8;
};

struct DeltaGradOut {
  void *dq, *dk;   // packed
  float *ddecay, *drate;
};

// dQ, dK and the gates of a chunk of one key head, its heads one after the other.  A
// wavefront has 16 steps, as rows of its results and as columns of the four products
// z dy', z x', dy z', x z' over the values, whose sums are the operands that multiply
// K and Q.
template <class T, bool VEC, bool VECV, int DK>
__global__ void __launch_bounds__(kChunk<T> * 4)
    k_delta_grad(DeltaArgs p, const T* q, const T* k, const T* dy, const float* decay, const float* rate,
                 const float* states, const float* errors, const float* dstates, const float* xs, DeltaGradOut out) {
  using Lds = GradLds<T, DK>;
  constexpr int C = kChunk<T>, PI = kIn<T>, NT = DK / 16, RT = C / 16, KC = C / 32, threads = C * 4;
  extern __shared__ __align__(16) char lds[];
  float* const sc = (float*)(lds + Lds::sums);   // e, o, b
  float* const dg = sc + 3 * C;                  // gradients of G
  float* const red = dg + C;
  double* const sum = (double*)(red + 16);
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64, g = lane / 16;
  const int at = (lane % 16 ^ g) + 16 * g, as = (lane % 16 ^ 4 * g) + 16 * g;
  const int key_heads = p.heads / p.group;
  const int64_t all = p.batch * key_heads * p.nchunk;
  for (int64_t u = blockIdx.x; u < all; u += gridDim.x) {
    const int64_t chunk = u % p.nchunk, b = u / p.nchunk / key_heads, t0 = chunk * C;
    const int kh = (int)(u / p.nchunk % key_heads);
    const int len = p.lengths ? min(max(p.lengths[b], 0), p.steps) : p.steps;
    const int n = (int)max((int64_t)0, min((int64_t)C, len - t0)), in = (int)min((int64_t)C, p.steps - t0);
    const T *kb = k + b * p.k.b + t0 * p.k.t + kh * p.k.h, *qb = q + b * p.q.b + t0 * p.q.t + kh * p.q.h;
    f32x4 dq[NT], dk[NT];
#pragma unroll
    for (int m = 0; m < NT; ++m) dq[m] = dk[m] = zero4();
    __syncthreads();
    if (n > 0) {
      stage_operands<T, VEC, C, DK, false, true>(kb, p.k.t, n, p.dk, nullptr, lds + Lds::kc, tid, threads);
      stage_operands<T, VEC, C, DK, false, true>(qb, p.q.t, n, p.dk, nullptr, lds + Lds::qc, tid, threads);
    }
    for (int h = 0; h < p.group; ++h) {
      const int head = kh * p.group + h;
      const int64_t bh = b * p.heads + head, cell = bh * p.nchunk + chunk, gate = (b * p.steps + t0) * p.heads + head;
      if (n == 0) {
        for (int t = tid; t < in; t += threads) out.ddecay[gate + (int64_t)t * p.heads] = out.drate[gate + (int64_t)t * p.heads] = 0.0f;
        continue;
      }
      bool forgets = false;
      if (tid < C) {
        double d = 0.0;
        float r = 0.0f;
        if (tid < n) {
          const float x = decay[b * p.decay.b + (t0 + tid) * p.decay.t + head * p.decay.h];
          forgets = x < -200.0f;
          d = x < -200.0f ? -200.0 : (double)x;
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
      f32x4 eq[NT], er[NT], ew[NT], zy[RT], zx[RT], yz[RT], xz[RT];
      float inner = 0.0f;   // <dS, S>, this thread's part
#pragma unroll
      for (int m = 0; m < NT; ++m) eq[m] = er[m] = ew[m] = zero4();
#pragma unroll
      for (int m = 0; m < RT; ++m) zy[m] = zx[m] = yz[m] = xz[m] = zero4();
      for (int c0 = 0; c0 < p.dv; c0 += 32) {
        const int width = p.dv - c0;
        __syncthreads();
        stage_slab<kState, float, VECV>(states + cell * p.dk * p.dv + c0, p.dv, DK, p.dk, width, lds + Lds::s, tid, threads);
        stage_slab<kState, float, VECV>(dstates + cell * p.dk * p.dv + c0, p.dv, DK, p.dk, width, lds + Lds::ds, tid, threads);
        stage_slab<kState, float, VECV>(errors + cell * C * p.dv + c0, p.dv, C, n, width, lds + Lds::z, tid, threads);
        stage_slab<kState, float, VECV>(xs + cell * C * p.dv + c0, p.dv, C, n, width, lds + Lds::x, tid, threads);
        stage_slab<PI, T, VECV>(dy + b * p.y.b + t0 * p.y.t + head * p.y.h + c0, p.y.t, C, n, width, lds + Lds::dy, tid, threads);
        for (int w = tid; w < p.dk * 4; w += threads) {
          float x[8], y[8];
          const int64_t from = (cell * p.dk + w / 4) * p.dv + c0 + w % 4 * 8;
          const int there = width - w % 4 * 8;
          load8<float, VECV>(states + (there > 0 ? from : 0), there, x);
          load8<float, VECV>(dstates + (there > 0 ? from : 0), there, y);
#pragma unroll
          for (int j = 0; j < 8; ++j) inner = fmaf(x[j], y[j], inner);
        }
        __syncthreads();
        const Op<kState> zo = op_take<kState>(lds + Lds::z, RT, wave, as), xo = op_take<kState>(lds + Lds::x, RT, wave, as);
        const Op<PI> yo = op_take<PI>(lds + Lds::dy, RT, wave, as);
#pragma unroll
        for (int m = 0; m < NT; ++m) {
          const Op<kState> so = op_take<kState>(lds + Lds::s, NT, m, as), go = op_take<kState>(lds + Lds::ds, NT, m, as);
          eq[m] = op_mul<kState>(yo, so, eq[m]);
          er[m] = op_mul<kState>(xo, so, er[m]);
          ew[m] = op_mul<kState>(zo, go, ew[m]);
        }
#pragma unroll
        for (int m = 0; m < RT; ++m) {
          const Op<kState> za = op_take<kState>(lds + Lds::z, RT, m, as);
          if (m <= wave) {
            zy[m] = op_mul<kState>(za, yo, zy[m]);
            zx[m] = op_mul<kState>(za, xo, zx[m]);
          }
          if (m >= wave) {
            yz[m] = op_mul<kState>(op_take<PI>(lds + Lds::dy, RT, m, as), zo, yz[m]);
            xz[m] = op_mul<kState>(op_take<kState>(lds + Lds::x, RT, m, as), zo, xz[m]);
          }
        }
      }
      // this lane's column of the four products is step `own`
      const int own = wave * 16 + lane % 16;
      const double here = sum[own];
#pragma unroll
      for (int m = 0; m < RT; ++m)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int t = m * 16 + g * 4 + r;
          const float before = t <= own ? __builtin_amdgcn_exp2f((float)(here - sum[t])) * sc[2 * C + t] : 0.0f;
          const float after = t >= own ? __builtin_amdgcn_exp2f((float)(sum[t] - here)) : 0.0f;
          zy[m][r] = t <= own ? zy[m][r] * before * p.scale : 0.0f;
          zx[m][r] = t < own ? zx[m][r] * before : 0.0f;
          yz[m][r] = t >= own ? yz[m][r] * after * p.scale : 0.0f;
          xz[m][r] = t > own ? -xz[m][r] * after : 0.0f;
        }
      float end = 0.0f;   // o[t] b[t] k[t] dS z[t], this lane's part: <dS, K' diag(o b) Z>
      float rows[4], wk[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) rows[r] = wk[r] = 0.0f;
      const f32x4 re = *(const f32x4*)(sc + wave * 16 + g * 4), ro = *(const f32x4*)(sc + C + wave * 16 + g * 4),
                  rb = *(const f32x4*)(sc + 2 * C + wave * 16 + g * 4);
      Op<kState> zyp[KC], zxp[KC], yzp[KC], xzp[KC];
#pragma unroll
      for (int ks = 0; ks < KC; ++ks) {
        zyp[ks] = op_of<kState>(zy[2 * ks], zy[2 * ks + 1]);
        zxp[ks] = op_of<kState>(zx[2 * ks], zx[2 * ks + 1]);
        yzp[ks] = op_of<kState>(yz[2 * ks], yz[2 * ks + 1]);
        xzp[ks] = op_of<kState>(xz[2 * ks], xz[2 * ks + 1]);
      }
#pragma unroll
      for (int m = 0; m < NT; ++m) {
        float kv[4], qv[4];
        const int d = m * 16 + lane % 16;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int t = wave * 16 + g * 4 + r;
          const bool there = t < n && d < p.dk;
          kv[r] = there ? as_f32(kb[t * p.k.t + d]) : 0.0f;
          qv[r] = there ? as_f32(qb[t * p.q.t + d]) : 0.0f;
          eq[m][r] = share_of(re[r], eq[m][r]) * p.scale;
          er[m][r] = share_of(re[r], er[m][r]);
          ew[m][r] = share_of(ro[r], ew[m][r]);
          end = fmaf(rb[r] * kv[r], ew[m][r], end);
        }
#pragma unroll
        for (int ks = 0; ks < KC; ++ks) {
          const Op<PI> kc = op_take<PI>(lds + Lds::kc, NT * KC, m * KC + ks, at), qc = op_take<PI>(lds + Lds::qc, NT * KC, m * KC + ks, at);
          if (ks <= wave / 2) {
            eq[m] = op_mul<kState>(zyp[ks], kc, eq[m]);
            er[m] = op_mul<kState>(zxp[ks], kc, er[m]);
          }
          if (ks >= wave / 2) {
            ew[m] = op_mul<kState>(yzp[ks], qc, ew[m]);
            ew[m] = op_mul<kState>(xzp[ks], kc, ew[m]);
          }
        }
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
      if (lane == 0) red[wave] = inner;
      if (lane % 16 == 0)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int t = wave * 16 + g * 4 + r;
          dg[t] = rows[r] - rb[r] * wk[r];
          if (t < in) out.drate[gate + (int64_t)t * p.heads] = t < n ? wk[r] : 0.0f;
        }
      __syncthreads();
      if (tid < C) {
        float s = dg[tid];
        if (tid == C - 1)
          for (int w = 0; w < threads / 64; ++w) s += red[w];
#pragma unroll
        for (int o = 1; o < C; o *= 2) {
          const float x = __shfl_down(s, o, 64);
          if (tid + o < C) s += x;
        }
        if (tid < in) out.ddecay[gate + (int64_t)tid * p.heads] = tid < n && !forgets ? s : 0.0f;
      }
    }
    T* const dqb = (T*)out.dq + ((b * p.steps + t0) * key_heads + kh) * p.dk;
    T* const dkb = (T*)out.dk + ((b * p.steps + t0) * key_heads + kh) * p.dk;
#pragma unroll
    for (int m = 0; m < NT; ++m)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int t = wave * 16 + g * 4 + r, d = m * 16 + lane % 16;
        if (t < in && d < p.dk) {
          dqb[(int64_t)t * key_heads * p.dk + d] = (T)dq[m][r];
          dkb[(int64_t)t * key_heads * p.dk + d] = (T)dk[m][r];
        }
      }
  }
}
