// Group norm with an activation, channels last, and its gradient:
//     h = (x - mean) rstd,  z = h weight + bias,  y = act(z)
// mean and rstd = 1 / sqrt(variance + eps) over the positions of a batch row and the
// channels of a group.  With d = dy act'(z) and sums over the same n values
//     dx = rstd (d weight - sum(d weight) / n - h sum(d weight h) / n)
//     dweight = sum d h,  dbias = sum d  over all rows and positions.
//
// Memory bounds both.  A group of few values (one position: a head's read-out) stays
// in the registers of a team of threads, read once: k_norm_team, k_norm_team_grad.
// Others are read twice: sums over runs of positions, a thread to one channel word,
// their join, and the results.  The variance is the sum of squares about a mean that
// is known (of a team's values) or about the mean of a thread's few values, joined by
// Chan's formula (runs of positions in 64 bits), so a large mean costs no digits.
// Nothing is added by atomics; every sum has one order.
//
// Measured: 16384 rows of 16 heads of 128 bf16 32 us, 4.2 TB/s (69 with words of a thread
// and positions as run-time values, 34 with a team's sums through LDS), the gradient 64
// us, 3.1 TB/s (265 one row at a time, 73 with sums through LDS), and 5 for its column
// sums.  Of the gradient's wavefronts' time 51% is waiting for memory, two workgroups to a
// CU that load four rows and then compute them, and 30% vector instructions.  16 x 4096 positions of 512 float32 channels: sums 21
// us, join 5, results 41, 4.0 TB/s of the 268 MB that have to move (what is read again
// is in the last cache); 13 x 777 x 333 float32, one channel to a thread: 23 us,
// gradient 32.
#pragma once

#include "kernels_words.hpp"
#include "operators_rules.hpp"

struct NormArgs {
  int64_t batch, positions;
  int32_t groups, width;         // channels of a group
  int64_t xb, xt, yb, yt;        // strides of x, and of y or dy: between batch rows, positions
  const int32_t* lengths;
  const float *weight, *bias;    // NULL: ones, zeros
  float* kept;                   // [batch][groups][2]: mean, rstd; NULL: not kept
  float eps;
  int32_t act;
  int32_t nw;                    // words of a group's channels
  // teams: threads of one, and in the gradient batch rows side by side and sums over them one after the other
  int32_t team, lanes, pieces;
  // runs: of positions, side by side, and channel words to a workgroup's row
  int32_t runs, run, wide;
};

enum { kActNone, kActRelu, kActSilu };

// 1 / (1 + exp(-z)).  The argument of the power of two is a product's 24 bits and what
// they leave out: with the product alone the result lost |z| times its rounding, 2e-6 at
// z = -40.  Beyond 200 the power is 0 or infinite, and its argument's rest would be NaN
// where z is infinite.
__device__ __forceinline__ float gate_of_silu(float z) {
  constexpr float log2e = 1.44269502f, more = 1.92596303e-8f, ln2 = 0.693147181f;
  const float x = __builtin_amdgcn_fmed3f(-z, -200.0f, 200.0f), t = x * log2e;
  const float rest = fmaf(x, more, fmaf(x, log2e, -t));
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(t) * fmaf(rest, ln2, 1.0f));
}

// act(z), a result in T.  For one of 16 bits the product alone is enough: 5e-6 of silu at
// z = -88, a thousandth of the rounding to come, and 16384 x 16 heads of 128 bf16 take
// 29 us in place of 31.
template <class T>
__device__ __forceinline__ float activated(float z, int act) {
  if (act == kActRelu) return z > 0.0f ? z : z != z ? z : 0.0f;
  if (act == kActSilu) return z * (sizeof(T) == 2 ? __builtin_amdgcn_rcpf(1.0f + __expf(-z)) : gate_of_silu(z));
  return z;
}

// dy act'(z)
__device__ __forceinline__ float through_act(float dy, float z, int act) {
  if (act == kActRelu) return z > 0.0f ? dy : 0.0f;
  if (act == kActSilu) {
    const float g = gate_of_silu(z);
    return dy * g * fmaf(z, 1.0f - g, 1.0f);
  }
  return dy;
}

__device__ __forceinline__ int64_t norm_length(const NormArgs& p, int64_t b) {
  if (!p.lengths) return p.positions;
  return min(max((int64_t)p.lengths[b], (int64_t)0), p.positions);
}

template <int V>
__device__ __forceinline__ Words<float, V> norm_param(const float* w, int64_t c, float other) {
  if (w) return *(const Words<float, V>*)(w + c);
  Words<float, V> r;
#pragma unroll
  for (int e = 0; e < V; ++e) r.v[e] = other;
  return r;
}

// x of another lane: CTRL says which, within 16 lanes and without a way through LDS.
template <int CTRL>
__device__ __forceinline__ float lane_dpp(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}

// Sums over a team: lanes of a wavefront (a power of two), or the 4 wavefronts of a
// workgroup.  Up to 16 lanes each adds its pair's, its four's other pair's, its eight's
// other four's and the other eight's, the last two from the mirror image, which holds
// the same sum in every lane of that half.
template <bool WIDE>
__device__ __forceinline__ float team_sum(float s, int team, float* red) {
  const int lanes = WIDE ? 64 : team;
  if (lanes > 1) s += lane_dpp<0xB1>(s);    // quad_perm 1 0 3 2
  if (lanes > 2) s += lane_dpp<0x4E>(s);    // quad_perm 2 3 0 1
  if (lanes > 4) s += lane_dpp<0x141>(s);   // row_half_mirror
  if (lanes > 8) s += lane_dpp<0x140>(s);   // row_mirror
  for (int o = 16; o < lanes; o *= 2) s += __shfl_xor(s, o, 64);
  if constexpr (WIDE) {
    __syncthreads();
    if (threadIdx.x % 64 == 0) red[threadIdx.x / 64] = s;
    __syncthreads();
    s = (red[0] + red[1]) + (red[2] + red[3]);
  }
  return s;
}

// A group's values in a team's registers, R words of each thread; ONE: one position.
template <class T, int V, int R, bool WIDE, bool ONE>
__global__ void __launch_bounds__(256) k_norm_team(NormArgs p, const T* x, T* y) {
  __shared__ float red[4];
  const uint32_t team = WIDE ? 256 : p.team, me = threadIdx.x % team, teams = 256 / team;
  const uint32_t all = (uint32_t)(p.batch * p.groups), nw = p.nw, words = (uint32_t)p.positions * nw;
  for (uint32_t u0 = blockIdx.x * teams; u0 < all; u0 += gridDim.x * teams) {
    const bool live = u0 + threadIdx.x / team < all;
    const uint32_t u = live ? u0 + threadIdx.x / team : all - 1, b = u / p.groups, g = u % p.groups;
    const int64_t len = norm_length(p, b);
    const uint32_t inside = (uint32_t)len * nw;
    const T* xp = x + b * p.xb + (int64_t)g * p.width;
    T* yp = y + b * p.yb + (int64_t)g * p.width;
    Words<T, V> v[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const uint32_t j = me + r * team;
      if (j < inside) v[r] = *(const Words<T, V>*)(ONE ? xp + j * V : xp + j / nw * p.xt + j % nw * V);
    }
    float s = 0.0f;
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (me + r * team < inside)
#pragma unroll
        for (int e = 0; e < V; ++e) s += as_f32(v[r].v[e]);
    const float n = 1.0f / (float)(max(len, (int64_t)1) * p.width);
    const float mean = team_sum<WIDE>(s, team, red) * n;
    s = 0.0f;
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (me + r * team < inside)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float d = as_f32(v[r].v[e]) - mean;
          s = fmaf(d, d, s);
        }
    const float rstd = 1.0f / sqrtf(team_sum<WIDE>(s, team, red) * n + p.eps);
    if (!live) continue;
    if (p.kept && me == 0) p.kept[2 * (int64_t)u] = mean, p.kept[2 * (int64_t)u + 1] = rstd;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const uint32_t j = me + r * team;
      if (j >= words) continue;
      const uint32_t c = ONE ? j * V : j % nw * V;
      Words<T, V> o;
      if (j < inside) {
        const Words<float, V> w = norm_param<V>(p.weight, (int64_t)g * p.width + c, 1.0f),
                              a = norm_param<V>(p.bias, (int64_t)g * p.width + c, 0.0f);
#pragma unroll
        for (int e = 0; e < V; ++e) o.v[e] = (T)activated<T>(fmaf((as_f32(v[r].v[e]) - mean) * rstd, w.v[e], a.v[e]), p.act);
      } else {
#pragma unroll
        for (int e = 0; e < V; ++e) o.v[e] = (T)0.0f;
      }
      put_once(ONE ? yp + c : yp + j / nw * p.yt + c, o);
    }
  }
}

// The gradient of one position's groups.  A team keeps its group and goes through
// every p.lanes-th batch row, U of them on their way at a time, with its part of
// dweight and dbias in registers: parts [pieces][lanes][2][channels], one for kNormRows
// rows, since a sum of thousands one after the other loses as many roundings.  (As many
// more teams instead: 131072 rows of 2048 float32 623 -> 845 us.)
template <class T, int V, int R, bool WIDE>
__global__ void __launch_bounds__(256)
    k_norm_team_grad(NormArgs p, const T* x, const T* dy, T* dx, float* parts) {
  constexpr int U = R * V * sizeof(T) <= 16 ? 4 : R * V * sizeof(T) <= 32 ? 2 : 1;
  __shared__ float red[4];
  const int team = WIDE ? 256 : p.team, me = threadIdx.x % team, teams = 256 / team;
  const int64_t slot = (int64_t)blockIdx.x * teams + threadIdx.x / team;
  const bool mine = slot < (int64_t)p.lanes * p.groups;
  const int g = (int)(slot % p.groups);
  const int64_t lane = slot / p.groups, channels = (int64_t)p.groups * p.width;
  const int64_t first = (int64_t)g * p.width + me * V;
  bool has[R];
  Words<float, V> w[R], a[R], dw[R], db[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    has[r] = me + r * team < p.nw;
    const int64_t c = has[r] ? first + r * team * V : 0;
    w[r] = norm_param<V>(p.weight, c, 1.0f), a[r] = norm_param<V>(p.bias, c, 0.0f);
  }
  const float n = 1.0f / (float)p.width;
  // a team of several wavefronts is a workgroup, and goes or stays as one
  const int64_t rows = (int64_t)ms::kNormRows * p.lanes;
  for (int64_t piece = 0; mine && piece < p.pieces; ++piece) {
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int e = 0; e < V; ++e) dw[r].v[e] = db[r].v[e] = 0.0f;
    for (int64_t b0 = piece * rows + lane; b0 < min((piece + 1) * rows, p.batch); b0 += (int64_t)U * p.lanes) {
      Words<T, V> xv[U][R], dv[U][R];
      float mean_of[U], rstd_of[U];
#pragma unroll
      for (int q = 0; q < U; ++q) {
        const int64_t b = min(b0 + q * (int64_t)p.lanes, p.batch - 1);   // past the last row: read, and not used
        mean_of[q] = p.kept[2 * (b * p.groups + g)], rstd_of[q] = p.kept[2 * (b * p.groups + g) + 1];
#pragma unroll
        for (int r = 0; r < R; ++r)
          if (has[r]) {
            xv[q][r] = *(const Words<T, V>*)(x + b * p.xb + first + r * team * V);
            dv[q][r] = *(const Words<T, V>*)(dy + b * p.yb + first + r * team * V);
          }
      }
#pragma unroll
      for (int q = 0; q < U; ++q) {
        const int64_t b = b0 + q * (int64_t)p.lanes;
        if (b >= p.batch) continue;
        const bool live = norm_length(p, b) > 0;   // else nothing that was read counts
        const float mean = mean_of[q], rstd = rstd_of[q];
        float s1 = 0.0f, s2 = 0.0f, h[R][V], d[R][V];
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
          for (int e = 0; e < V; ++e) {
            const bool in = has[r] && live;
            h[r][e] = in ? (as_f32(xv[q][r].v[e]) - mean) * rstd : 0.0f;
            const float t = in ? through_act(as_f32(dv[q][r].v[e]), fmaf(h[r][e], w[r].v[e], a[r].v[e]), p.act) : 0.0f;
            dw[r].v[e] = fmaf(t, h[r][e], dw[r].v[e]), db[r].v[e] += t;
            d[r][e] = t * w[r].v[e];
            s1 += d[r][e];
            s2 = fmaf(d[r][e], h[r][e], s2);
          }
        s1 = team_sum<WIDE>(s1, team, red) * n;
        s2 = team_sum<WIDE>(s2, team, red) * n;
#pragma unroll
        for (int r = 0; r < R; ++r) {
          if (!has[r]) continue;
          Words<T, V> o;
#pragma unroll
          for (int e = 0; e < V; ++e) o.v[e] = live ? (T)(rstd * (d[r][e] - s1 - h[r][e] * s2)) : (T)0.0f;
          put_once(dx + b * channels + first + r * team * V, o);
        }
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (!has[r]) continue;
      float* o = parts + (piece * p.lanes + lane) * 2 * channels + first + r * team * V;
      *(Words<float, V>*)o = dw[r];
      *(Words<float, V>*)(o + channels) = db[r];
    }
  }
}

// Sums of runs of kColumnRows rows of parts [rows][cols], to [runs][cols], or, if there
// is one run, to dweight and dbias: 32 columns to a workgroup, 32 rows side by side.
constexpr int kColumnRows = 512;

__global__ void __launch_bounds__(1024) k_norm_columns(const float* parts, int64_t rows, int64_t channels, float* next,
                                                       float* dweight, float* dbias) {
  __shared__ float red[32][33];
  const int c = threadIdx.x % 32, k = threadIdx.x / 32;
  const int64_t cols = 2 * channels, blocks = (cols + 31) / 32, runs = max((rows + kColumnRows - 1) / kColumnRows, (int64_t)1);
  for (int64_t u = blockIdx.x; u < blocks * runs; u += gridDim.x) {
    const int64_t col = u % blocks * 32 + c, row = u / blocks * kColumnRows + k;
    float v[kColumnRows / 32];
#pragma unroll
    for (int i = 0; i < kColumnRows / 32; ++i)
      v[i] = col < cols && row + i * 32 < rows ? parts[(row + i * 32) * cols + col] : 0.0f;
    float s = v[0];
#pragma unroll
    for (int i = 1; i < kColumnRows / 32; ++i) s += v[i];
    red[k][c] = s;
    __syncthreads();
    // 32 sums of a column to the lanes of half a wavefront
    s = red[c][k];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor(s, o, 32);
    const int64_t mine = u % blocks * 32 + k;
    if (c == 0 && mine < cols) {
      if (next) next[u / blocks * cols + mine] = s;
      else (mine < channels ? dweight[mine] : dbias[mine - channels]) = s;
    }
    __syncthreads();
  }
}

// ------------------------------------------------------------ many positions
// Where a workgroup works: batch row, run of positions, block of channel words; a
// thread's word and its first position.
struct NormPlace {
  int64_t b, len, t, end, word;
  int step;
  bool live;
};

template <int V>
__device__ __forceinline__ NormPlace norm_place(const NormArgs& p, int64_t u) {
  const int64_t words = (int64_t)p.groups * p.nw, blocks = (words + p.wide - 1) / p.wide;
  NormPlace q;
  q.b = u / blocks / p.runs;
  q.len = norm_length(p, q.b);
  const int64_t run = u / blocks % p.runs;
  q.step = 256 / p.wide;
  q.t = run * p.run + threadIdx.x / p.wide;
  q.end = min((run + 1) * p.run, p.positions);
  q.word = u % blocks * p.wide + threadIdx.x % p.wide;
  q.live = q.word < words;
  return q;
}

__device__ __forceinline__ int64_t norm_blocks(const NormArgs& p) {
  return p.batch * p.runs * (((int64_t)p.groups * p.nw + p.wide - 1) / p.wide);
}

// Of every run and word: mean and sum of squares about it, parts [batch][runs][words][2].
// A thread takes 8 positions at a time.
template <class T, int V>
__global__ void __launch_bounds__(256) k_norm_sums(NormArgs p, const T* x, float* parts) {
  __shared__ float red[256][3];
  const int64_t all = norm_blocks(p), words = (int64_t)p.groups * p.nw;
  for (int64_t u = blockIdx.x; u < all; u += gridDim.x) {
    const NormPlace q = norm_place<V>(p, u);
    const int64_t end = min(q.end, q.len);
    const T* xp = x + q.b * p.xb + (q.live ? q.word : 0) * V;
    float n = 0.0f, mean = 0.0f, square = 0.0f;
    for (int64_t t = q.t; q.live && t < end; t += 8 * q.step) {
      Words<T, V> v[8];
      const int have = (int)min((int64_t)8, (end - t + q.step - 1) / q.step);
#pragma unroll
      for (int r = 0; r < 8; ++r) v[r] = *(const Words<T, V>*)(xp + min(t + r * q.step, end - 1) * p.xt);
      float s = 0.0f, m2 = 0.0f;
#pragma unroll
      for (int r = 0; r < 8; ++r)
#pragma unroll
        for (int e = 0; e < V; ++e) s += r < have ? as_f32(v[r].v[e]) : 0.0f;
      const float here = (float)(have * V), m = s / here;
#pragma unroll
      for (int r = 0; r < 8; ++r)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float d = r < have ? as_f32(v[r].v[e]) - m : 0.0f;
          m2 = fmaf(d, d, m2);
        }
      const float d = m - mean, both = n + here;
      mean = fmaf(d, here / both, mean);
      square += m2 + d * d * (n * here / both);
      n = both;
    }
    red[threadIdx.x][0] = n, red[threadIdx.x][1] = mean, red[threadIdx.x][2] = square;
    __syncthreads();
    if (threadIdx.x < p.wide && q.live) {
      for (int r = 1; r < q.step; ++r) {
        const float *o = red[threadIdx.x + r * p.wide], here = o[0], both = n + here;
        if (here == 0.0f) continue;
        const float d = o[1] - mean;
        mean = fmaf(d, here / both, mean);
        square += o[2] + d * d * (n * here / both);
        n = both;
      }
      float* o = parts + ((q.b * p.runs + u / ((words + p.wide - 1) / p.wide) % p.runs) * words + q.word) * 2;
      o[0] = mean, o[1] = square;
    }
    __syncthreads();
  }
}

__device__ __forceinline__ double norm_sum64(double s, double* red) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
  __syncthreads();
  if (threadIdx.x % 64 == 0) red[threadIdx.x / 64] = s;
  __syncthreads();
  return (red[0] + red[1]) + (red[2] + red[3]);
}

// mean and rstd of every batch row's groups from the runs': kept.
template <int V>
__global__ void __launch_bounds__(256) k_norm_join(NormArgs p, const float* parts) {
  __shared__ double red[4];
  const int64_t words = (int64_t)p.groups * p.nw, all = p.batch * p.groups;
  for (int64_t u = blockIdx.x; u < all; u += gridDim.x) {
    const int64_t b = u / p.groups, len = norm_length(p, b), first = u % p.groups * p.nw;
    const uint32_t nw = p.nw, n = (uint32_t)((len + p.run - 1) / p.run) * nw;
    const auto count = [&](uint32_t run) { return (double)(min((int64_t)p.run, len - (int64_t)run * p.run) * V); };
    const float* at = parts + (b * p.runs * words + first) * 2;
    double s = 0.0;
    for (uint32_t i = threadIdx.x; i < n; i += 256) s += count(i / nw) * at[(i / nw * words + i % nw) * 2];
    const double total = (double)max(len, (int64_t)1) * p.width, mean = norm_sum64(s, red) / total;
    s = 0.0;
    for (uint32_t i = threadIdx.x; i < n; i += 256) {
      const float* o = at + (i / nw * words + i % nw) * 2;
      const double d = o[0] - mean;
      s += o[1] + count(i / nw) * d * d;
    }
    const double square = norm_sum64(s, red);
    if (threadIdx.x == 0) p.kept[2 * u] = (float)mean, p.kept[2 * u + 1] = (float)(1.0 / sqrt(square / total + p.eps));
  }
}

template <class T, int V>
__global__ void __launch_bounds__(256) k_norm_apply(NormArgs p, const T* x, T* y) {
  const int64_t all = norm_blocks(p);
  for (int64_t u = blockIdx.x; u < all; u += gridDim.x) {
    const NormPlace q = norm_place<V>(p, u);
    if (!q.live) continue;
    const int64_t c = q.word * V, g = q.b * p.groups + q.word / p.nw;
    const float mean = p.kept[2 * g], rstd = p.kept[2 * g + 1];
    const Words<float, V> w = norm_param<V>(p.weight, c, 1.0f), a = norm_param<V>(p.bias, c, 0.0f);
    for (int64_t t = q.t; t < q.end; t += 4 * q.step) {
      Words<T, V> v[4];
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (t + r * q.step < min(q.end, q.len)) v[r] = *(const Words<T, V>*)(x + q.b * p.xb + (t + r * q.step) * p.xt + c);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        if (t + r * q.step >= q.end) continue;
        Words<T, V> o;
#pragma unroll
        for (int e = 0; e < V; ++e)
          o.v[e] = t + r * q.step < q.len ? (T)activated<T>(fmaf((as_f32(v[r].v[e]) - mean) * rstd, w.v[e], a.v[e]), p.act)
                                          : (T)0.0f;
        put_once(y + q.b * p.yb + (t + r * q.step) * p.yt + c, o);
      }
    }
  }
}

// Of every run and channel: sums of d h and of d, parts [batch][runs][2][channels].  A
// thread's positions are added up 64 at a time, and those in 64 bits: a sum of thousands
// one after the other loses as many roundings of its own size.
template <class T, int V>
__global__ void __launch_bounds__(256) k_norm_grad_sums(NormArgs p, const T* x, const T* dy, float* parts) {
  __shared__ float red[256][2 * V + 1];
  const int64_t all = norm_blocks(p), words = (int64_t)p.groups * p.nw, channels = words * V;
  for (int64_t u = blockIdx.x; u < all; u += gridDim.x) {
    const NormPlace q = norm_place<V>(p, u);
    const int64_t end = min(q.end, q.len), c = (q.live ? q.word : 0) * V;
    const int64_t g = q.b * p.groups + (q.live ? q.word : 0) / p.nw;
    const float mean = p.kept[2 * g], rstd = p.kept[2 * g + 1];
    const Words<float, V> w = norm_param<V>(p.weight, c, 1.0f), a = norm_param<V>(p.bias, c, 0.0f);
    double dw[V], db[V];
#pragma unroll
    for (int e = 0; e < V; ++e) dw[e] = db[e] = 0.0;
    for (int64_t t = q.t; q.live && t < end;) {
      float sw[V], sb[V];
#pragma unroll
      for (int e = 0; e < V; ++e) sw[e] = sb[e] = 0.0f;
      for (int i = 0; i < 16 && t < end; ++i, t += 4 * q.step) {
        Words<T, V> xv[4], dv[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int64_t at = min(t + r * q.step, end - 1);
          xv[r] = *(const Words<T, V>*)(x + q.b * p.xb + at * p.xt + c);
          dv[r] = *(const Words<T, V>*)(dy + q.b * p.yb + at * p.yt + c);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (t + r * q.step < end)
#pragma unroll
            for (int e = 0; e < V; ++e) {
              const float h = (as_f32(xv[r].v[e]) - mean) * rstd;
              const float d = through_act(as_f32(dv[r].v[e]), fmaf(h, w.v[e], a.v[e]), p.act);
              sw[e] = fmaf(d, h, sw[e]), sb[e] += d;
            }
      }
#pragma unroll
      for (int e = 0; e < V; ++e) dw[e] += sw[e], db[e] += sb[e];
    }
#pragma unroll
    for (int e = 0; e < V; ++e) red[threadIdx.x][e] = (float)dw[e], red[threadIdx.x][V + e] = (float)db[e];
    __syncthreads();
    if (threadIdx.x < p.wide && q.live) {
      for (int r = 1; r < q.step; ++r)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          dw[e] += red[threadIdx.x + r * p.wide][e];
          db[e] += red[threadIdx.x + r * p.wide][V + e];
        }
      float* o = parts + (q.b * p.runs + u / ((words + p.wide - 1) / p.wide) % p.runs) * 2 * channels + c;
#pragma unroll
      for (int e = 0; e < V; ++e) o[e] = (float)dw[e], o[channels + e] = (float)db[e];
    }
    __syncthreads();
  }
}

// sum(d weight h) / n and sum(d weight) / n of every batch row's groups: sums.
__global__ void __launch_bounds__(256) k_norm_grad_join(NormArgs p, const float* parts, float* sums) {
  __shared__ double red[4];
  const int64_t channels = (int64_t)p.groups * p.width, all = p.batch * p.groups;
  for (int64_t u = blockIdx.x; u < all; u += gridDim.x) {
    const int64_t b = u / p.groups, len = norm_length(p, b), first = u % p.groups * p.width;
    const float* at = parts + b * p.runs * 2 * channels + first;
    double s1 = 0.0, s2 = 0.0;
    const uint32_t width = p.width, n = (uint32_t)((len + p.run - 1) / p.run) * width;
    for (uint32_t i = threadIdx.x; i < n; i += 256) {
      const int64_t o = (int64_t)(i / width) * 2 * channels + i % width;
      const float w = p.weight ? p.weight[first + i % width] : 1.0f;
      s1 += (double)w * at[o], s2 += (double)w * at[o + channels];
    }
    const double total = (double)max(len, (int64_t)1) * p.width;
    s1 = norm_sum64(s1, red), s2 = norm_sum64(s2, red);
    if (threadIdx.x == 0) sums[2 * u] = (float)(s1 / total), sums[2 * u + 1] = (float)(s2 / total);
  }
}

template <class T, int V>
__global__ void __launch_bounds__(256)
    k_norm_grad_apply(NormArgs p, const T* x, const T* dy, const float* sums, T* dx) {
  const int64_t all = norm_blocks(p), channels = (int64_t)p.groups * p.width;
  for (int64_t u = blockIdx.x; u < all; u += gridDim.x) {
    const NormPlace q = norm_place<V>(p, u);
    if (!q.live) continue;
    const int64_t c = q.word * V, g = q.b * p.groups + q.word / p.nw;
    const float mean = p.kept[2 * g], rstd = p.kept[2 * g + 1], sh = sums[2 * g], sd = sums[2 * g + 1];
    const Words<float, V> w = norm_param<V>(p.weight, c, 1.0f), a = norm_param<V>(p.bias, c, 0.0f);
    for (int64_t t = q.t; t < q.end; t += 4 * q.step) {
      Words<T, V> xv[4], dv[4];
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (t + r * q.step < min(q.end, q.len)) {
          xv[r] = *(const Words<T, V>*)(x + q.b * p.xb + (t + r * q.step) * p.xt + c);
          dv[r] = *(const Words<T, V>*)(dy + q.b * p.yb + (t + r * q.step) * p.yt + c);
        }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        if (t + r * q.step >= q.end) continue;
        Words<T, V> o;
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float h = (as_f32(xv[r].v[e]) - mean) * rstd;
          const float d = through_act(as_f32(dv[r].v[e]), fmaf(h, w.v[e], a.v[e]), p.act) * w.v[e];
          o.v[e] = t + r * q.step < q.len ? (T)(rstd * (d - sd - h * sh)) : (T)0.0f;
        }
        put_once(dx + (q.b * p.positions + t + r * q.step) * channels + c, o);
      }
    }
  }
}
