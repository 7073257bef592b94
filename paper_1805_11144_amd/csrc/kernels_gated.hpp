// The gated lowpass y[t] = a[t] y[t-1] + (1 - a[t]) v[t], a = 1 / (1 + exp(-g)),
// over whole sequences, its gradient, and its single step.
//
// A run of steps maps the state that enters it to the one that leaves it by
// y -> A y + Y, A the product of its a[t] and Y what it leaves from zero, so
// runs can be taken at once and joined: with (A1, Y1) before (A2, Y2) the two
// together are (A1 A2, A2 Y1 + Y2).  Each channel's steps are cut into chunks;
// one kernel leaves every chunk's (A, Y), the next joins those before its own
// and goes through its steps from the state that it finds.  The gradient runs
// the same way from the end: m = a d goes from a step to the one before it, with
// d[t] = dy[t] + m[t+1].
#pragma once

#include "kernels_embed.hpp"

// Steps between the states that the forward pass leaves for the gradient.  The
// gradient computes the states between them again, in registers.
constexpr int kKeep = 16;

// A thread takes V neighbouring channels of one batch row: thread i of the
// grid's x axis is row i / nv and channels (i % nv) V .. + V; blockIdx.y is the
// chunk.
struct GatedArgs {
  int64_t batch, steps, dim, nv;    // nv = dim / V
  int64_t vb, vt, gb, gt, yb, yt;   // strides of v, g and y (dy in the gradient)
  const int32_t* lengths;
  int32_t chunk, nchunk;            // steps per chunk (a multiple of kKeep), chunks
};

__device__ __forceinline__ int32_t row_length(const GatedArgs& p, int64_t b) {
  if (!p.lengths) return (int32_t)p.steps;
  return min(max(p.lengths[b], 0), (int32_t)p.steps);
}

// a and 1 - a from the logit: both to full precision, also where one is small.
__device__ __forceinline__ void gate(float g, float& a, float& rest) {
  const float e = __expf(-fabsf(g));
  const float big = __builtin_amdgcn_rcpf(1.0f + e), small = e * big;
  a = g >= 0.0f ? big : small;
  rest = g >= 0.0f ? small : big;
  if (g != g) a = rest = g;
}

// One step of the filter.
__device__ __forceinline__ float gated_step(float y, float g, float v) {
  float a, r;
  gate(g, a, r);
  return fmaf(a, y, r * v);
}

// (A, Y) of each chunk to join[batch][chunk][2][dim].
template <class T, int V>
__global__ void __launch_bounds__(256) k_gated_part(GatedArgs p, const T* v, const T* g, float* join) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= p.batch * p.nv) return;
  const int64_t b = i / p.nv, c = (i - b * p.nv) * V;
  const int32_t t0 = blockIdx.y * p.chunk, t1 = min(t0 + p.chunk, row_length(p, b));
  float A[V], Y[V];
#pragma unroll
  for (int e = 0; e < V; ++e) A[e] = 1.0f, Y[e] = 0.0f;
  const T *vp = v + b * p.vb + c, *gp = g + b * p.gb + c;
#pragma unroll 8
  for (int32_t t = t0; t < t1; ++t) {
    const Words<T, V> x = *(const Words<T, V>*)(vp + t * p.vt), q = *(const Words<T, V>*)(gp + t * p.gt);
#pragma unroll
    for (int e = 0; e < V; ++e) {
      float a, r;
      gate(as_f32(q.v[e]), a, r);
      A[e] *= a;
      Y[e] = fmaf(a, Y[e], r * as_f32(x.v[e]));
    }
  }
  float* o = join + ((b * p.nchunk + blockIdx.y) * 2) * p.dim + c;
#pragma unroll
  for (int e = 0; e < V; ++e) o[e] = A[e], o[p.dim + e] = Y[e];
}

// The filter's steps of one chunk, from y0 and the chunks before it.
template <class T, int V>
__global__ void __launch_bounds__(256) k_gated(GatedArgs p, const T* v, const T* g, const float* y0, const float* join,
                                               T* y, float* last, float* kept) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= p.batch * p.nv) return;
  const int64_t b = i / p.nv, c = (i - b * p.nv) * V;
  const int32_t len = row_length(p, b);
  const int32_t t0 = blockIdx.y * p.chunk, tend = (int32_t)min((int64_t)t0 + p.chunk, p.steps);
  const int32_t t1 = min(tend, len);
  float h[V];
#pragma unroll
  for (int e = 0; e < V; ++e) h[e] = y0 ? y0[b * p.dim + c + e] : 0.0f;
  const float* j = join + b * p.nchunk * 2 * p.dim + c;
  for (int32_t k = 0; k < (int32_t)blockIdx.y; ++k, j += 2 * p.dim) {
#pragma unroll
    for (int e = 0; e < V; ++e) h[e] = fmaf(j[e], h[e], j[p.dim + e]);
  }
  const T *vp = v + b * p.vb + c, *gp = g + b * p.gb + c;
  T* yp = y + b * p.yb + c;
  float* kp = kept + (b * ((p.steps + kKeep - 1) / kKeep)) * p.dim + c;
#pragma unroll 8
  for (int32_t t = t0; t < t1; ++t) {
    if (kept && t % kKeep == 0) {
#pragma unroll
      for (int e = 0; e < V; ++e) kp[(t / kKeep) * p.dim + e] = h[e];
    }
    const Words<T, V> x = *(const Words<T, V>*)(vp + t * p.vt), q = *(const Words<T, V>*)(gp + t * p.gt);
    Words<T, V> o;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      h[e] = gated_step(h[e], as_f32(q.v[e]), as_f32(x.v[e]));
      o.v[e] = (T)h[e];
    }
    put_once(yp + t * p.yt, o);
  }
  Words<T, V> zero;
#pragma unroll
  for (int e = 0; e < V; ++e) zero.v[e] = (T)0.0f;
  for (int32_t t = max(t0, t1); t < tend; ++t) *(Words<T, V>*)(yp + t * p.yt) = zero;
  // the chunk that holds the row's end (the first one of an empty row)
  if (last && (len == 0 ? t0 == 0 : len > t0 && len <= t0 + p.chunk)) {
#pragma unroll
    for (int e = 0; e < V; ++e) last[b * p.dim + c + e] = h[e];
  }
}

// last of rows without steps.
__global__ void __launch_bounds__(256) k_gated_none(const float* from, float* to, int64_t n) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i < n) to[i] = from ? from[i] : 0.0f;
}

// The gradient's chunk: (A, M) with m = A m' + M for the m' that enters at its end.
template <class T, int V>
__global__ void __launch_bounds__(256) k_gated_grad_part(GatedArgs p, const T* g, const T* dy, float* join) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= p.batch * p.nv) return;
  const int64_t b = i / p.nv, c = (i - b * p.nv) * V;
  const int32_t t0 = blockIdx.y * p.chunk, t1 = min(t0 + p.chunk, row_length(p, b));
  float A[V], M[V];
#pragma unroll
  for (int e = 0; e < V; ++e) A[e] = 1.0f, M[e] = 0.0f;
  const T *gp = g + b * p.gb + c, *dp = dy + b * p.yb + c;
#pragma unroll 8
  for (int32_t t = t1 - 1; t >= t0; --t) {
    const Words<T, V> x = *(const Words<T, V>*)(dp + t * p.yt), q = *(const Words<T, V>*)(gp + t * p.gt);
#pragma unroll
    for (int e = 0; e < V; ++e) {
      float a, r;
      gate(as_f32(q.v[e]), a, r);
      A[e] *= a;
      M[e] = a * (as_f32(x.v[e]) + M[e]);
    }
  }
  float* o = join + ((b * p.nchunk + blockIdx.y) * 2) * p.dim + c;
#pragma unroll
  for (int e = 0; e < V; ++e) o[e] = A[e], o[p.dim + e] = M[e];
}

template <class T, int V>
__global__ void __launch_bounds__(256) k_gated_grad(GatedArgs p, const T* v, const T* g, const float* kept, const T* dy,
                                                    const float* dlast, const float* join, T* dv, T* dg, float* dy0) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= p.batch * p.nv) return;
  const int64_t b = i / p.nv, c = (i - b * p.nv) * V;
  const int32_t t0 = blockIdx.y * p.chunk, tend = (int32_t)min((int64_t)t0 + p.chunk, p.steps);
  const int32_t t1 = min(tend, row_length(p, b));
  float m[V];
#pragma unroll
  for (int e = 0; e < V; ++e) m[e] = dlast ? dlast[b * p.dim + c + e] : 0.0f;
  for (int32_t k = p.nchunk - 1; k > (int32_t)blockIdx.y; --k) {
    const float* j = join + (b * p.nchunk + k) * 2 * p.dim + c;
#pragma unroll
    for (int e = 0; e < V; ++e) m[e] = fmaf(j[e], m[e], j[p.dim + e]);
  }
  const T *vp = v + b * p.vb + c, *gp = g + b * p.gb + c, *dp = dy + b * p.yb + c;
  T *dvp = dv + b * p.steps * p.dim + c, *dgp = dg + b * p.steps * p.dim + c;
  Words<T, V> zero;
#pragma unroll
  for (int e = 0; e < V; ++e) zero.v[e] = (T)0.0f;
  for (int32_t t = max(t0, t1); t < tend; ++t) {
    *(Words<T, V>*)(dvp + t * p.dim) = zero;
    *(Words<T, V>*)(dgp + t * p.dim) = zero;
  }
  const int64_t nkeep = (p.steps + kKeep - 1) / kKeep;
  for (int32_t s0 = t1 > t0 ? (t1 - 1) / kKeep * kKeep : t0 - 1; s0 >= t0; s0 -= kKeep) {
    const int n = min(kKeep, t1 - s0);
    Words<T, V> xv[kKeep], xg[kKeep];
    float before[kKeep][V];   // y[t - 1]
#pragma unroll
    for (int k = 0; k < kKeep; ++k)
      if (k < n) {
        xv[k] = *(const Words<T, V>*)(vp + (s0 + k) * p.vt);
        xg[k] = *(const Words<T, V>*)(gp + (s0 + k) * p.gt);
      }
    float h[V];
#pragma unroll
    for (int e = 0; e < V; ++e) h[e] = kept[(b * nkeep + s0 / kKeep) * p.dim + c + e];
#pragma unroll
    for (int k = 0; k < kKeep; ++k)
      if (k < n) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
          before[k][e] = h[e];
          h[e] = gated_step(h[e], as_f32(xg[k].v[e]), as_f32(xv[k].v[e]));
        }
      }
#pragma unroll
    for (int k = kKeep - 1; k >= 0; --k)
      if (k < n) {
        const Words<T, V> x = *(const Words<T, V>*)(dp + (s0 + k) * p.yt);
        Words<T, V> ov, og;
#pragma unroll
        for (int e = 0; e < V; ++e) {
          float a, r;
          gate(as_f32(xg[k].v[e]), a, r);
          const float d = as_f32(x.v[e]) + m[e];
          ov.v[e] = (T)(r * d);
          og.v[e] = (T)(a * r * (before[k][e] - as_f32(xv[k].v[e])) * d);
          m[e] = a * d;
        }
        put_once(dvp + (s0 + k) * p.dim, ov);
        put_once(dgp + (s0 + k) * p.dim, og);
      }
  }
  if (dy0 && t0 == 0) {
#pragma unroll
    for (int e = 0; e < V; ++e) dy0[b * p.dim + c + e] = m[e];
  }
}

// One step for each served row; `tpr` threads per row (a power of two, at most 256).
template <class T, int V>
__global__ void __launch_bounds__(256) k_gated_served(const T* v, const T* g, float* state, const int32_t* slots, T* y,
                                                      int64_t rows, int64_t n_slots, int32_t nv, int32_t tpr, int64_t vs,
                                                      int64_t gs, int64_t ys, int64_t ss) {
  const int32_t rpb = 256 / tpr;
  for (int64_t i = (int64_t)blockIdx.x * rpb + threadIdx.x / tpr; i < rows; i += (int64_t)gridDim.x * rpb) {
    const int64_t slot = slots ? (int64_t)slots[i] : i;
    const bool idle = slot < 0 || slot >= n_slots;
    for (int32_t k = threadIdx.x % tpr; k < nv; k += tpr) {
      const int64_t c = (int64_t)k * V;
      Words<T, V> o;
      if (idle) {
#pragma unroll
        for (int e = 0; e < V; ++e) o.v[e] = (T)0.0f;
      } else {
        const Words<T, V> x = *(const Words<T, V>*)(v + i * vs + c), q = *(const Words<T, V>*)(g + i * gs + c);
        Words<float, V> h = *(const Words<float, V>*)(state + slot * ss + c);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          h.v[e] = gated_step(h.v[e], as_f32(q.v[e]), as_f32(x.v[e]));
          o.v[e] = (T)h.v[e];
        }
        *(Words<float, V>*)(state + slot * ss + c) = h;
      }
      *(Words<T, V>*)(y + i * ys + c) = o;
    }
  }
}
