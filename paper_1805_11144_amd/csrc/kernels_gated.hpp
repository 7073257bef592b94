// The gated lowpass y[t] = a[t] y[t-1] + (1 - a[t]) v[t], a = 1 / (1 + exp(-g)),
// over whole sequences, its gradient, and its single step.
//
// A run of steps maps the state that enters it to the one that leaves it by
// y -> A y + Y, A the product of its a[t] and Y what it leaves from zero.  The
// gradient runs the same way from the end: m = a d goes from a step to the one
// before it, with d[t] = dy[t] + m[t+1], so a run maps m -> A m + M.
//
// Memory bounds it: each array has to be read or written once, a step costs
// two transcendental instructions and about ten others for its 3 (gradient: 5)
// values.  So every value is read once and stays in registers until its result
// is known.  A wavefront takes kKeep = 16 steps of 64 V channels, fetched
// together; its lanes know their runs' maps, and the wavefronts of a workgroup,
// which hold consecutive runs, join them in LDS.  Sequences longer than a
// workgroup's 128 steps are cut into such chunks.  With enough channels, or a
// few chunks, a workgroup goes through its chunks one after the other (LINK =
// false).  Otherwise the chunks run side by side (LINK): each leaves its map
// for the later ones, and every kSpan-th the state that it ends with; a chunk
// waits for the state at its span's beginning and the maps in between.  The
// order of these operations is fixed, so the result does not depend on timing.
#pragma once

#include "kernels_embed.hpp"

// Steps of a wavefront, and between the states that the forward pass leaves for
// the gradient, which computes the states between them again.
constexpr int kKeep = 16;
constexpr int kSpan = 8;   // chunks from one published state to the next

// A lane takes V neighbouring channels of one batch row: lane i of all is row
// i / nv and channels (i % nv) V .. + V.
struct GatedArgs {
  int64_t batch, steps, dim, nv;    // nv = dim / V
  int64_t vb, vt, gb, gt, yb, yt;   // strides of v, g and y (dy in the gradient)
  const int32_t* lengths;
  int32_t nchunk, groups;           // chunks of blockDim / 64 * kKeep steps; workgroups per chunk
  // LINK: what chunks leave for each other, all ones before the launch
  uint64_t* maps;                   // [nchunk][batch * dim]: (A, Y)
  uint32_t* states;                 // [nchunk / kSpan][batch * dim]
  uint32_t* ticket;
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
}

// One step of the filter.
__device__ __forceinline__ float gated_step(float y, float g, float v) {
  float a, r;
  gate(g, a, r);
  return fmaf(a, y, r * v);
}

// What is published is never all ones, which stands for "not yet": a NaN's bits
// can come from the inputs, so NaN is published as the one of this pattern.
__device__ __forceinline__ uint32_t published(float x) {
  return x != x ? 0x7fc00000u : __builtin_bit_cast(uint32_t, x);
}

__global__ void __launch_bounds__(256) k_gated_clear(uint32_t* words, int64_t n, uint32_t* ticket) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i == 0) *ticket = 0;
  for (int64_t k = i; k < n; k += (int64_t)gridDim.x * 256) words[k] = ~0u;
}

// last (dy0) of rows without steps.
__global__ void __launch_bounds__(256) k_gated_none(const float* from, float* to, int64_t n) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i < n) to[i] = from ? from[i] : 0.0f;
}

// The chunk and the channel group of a workgroup.  Chunks that wait for others
// take theirs in the order in which they start (`order` counts along the
// direction of the recurrence), so a workgroup waits only for such that started
// before it, and these publish their maps without waiting for anyone: every
// wait ends.
struct GatedPlace {
  int32_t order;
  int64_t group;
};

template <bool LINK>
__device__ __forceinline__ GatedPlace gated_place(const GatedArgs& p, uint32_t* box) {
  if (!LINK) return {0, (int64_t)blockIdx.x};
  if (threadIdx.x == 0) *box = __hip_atomic_fetch_add(p.ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  const uint32_t t = __builtin_amdgcn_readfirstlane(*box);
  return {(int32_t)(t / (uint32_t)p.groups), (int64_t)(t % (uint32_t)p.groups)};
}

// The value that enters chunk number `order` for the channels at `at`: `first`
// at the beginning, else from what earlier chunks published.  A, Y: the chunk's
// own map.  Every word is one atomic access of its own, so a word that is there
// is whole; a chunk's words need no order among themselves.
template <int V>
__device__ __forceinline__ void gated_link(const GatedArgs& p, int32_t order, int64_t at, const float* A, const float* Y,
                                           const float* first, float* h) {
  const int64_t channels = p.batch * p.dim;
  const int32_t span = order / kSpan, from = span * kSpan;
  if (order + 1 < p.nchunk) {
#pragma unroll
    for (int e = 0; e < V; ++e)
      __hip_atomic_store(p.maps + order * channels + at + e, (uint64_t)published(Y[e]) << 32 | published(A[e]),
                         __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  uint64_t map[kSpan - 1][V];
  uint32_t state[V];
  bool wait;
  do {
    wait = false;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      state[e] = 0;
      if (span > 0)
        state[e] = __hip_atomic_load(p.states + (span - 1) * channels + at + e, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      wait |= state[e] == ~0u;
    }
#pragma unroll
    for (int k = 0; k < kSpan - 1; ++k)
      if (from + k < order)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          map[k][e] = __hip_atomic_load(p.maps + (from + k) * channels + at + e, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
          wait |= map[k][e] == ~0ull;
        }
    if (wait) __builtin_amdgcn_s_sleep(1);
  } while (wait);
#pragma unroll
  for (int e = 0; e < V; ++e) h[e] = span > 0 ? __builtin_bit_cast(float, state[e]) : first[e];
#pragma unroll
  for (int k = 0; k < kSpan - 1; ++k)
    if (from + k < order)
#pragma unroll
      for (int e = 0; e < V; ++e)
        h[e] = fmaf(__builtin_bit_cast(float, (uint32_t)map[k][e]), h[e],
                    __builtin_bit_cast(float, (uint32_t)(map[k][e] >> 32)));
  if (order % kSpan == kSpan - 1 && order + 1 < p.nchunk) {
#pragma unroll
    for (int e = 0; e < V; ++e)
      __hip_atomic_store(p.states + span * channels + at + e, published(fmaf(A[e], h[e], Y[e])), __ATOMIC_RELAXED,
                         __HIP_MEMORY_SCOPE_AGENT);
  }
}

// A workgroup's runs: each wavefront's map, and what enters the chunk.
template <int V>
struct GatedRuns {
  float A[8][V][64], Y[8][V][64];
};

// The value that enters this wavefront's run.  `run` counts wavefronts along
// the direction of the recurrence; `carry` holds, in wavefront 0 and on its
// own, what enters the next chunk.  Called by all wavefronts.
template <bool LINK, int V>
__device__ __forceinline__ void gated_enter(const GatedArgs& p, GatedRuns<V>& runs, float (*enter)[64], int run, int nrun,
                                            int32_t order, int64_t at, bool live, const float* A, const float* Y,
                                            float* carry, float* h) {
  const int lane = threadIdx.x % 64;
#pragma unroll
  for (int e = 0; e < V; ++e) runs.A[run][e][lane] = A[e], runs.Y[run][e][lane] = Y[e];
  __syncthreads();
  if (run == 0) {
    float cA[V], cY[V];   // the chunk's map
#pragma unroll
    for (int e = 0; e < V; ++e) cA[e] = A[e], cY[e] = Y[e];
    for (int w = 1; w < nrun; ++w)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float a = runs.A[w][e][lane];
        cA[e] *= a;
        cY[e] = fmaf(a, cY[e], runs.Y[w][e][lane]);
      }
    if (LINK && live) gated_link<V>(p, order, at, cA, cY, carry, carry);
#pragma unroll
    for (int e = 0; e < V; ++e) {
      enter[e][lane] = carry[e];
      if (!LINK) carry[e] = fmaf(cA[e], carry[e], cY[e]);
    }
  }
  __syncthreads();
#pragma unroll
  for (int e = 0; e < V; ++e) h[e] = enter[e][lane];
  for (int w = 0; w < run; ++w)
#pragma unroll
    for (int e = 0; e < V; ++e) h[e] = fmaf(runs.A[w][e][lane], h[e], runs.Y[w][e][lane]);
}

template <class T, int V, bool LINK>
__global__ void __launch_bounds__(512) k_gated(GatedArgs p, const T* v, const T* g, const float* y0, T* y, float* last,
                                               float* kept) {
  __shared__ GatedRuns<V> runs[2];
  __shared__ float enter[V][64];
  __shared__ uint32_t box;
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), waves = blockDim.x / 64;
  const GatedPlace place = gated_place<LINK>(p, &box);
  const int64_t i = place.group * 64 + lane;
  const bool live = i < p.batch * p.nv;
  const int64_t b = live ? i / p.nv : 0, c = live ? (i - b * p.nv) * V : 0, at = b * p.dim + c;
  const int32_t len = live ? row_length(p, b) : 0;
  const T *vp = v + b * p.vb + c, *gp = g + b * p.gb + c;
  T* yp = y + b * p.yb + c;
  const int64_t keeps = (p.steps + kKeep - 1) / kKeep;
  float carry[V] = {};
  if (wave == 0 && live && y0)
#pragma unroll
    for (int e = 0; e < V; ++e) carry[e] = y0[at + e];
  for (int32_t k = place.order; k < (LINK ? place.order + 1 : p.nchunk); ++k) {
    const int64_t s0 = ((int64_t)k * waves + wave) * kKeep;
    float a[kKeep][V], u[kKeep][V];   // y -> a y + u
    const bool full = __all(s0 + kKeep <= len);
    if (full) {
      Words<T, V> xv[kKeep], xg[kKeep];
#pragma unroll
      for (int q = 0; q < kKeep; ++q) {
        xg[q] = take_once<T, V>(gp + (s0 + q) * p.gt);
        xv[q] = take_once<T, V>(vp + (s0 + q) * p.vt);
      }
#pragma unroll
      for (int q = 0; q < kKeep; ++q)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          float r;
          gate(as_f32(xg[q].v[e]), a[q][e], r);
          u[q][e] = r * as_f32(xv[q].v[e]);
        }
    } else {
#pragma unroll
      for (int q = 0; q < kKeep; ++q) {
#pragma unroll
        for (int e = 0; e < V; ++e) a[q][e] = 1.0f, u[q][e] = 0.0f;
        if (s0 + q < len) {
          const Words<T, V> xg = take_once<T, V>(gp + (s0 + q) * p.gt), xv = take_once<T, V>(vp + (s0 + q) * p.vt);
#pragma unroll
          for (int e = 0; e < V; ++e) {
            float r;
            gate(as_f32(xg.v[e]), a[q][e], r);
            u[q][e] = r * as_f32(xv.v[e]);
          }
        }
      }
    }
    float A[V], Y[V], h[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
      A[e] = a[0][e], Y[e] = u[0][e];
#pragma unroll
      for (int q = 1; q < kKeep; ++q) A[e] *= a[q][e], Y[e] = fmaf(a[q][e], Y[e], u[q][e]);
    }
    gated_enter<LINK, V>(p, runs[k & 1], enter, wave, waves, k, at, live, A, Y, carry, h);
    if (live && s0 < p.steps) {
      if (kept) {
        Words<float, V> x;
#pragma unroll
        for (int e = 0; e < V; ++e) x.v[e] = h[e];
        put_once(kept + (b * keeps + s0 / kKeep) * p.dim + c, x);
      }
#pragma unroll
      for (int q = 0; q < kKeep; ++q) {
        Words<T, V> o;
#pragma unroll
        for (int e = 0; e < V; ++e) {
          h[e] = fmaf(a[q][e], h[e], u[q][e]);
          o.v[e] = full || s0 + q < len ? (T)h[e] : (T)0.0f;
        }
        if (full || s0 + q < p.steps) put_once(yp + (s0 + q) * p.yt, o);
      }
    }
    // steps past a row's length keep its state, so the last run ends with it
    if (last && live && k == p.nchunk - 1 && wave == waves - 1)
#pragma unroll
      for (int e = 0; e < V; ++e) last[at + e] = h[e];
  }
}

// The gradient.  A wavefront's states come from the one that the forward pass
// left at its first step.
template <class T, int V, bool LINK>
__global__ void __launch_bounds__(512) k_gated_grad(GatedArgs p, const T* v, const T* g, const float* kept, const T* dy,
                                                    const float* dlast, T* dv, T* dg, float* dy0) {
  __shared__ GatedRuns<V> runs[2];
  __shared__ float enter[V][64];
  __shared__ uint32_t box;
  const int lane = threadIdx.x % 64, waves = blockDim.x / 64;
  const int run = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), wave = waves - 1 - run;
  const GatedPlace place = gated_place<LINK>(p, &box);
  const int64_t i = place.group * 64 + lane;
  const bool live = i < p.batch * p.nv;
  const int64_t b = live ? i / p.nv : 0, c = live ? (i - b * p.nv) * V : 0, at = b * p.dim + c;
  const int32_t len = live ? row_length(p, b) : 0;
  const T *vp = v + b * p.vb + c, *gp = g + b * p.gb + c, *dp = dy + b * p.yb + c;
  T *dvp = dv + b * p.steps * p.dim + c, *dgp = dg + b * p.steps * p.dim + c;
  const int64_t keeps = (p.steps + kKeep - 1) / kKeep;
  float carry[V] = {};
  if (run == 0 && live && dlast)
#pragma unroll
    for (int e = 0; e < V; ++e) carry[e] = dlast[at + e];
  for (int32_t k = place.order; k < (LINK ? place.order + 1 : p.nchunk); ++k) {
    const int64_t s0 = ((int64_t)(p.nchunk - 1 - k) * waves + wave) * kKeep;
    const bool some = live && s0 < len, full = __all(s0 + kKeep <= len);
    float a[kKeep][V], r[kKeep][V], x[kKeep][V], z[kKeep][V];   // z: dy
    float h[V];
#pragma unroll
    for (int e = 0; e < V; ++e) h[e] = some ? kept[(b * keeps + s0 / kKeep) * p.dim + c + e] : 0.0f;
    if (full) {
      Words<T, V> xv[kKeep], xg[kKeep], xd[kKeep];
#pragma unroll
      for (int q = 0; q < kKeep; ++q) {
        xg[q] = take_once<T, V>(gp + (s0 + q) * p.gt);
        xv[q] = take_once<T, V>(vp + (s0 + q) * p.vt);
        xd[q] = take_once<T, V>(dp + (s0 + q) * p.yt);
      }
#pragma unroll
      for (int q = 0; q < kKeep; ++q)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          gate(as_f32(xg[q].v[e]), a[q][e], r[q][e]);
          x[q][e] = as_f32(xv[q].v[e]);
          z[q][e] = as_f32(xd[q].v[e]);
        }
    } else {
#pragma unroll
      for (int q = 0; q < kKeep; ++q) {
#pragma unroll
        for (int e = 0; e < V; ++e) a[q][e] = 1.0f, r[q][e] = x[q][e] = z[q][e] = 0.0f;
        if (s0 + q < len) {
          const Words<T, V> xg = take_once<T, V>(gp + (s0 + q) * p.gt), xv = take_once<T, V>(vp + (s0 + q) * p.vt),
                            xd = take_once<T, V>(dp + (s0 + q) * p.yt);
#pragma unroll
          for (int e = 0; e < V; ++e) {
            gate(as_f32(xg.v[e]), a[q][e], r[q][e]);
            x[q][e] = as_f32(xv.v[e]);
            z[q][e] = as_f32(xd.v[e]);
          }
        }
      }
    }
    // x <- a (1 - a) (y[t-1] - v)
#pragma unroll
    for (int q = 0; q < kKeep; ++q)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float before = h[e];
        h[e] = fmaf(a[q][e], h[e], r[q][e] * x[q][e]);
        x[q][e] = a[q][e] * r[q][e] * (before - x[q][e]);
      }
    float A[V], M[V], m[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
      A[e] = a[kKeep - 1][e], M[e] = a[kKeep - 1][e] * z[kKeep - 1][e];
#pragma unroll
      for (int q = kKeep - 2; q >= 0; --q) A[e] *= a[q][e], M[e] = a[q][e] * (z[q][e] + M[e]);
    }
    gated_enter<LINK, V>(p, runs[k & 1], enter, run, waves, k, at, live, A, M, carry, m);
    if (live && s0 < p.steps) {
#pragma unroll
      for (int q = kKeep - 1; q >= 0; --q) {
        Words<T, V> ov, og;
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float d = z[q][e] + m[e];
          ov.v[e] = (T)(r[q][e] * d);
          og.v[e] = (T)(x[q][e] * d);
          if (full || s0 + q < len) m[e] = a[q][e] * d;
          else ov.v[e] = og.v[e] = (T)0.0f;
        }
        if (full || s0 + q < p.steps) {
          put_once(dvp + (s0 + q) * p.dim, ov);
          put_once(dgp + (s0 + q) * p.dim, og);
        }
      }
    }
    if (dy0 && live && k == p.nchunk - 1 && run == waves - 1)
#pragma unroll
      for (int e = 0; e < V; ++e) dy0[at + e] = m[e];
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
