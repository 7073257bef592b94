// The gated lowpass y[t] = a[t] y[t-1] + (1 - a[t]) v[t], a = 1 / (1 + exp(-g)),
// over whole sequences, its gradient, and its single step.
//
// A run of steps maps the state that enters it to the one that leaves it by
// y -> A y + Y, A the product of its a[t] and Y what it leaves from zero.  The
// gradient runs the same way from the end: m = a d goes from a step to the one
// before it, with d[t] = dy[t] + m[t+1], so a run maps m -> A m + M.
//
// Infinities and NaN: where a is 0 nothing of the state is taken, and where 1 - a
// is 0 nothing of the input, whatever they are (the products are not made), so a
// sequence that went wrong ends where the next one of its row begins.  A
// product of gates above 0 is held above 0: an infinite state stays infinite in
// a joined run as it does step by step.  The looks at every gate take 4 x 16384 x
// 2048 bf16 from 164 to 176 us and the gradient of 8 x 4096 x 2048 from 143 to
// 146; looking only where a wavefront has such a gate or value costs as much.
//
// Memory bounds it: each array has to be read or written once, a step costs
// two transcendental instructions and about fifteen others for its 3 (gradient:
// 5) values.  So every value is read once and stays in registers until its
// result is known.  A wavefront takes kKeep = 16 steps of 64 V channels,
// fetched together; its lanes find their runs' maps, and the wavefronts of a
// workgroup, which hold consecutive runs, join them in LDS.  Sequences longer
// than a workgroup's 128 steps are cut into such chunks.  A few chunks are gone
// through by one workgroup, one after the other (LINK = false).  Otherwise the
// chunks run side by side (LINK): each publishes its map for the later ones,
// and every kSpan-th the state that it ends with; a chunk waits for the state at
// its span's beginning and the maps in between, a wavefront for each.  The order
// of the operations is fixed, so the result does not depend on timing.
//
// Measured at 4 x 16384 x 2048 bf16 (0.81 GB): 165 to 180 us, 4.9 TB/s at best.
// Step by step, before the looks at gates: 445 us in two passes (maps, then
// steps: v and g are read twice), 190 us in one with the first wavefront waiting
// for all maps, 152 to 163 us with a wavefront for each, 149 us without any
// waiting (a copy that is not correct, to know the cost), 146 us without the
// exponentials too.  Chunks of 64 steps took 235 us, of 256 steps 193; one channel
// per lane 229.  A third workgroup on each CU (gates kept as one number) did not
// help: 171.  The gradient of 8 x 4096 x 2048 bf16 (0.71 GB with the kept
// states): 145 to 150 us, 4.9 TB/s.
#pragma once

#include "kernels_embed.hpp"
#include "operators_rules.hpp"

using ms::kGatedWaves;
using ms::kKeep;   // steps of a wavefront

constexpr int kSpan = 8;         // chunks from one published state to the next

// A lane takes V neighbouring channels of one batch row, a word of at most 4
// bytes.
struct GatedArgs {
  int64_t batch, steps, dim, nv;    // nv = dim / V
  int64_t vb, vt, gb, gt, yb, yt;   // strides of v, g and y (dy in the gradient)
  const int32_t* lengths;
  int32_t nchunk, groups;           // chunks of blockDim / 64 * kKeep steps; workgroups per chunk
  int32_t per_row;                  // workgroups per batch row (SPAN = false)
  int64_t first;                    // the launch's first group (LINK = false)
  // LINK: what chunks leave for each other, all ones before the launch
  uint64_t* maps;                   // [nchunk][batch * dim]: (A, Y)
  uint32_t* states;                 // [nchunk / kSpan][batch * dim]
  uint32_t* ticket;
};

__device__ __forceinline__ int32_t row_length(const GatedArgs& p, int64_t b) {
  if (!p.lengths) return (int32_t)p.steps;
  return min(max(p.lengths[b], 0), (int32_t)p.steps);
}

// a and 1 - a from the logit, each to a few units of its last bit and |g| / ln 2
// half units of the exponential's argument, also where one is small (down to
// about 1e-38; what is smaller may be 0).
__device__ __forceinline__ void gate(float g, float& a, float& rest) {
  const float e = __expf(-fabsf(g));
  const float big = __builtin_amdgcn_rcpf(1.0f + e), small = e * big;
  a = g >= 0.0f ? big : small;
  rest = g >= 0.0f ? small : big;
}

// Both gates in one number: the smaller, negative where it is a.
__device__ __forceinline__ float gate_packed(float g) {
  const float e = __expf(-fabsf(g));
  const float small = e * __builtin_amdgcn_rcpf(1.0f + e);
  return g >= 0.0f ? small : -small;   // -0 at g = -inf
}

__device__ __forceinline__ void gate_of(float s, float& a, float& rest) {
  const float small = fabsf(s), big = 1.0f - small;
  const bool rest_small = !__builtin_signbit(s);
  a = rest_small ? big : small;
  rest = rest_small ? small : big;
}

// a x, and nothing of x where a is 0.
__device__ __forceinline__ float part_of(float a, float x) { return a == 0.0f ? 0.0f : a * x; }

// a y + u, and nothing of y where a is 0.
__device__ __forceinline__ float onto(float a, float y, float u) { return a == 0.0f ? u : fmaf(a, y, u); }

// A product of gates, from the rounded one and their smallest: 0 only if one of
// them is.  What it keeps of a state when it would round to 0 is 2^-149.
__device__ __forceinline__ float gates_product(float rounded, float smallest) {
  return fmaxf(rounded, fminf(smallest, __builtin_bit_cast(float, 1u)));
}

// Keeps the instructions of every fourth step apart, so that values of all
// steps are not wanted at once.
__device__ __forceinline__ void step_apart(int q) {
  if (q % 4 == 0) __builtin_amdgcn_sched_barrier(0);
}

// What follows from x is computed anew after this, not kept in registers.
template <class X>
__device__ __forceinline__ void again(X& x) {
  asm volatile("" : "+v"(x));
}

// A lane's V values of one step, as they come from memory, in one register.
template <class T, int V>
__device__ __forceinline__ uint32_t take_raw(const T* p) {
  static_assert(sizeof(T) * V <= 4, "one register");
  if constexpr (sizeof(T) * V == 4) return __builtin_nontemporal_load((const uint32_t*)p);
  else return __builtin_bit_cast(uint16_t, *p);
}

template <class T>
__device__ __forceinline__ float raw_value(uint32_t w, int e) {
  if constexpr (sizeof(T) == 4) return __builtin_bit_cast(float, w);
  else return __builtin_bit_cast(float, e ? w & 0xffff0000u : w << 16);
}

// One step of the filter.
__device__ __forceinline__ float gated_step(float y, float g, float v) {
  float a, r;
  gate(g, a, r);
  return onto(a, y, part_of(r, v));
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
  if (!LINK) return {0, p.first + (int64_t)blockIdx.x};
  if (threadIdx.x == 0) *box = __hip_atomic_fetch_add(p.ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  const uint32_t t = __builtin_amdgcn_readfirstlane(*box);
  return {(int32_t)(t / (uint32_t)p.groups), (int64_t)(t % (uint32_t)p.groups)};
}

// The channels of a lane.  SPAN: lanes are dealt to all rows' channels in
// order, for rows that would leave many of a wavefront's idle.  Otherwise a
// wavefront stays in one row: its addresses are a uniform part and one offset
// per lane.
struct GatedLane {
  bool live;
  int64_t b;
  uint32_t c;
  int32_t len;
};

template <bool SPAN, int V>
__device__ __forceinline__ GatedLane gated_lane(const GatedArgs& p, int64_t group) {
  const int lane = threadIdx.x % 64;
  GatedLane l;
  if constexpr (SPAN) {
    const int64_t i = group * 64 + lane;
    l.live = i < p.batch * p.nv;
    l.b = l.live ? i / p.nv : 0;
    l.c = l.live ? (uint32_t)(i - l.b * p.nv) * V : 0;
    l.len = l.live ? row_length(p, l.b) : 0;
  } else {
    const uint32_t row = __builtin_amdgcn_readfirstlane((uint32_t)group / (uint32_t)p.per_row);
    const int32_t i = (int32_t)((uint32_t)group - row * (uint32_t)p.per_row) * 64 + lane;
    l.b = row;
    l.live = i < p.nv;
    l.c = l.live ? (uint32_t)i * V : 0;
    l.len = __builtin_amdgcn_readfirstlane(row_length(p, l.b));
  }
  return l;
}

// What a workgroup's wavefronts tell each other: the maps of their runs, the
// value that enters the chunk or its span, and the maps of the span's earlier
// chunks.
template <int V>
struct GatedRuns {
  float A[kGatedWaves][V][64], Y[kGatedWaves][V][64];
};

template <bool LINK, int V>
struct GatedShared {
  GatedRuns<V> runs[2];   // LINK: this chunk's, and the span's earlier ones; else one for every other chunk
  float enter[V][64];
};

__device__ __forceinline__ uint32_t link_load(const uint32_t* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ uint64_t link_load(const uint64_t* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Waits for V published words.
template <int V, class W>
__device__ __forceinline__ void link_wait(const W* p, W* w) {
  bool wait;
  do {
    wait = false;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      w[e] = link_load(p + e);
      wait |= w[e] == (W)~(W)0;
    }
  } while (wait);
}

// The value that enters this wavefront's run.  `run` counts wavefronts, and
// `order` chunks, along the direction of the recurrence; `carry` holds, in
// wavefront 0, what enters the first chunk, and with LINK = false then the next
// one.  Called by all wavefronts.  Published words are atomic accesses of their
// own, so a word that is there is whole; they need no order among themselves.
template <bool LINK, int V>
__device__ __forceinline__ void gated_enter(const GatedArgs& p, GatedShared<LINK, V>& sh, int run, int nrun, int32_t order,
                                            int64_t at, bool live, const float* A, const float* Y, float* carry, float* h) {
  const int lane = threadIdx.x % 64;
  GatedRuns<V>& runs = sh.runs[LINK ? 0 : order & 1];
#pragma unroll
  for (int e = 0; e < V; ++e) runs.A[run][e][lane] = A[e], runs.Y[run][e][lane] = Y[e];
  __syncthreads();
  const int64_t channels = p.batch * p.dim;
  const int32_t span = order / kSpan, from = span * kSpan;
  float cA[V], cY[V];   // the chunk's map, in wavefront 0
  if (run == 0) {
#pragma unroll
    for (int e = 0; e < V; ++e) cA[e] = A[e], cY[e] = Y[e];
    for (int w = 1; w < nrun; ++w)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float a = runs.A[w][e][lane];
        cA[e] = gates_product(cA[e] * a, fminf(cA[e], a));
        cY[e] = onto(a, cY[e], runs.Y[w][e][lane]);
      }
    if (LINK && live && order + 1 < p.nchunk)
#pragma unroll
      for (int e = 0; e < V; ++e)
        __hip_atomic_store(p.maps + order * channels + at + e, (uint64_t)published(cY[e]) << 32 | published(cA[e]),
                           __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (!LINK || span == 0)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        sh.enter[e][lane] = carry[e];
        if (!LINK) carry[e] = onto(cA[e], carry[e], cY[e]);
      }
  }
  if constexpr (LINK) {   // eight wavefronts: one for each earlier map of the span, the last one for its state
    static_assert(kSpan == kGatedWaves, "a wavefront each");
    if (run < kSpan - 1 && from + run < order) {
      uint64_t w[V] = {};
      if (live) link_wait<V>(p.maps + (from + run) * channels + at, w);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        sh.runs[1].A[run][e][lane] = __builtin_bit_cast(float, (uint32_t)w[e]);
        sh.runs[1].Y[run][e][lane] = __builtin_bit_cast(float, (uint32_t)(w[e] >> 32));
      }
    }
    if (run == kSpan - 1 && span > 0) {
      uint32_t w[V] = {};
      if (live) link_wait<V>(p.states + (span - 1) * channels + at, w);
#pragma unroll
      for (int e = 0; e < V; ++e) sh.enter[e][lane] = __builtin_bit_cast(float, w[e]);
    }
  }
  __syncthreads();
#pragma unroll
  for (int e = 0; e < V; ++e) h[e] = sh.enter[e][lane];
  if constexpr (LINK) {
    for (int k = 0; from + k < order; ++k)
#pragma unroll
      for (int e = 0; e < V; ++e) h[e] = onto(sh.runs[1].A[k][e][lane], h[e], sh.runs[1].Y[k][e][lane]);
    if (run == 0 && live && order % kSpan == kSpan - 1 && order + 1 < p.nchunk)
#pragma unroll
      for (int e = 0; e < V; ++e)
        __hip_atomic_store(p.states + span * channels + at + e, published(onto(cA[e], h[e], cY[e])), __ATOMIC_RELAXED,
                           __HIP_MEMORY_SCOPE_AGENT);
  }
  for (int w = 0; w < run; ++w)
#pragma unroll
    for (int e = 0; e < V; ++e) h[e] = onto(runs.A[w][e][lane], h[e], runs.Y[w][e][lane]);
}

template <class T, int V, bool LINK, bool SPAN>
__global__ void __launch_bounds__(64 * kGatedWaves) k_gated(GatedArgs p, const T* v, const T* g, const float* y0, T* y, float* last,
                                               float* kept) {
  __shared__ GatedShared<LINK, V> shared;
  __shared__ uint32_t box;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), waves = blockDim.x / 64;
  const GatedPlace place = gated_place<LINK>(p, &box);
  const auto [live, b, c, len] = gated_lane<SPAN, V>(p, place.group);
  const int64_t at = b * p.dim + c, end = max(len, 1) - 1;   // steps past `end` are read there, and not used
  const T *vp = v + b * p.vb, *gp = g + b * p.gb;
  T* yp = y + b * p.yb;
  const int64_t keeps = (p.steps + kKeep - 1) / kKeep;
  float carry[V] = {};
  if (wave == 0 && live && y0)
#pragma unroll
    for (int e = 0; e < V; ++e) carry[e] = y0[at + e];
  for (int32_t k = place.order; k < (LINK ? place.order + 1 : p.nchunk); ++k) {
    const int64_t s0 = ((int64_t)k * waves + wave) * kKeep;
    float a[kKeep][V], u[kKeep][V];   // y -> a y + u
    const bool full = SPAN ? __all(s0 + kKeep <= len) : s0 + kKeep <= len;
    {
      uint32_t xv[kKeep], xg[kKeep];
#pragma unroll
      for (int q = 0; q < kKeep; ++q) {
        const int64_t s = full ? s0 + q : min(s0 + q, end);
        xg[q] = take_raw<T, V>(gp + s * p.gt + c);
        xv[q] = take_raw<T, V>(vp + s * p.vt + c);
      }
#pragma unroll
      for (int q = 0; q < kKeep; ++q)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          float r;
          gate(raw_value<T>(xg[q], e), a[q][e], r);
          u[q][e] = part_of(r, raw_value<T>(xv[q], e));
        }
    }
    if (!full) {
#pragma unroll
      for (int q = 0; q < kKeep; ++q)
        if (s0 + q >= len)
#pragma unroll
          for (int e = 0; e < V; ++e) a[q][e] = 1.0f, u[q][e] = 0.0f;
    }
    float A[V], Y[V], h[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
      float least = a[0][e];
      A[e] = a[0][e], Y[e] = u[0][e];
#pragma unroll
      for (int q = 1; q < kKeep; ++q) {
        A[e] *= a[q][e], least = fminf(least, a[q][e]);
        Y[e] = onto(a[q][e], Y[e], u[q][e]);
      }
      A[e] = gates_product(A[e], least);
    }
    gated_enter<LINK, V>(p, shared, wave, waves, k, at, live, A, Y, carry, h);
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
          h[e] = onto(a[q][e], h[e], u[q][e]);
          o.v[e] = full || s0 + q < len ? (T)h[e] : (T)0.0f;
        }
        if (full || s0 + q < p.steps) put_once(yp + (s0 + q) * p.yt + c, o);
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
template <class T, int V, bool LINK, bool SPAN>
__global__ void __launch_bounds__(64 * kGatedWaves) k_gated_grad(GatedArgs p, const T* v, const T* g, const float* kept, const T* dy,
                                                    const float* dlast, T* dv, T* dg, float* dy0) {
  __shared__ GatedShared<LINK, V> shared;
  __shared__ uint32_t box;
  const int waves = blockDim.x / 64;
  const int run = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), wave = waves - 1 - run;
  const GatedPlace place = gated_place<LINK>(p, &box);
  const auto [live, b, c, len] = gated_lane<SPAN, V>(p, place.group);
  const int64_t at = b * p.dim + c, end = max(len, 1) - 1;   // steps past `end` are read there, and not used
  const T *vp = v + b * p.vb, *gp = g + b * p.gb, *dp = dy + b * p.yb;
  T *dvp = dv + b * p.steps * p.dim, *dgp = dg + b * p.steps * p.dim;
  const int64_t keeps = (p.steps + kKeep - 1) / kKeep;
  float carry[V] = {};
  if (run == 0 && live && dlast)
#pragma unroll
    for (int e = 0; e < V; ++e) carry[e] = dlast[at + e];
  for (int32_t k = place.order; k < (LINK ? place.order + 1 : p.nchunk); ++k) {
    const int64_t s0 = ((int64_t)(p.nchunk - 1 - k) * waves + wave) * kKeep;
    const bool some = live && s0 < len, full = SPAN ? __all(s0 + kKeep <= len) : s0 + kKeep <= len;
    float s[kKeep][V], x[kKeep][V];   // the gates in one; a (1 - a) (y[t-1] - v)
    uint32_t z[kKeep];                // dy
    float h[V];
#pragma unroll
    for (int e = 0; e < V; ++e) h[e] = some ? kept[(b * keeps + s0 / kKeep) * p.dim + c + e] : 0.0f;
    {
      uint32_t xv[kKeep], xg[kKeep];
#pragma unroll
      for (int q = 0; q < kKeep; ++q) {
        const int64_t st = full ? s0 + q : min(s0 + q, end);
        xg[q] = take_raw<T, V>(gp + st * p.gt + c);
        xv[q] = take_raw<T, V>(vp + st * p.vt + c);
        z[q] = take_raw<T, V>(dp + st * p.yt + c);
      }
      __builtin_amdgcn_sched_barrier(0);   // all on their way before the first is used
#pragma unroll
      for (int q = 0; q < kKeep; ++q)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          s[q][e] = gate_packed(raw_value<T>(xg[q], e));
          x[q][e] = raw_value<T>(xv[q], e);
          if (e == V - 1) step_apart(q);
        }
    }
    if (!full) {   // a = 1 and nothing else
#pragma unroll
      for (int q = 0; q < kKeep; ++q)
        if (s0 + q >= len)
#pragma unroll
          for (int e = 0; e < V; ++e) s[q][e] = x[q][e] = 0.0f, z[q] = 0;
    }
#pragma unroll
    for (int q = 0; q < kKeep; ++q)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        float a, r;
        gate_of(s[q][e], a, r);
        const float before = h[e];
        h[e] = onto(a, h[e], part_of(r, x[q][e]));
        x[q][e] = part_of(a * r, before - x[q][e]);
        again(x[q][e]);   // and is computed here, not where it is used
        if (e == V - 1) step_apart(q);
      }
    float A[V], M[V], m[V], least[V];
#pragma unroll
    for (int e = 0; e < V; ++e) A[e] = least[e] = 1.0f, M[e] = 0.0f;
#pragma unroll
    for (int q = kKeep - 1; q >= 0; --q) {
#pragma unroll
      for (int e = 0; e < V; ++e) {
        float a, r;
        again(s[q][e]);
        gate_of(s[q][e], a, r);
        A[e] *= a, least[e] = fminf(least[e], a);
        M[e] = part_of(a, raw_value<T>(z[q], e) + M[e]);
      }
      step_apart(q);
    }
#pragma unroll
    for (int e = 0; e < V; ++e) A[e] = gates_product(A[e], least[e]);
    gated_enter<LINK, V>(p, shared, run, waves, k, at, live, A, M, carry, m);
#pragma unroll
    for (int q = 0; q < kKeep; ++q) again(z[q]);
    if (live && s0 < p.steps) {
#pragma unroll
      for (int q = kKeep - 1; q >= 0; --q) {
        Words<T, V> ov, og;
#pragma unroll
        for (int e = 0; e < V; ++e) {
          float a, r;
          again(s[q][e]);
          gate_of(s[q][e], a, r);
          const float d = raw_value<T>(z[q], e) + m[e];
          ov.v[e] = (T)part_of(r, d);
          og.v[e] = (T)(s[q][e] == 0.0f ? 0.0f : x[q][e] * d);   // one of the gates is 0
          if (full || s0 + q < len) m[e] = part_of(a, d);
          else ov.v[e] = og.v[e] = (T)0.0f;
        }
        if (full || s0 + q < p.steps) {
          put_once(dvp + (s0 + q) * p.dim + c, ov);
          put_once(dgp + (s0 + q) * p.dim + c, og);
        }
        step_apart(q);
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
