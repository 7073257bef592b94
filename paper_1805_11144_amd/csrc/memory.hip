// The operators of keyed memories in the C ABI: argument checks, workspace layouts
// and launches.  The kernels are in kernels_delta.hpp, kernels_delta_grad.hpp and
// kernels_norm.hpp.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <string>

#include "host.hpp"
#include "kernels_delta.hpp"
#include "kernels_delta_grad.hpp"
#include "kernels_norm.hpp"
#include "operators_host.hpp"
#include "operators_rules.hpp"

using namespace ms;

namespace {

// Calls f with a key head's padded width.
template <class F>
void with_keys(int64_t dk, F&& f) {
  if (dk <= 32) f(std::integral_constant<int, 32>{});
  else if (dk <= 64) f(std::integral_constant<int, 64>{});
  else f(std::integral_constant<int, 128>{});
}

template <class F>
void with_flag(bool b, F&& f) {
  if (b) f(std::true_type{});
  else f(std::false_type{});
}

template <class F>
void with_value(int32_t dtype, F&& f) {
  if (dtype == MS_DTYPE_BF16) f((__bf16)0.0f);
  else f(0.0f);
}

template <class K>
void allow_lds(K k, size_t lds) {
  if (lds > 65536) HIPCHECK(hipFuncSetAttribute((const void*)k, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
}

// ------------------------------------------------------------------- delta
Walk walk_of(const int64_t* s, int64_t steps, int64_t heads, int64_t dim) {
  Walk w{s[0], s[1], s[2]};
  if (s[0] == 0 && s[1] == 0 && s[2] == 0) w = {steps * heads * dim, heads * dim, dim};
  need(w.b >= 0 && w.t >= 0 && w.h >= 0 && w.b < kMaxStride && w.t < kMaxStride && w.h < kMaxStride,
       "strides must be in [0, 2^40)");
  return w;
}

// Whether runs of `dim` values at these strides are apart: ordered by stride, each
// steps over all that the ones before it reach.
bool walk_apart(Walk w, int64_t batch, int64_t steps, int64_t heads, int64_t dim) {
  if (batch == 0 || steps == 0 || heads == 0) return true;
  std::pair<int64_t, int64_t> d[3] = {{w.b, batch}, {w.t, steps}, {w.h, heads}};
  std::sort(d, d + 3);
  __int128 reach = dim;
  for (const auto& [stride, n] : d) {
    if (n == 1) continue;
    if (stride < reach) return false;
    reach += (__int128)stride * (n - 1);
  }
  return true;
}

// Runs of `run` bytes, n of them `stride` bytes apart, and so on outwards.
struct Runs {
  const void* at;
  int64_t run;
  std::pair<int64_t, int64_t> level[2];   // stride, n: outer, inner
};

// Whether two arrays may share a byte, the second one's begin `apart` bytes behind the
// first one's.  Exact where their levels have equal strides, and inner ones lie within
// a step of the outer (columns of one buffer); else as their whole ranges do.
bool may_share(const Runs& x, const Runs& y, int level, __int128 apart) {
  while (level < 2 && x.level[level].second == 1 && y.level[level].second == 1) ++level;
  const auto reach = [](const Runs& r, int from) {
    __int128 n = r.run;
    for (int i = from; i < 2; ++i) n += (__int128)r.level[i].first * (r.level[i].second - 1);
    return n;
  };
  if (apart >= reach(x, level) || -apart >= reach(y, level)) return false;
  if (level == 2) return true;
  const auto [sx, nx] = x.level[level];
  const auto [sy, ny] = y.level[level];
  const int64_t step = nx == 1 ? sy : sx;
  if ((ny > 1 && sy != step) || step <= 0 || reach(x, level + 1) > step || reach(y, level + 1) > step) return true;
  // y's run of the level j lies apart + (j - i) step behind x's i: only two differences can bring them together
  for (__int128 m = apart / step - 1; m <= apart / step + 1; ++m)
    if (-m < ny && m < nx && may_share(x, y, level + 1, apart - m * step)) return true;
  return false;
}

bool may_share(const Runs& x, const Runs& y) {
  return may_share(x, y, 0, (__int128)(uintptr_t)y.at - (__int128)(uintptr_t)x.at);
}

struct Delta {
  DeltaArgs a;
  int64_t chunks;            // of all heads and rows
  int64_t chunk_steps, work;   // bytes a chunk
  int blocks;   // of four tiles of 16 columns
};

Delta check_delta(const ms_gated_delta_desc* d) {
  need(d != nullptr, "NULL descriptor");
  need(d->steps >= 0 && d->steps < ((int64_t)1 << 31), "steps must be in [0, 2^31)");
  need(d->batch >= 0 && d->batch < ((int64_t)1 << 31), "batch must be in [0, 2^31)");
  need(d->key_heads >= 1 && d->heads >= 1 && d->heads <= 65536 && d->heads % d->key_heads == 0,
       "heads must be in [1, 65536], a multiple of key_heads");
  need(d->keys >= 1 && d->keys <= 128, "keys must be in [1, 128]");
  need(d->values >= 1 && d->values <= 65536, "values must be in [1, 65536]");
  need_dtype(d->dtype);
  need(std::isfinite((float)d->scale), "scale must be finite in 32 bits");
  Delta p{};
  DeltaArgs& a = p.a;
  a.batch = d->batch, a.steps = (int32_t)d->steps, a.heads = (int32_t)d->heads;
  a.group = (int32_t)(d->heads / d->key_heads), a.dk = (int32_t)d->keys, a.dv = (int32_t)d->values;
  a.scale = (float)d->scale;
  a.q = walk_of(d->q_stride, d->steps, d->key_heads, d->keys);
  a.k = walk_of(d->k_stride, d->steps, d->key_heads, d->keys);
  a.v = walk_of(d->v_stride, d->steps, d->heads, d->values);
  a.y = walk_of(d->y_stride, d->steps, d->heads, d->values);
  a.decay = walk_of(d->decay_stride, d->steps, d->heads, 1);
  a.rate = walk_of(d->rate_stride, d->steps, d->heads, 1);
  // a chunk's offsets from its first step are 32 bits
  need(std::max(a.v.t, a.y.t) < (1 << 24) && d->heads * d->values < (1 << 24),
       "heads * values and the strides between steps of v, y and dy must be below 2^24");
  const bool half = d->dtype == MS_DTYPE_BF16;
  p.chunk_steps = half ? kChunk<__bf16> : kChunk<float>;
  a.nchunk = (d->steps + p.chunk_steps - 1) / p.chunk_steps;
  const int tiles = (int)((d->values + 15) / 16);
  p.blocks = (tiles + 3) / 4;
  need(d->batch * d->heads <= kMaxBlocks / 2 / p.blocks - 8, "batch * heads * values is too large");
  p.chunks = d->batch * d->heads * a.nchunk;
  need(p.chunks < ((int64_t)1 << 31), "batch * heads * steps is too large");
  p.work = half ? ChunkWork<kChunk<__bf16>>::bytes : ChunkWork<kChunk<float>>::bytes;
  return p;
}

// What the gradient starts from: each chunk's state, then the errors.
int64_t kept_states(const Delta& p) { return p.chunks * pad_keys(p.a.dk) * pad_columns(p.a.dv); }
int64_t kept_rows(const Delta& p) { return p.chunks * p.chunk_steps * pad_columns(p.a.dv); }

struct DeltaWork {
  char* chunk;
  float *dstates, *xs;
  int64_t bytes;
};

DeltaWork delta_work(const Delta& p, bool grad, void* ws) {
  Carve c{(char*)ws};
  DeltaWork w{};
  if (p.chunks > 0) {
    w.chunk = c.take<char>(p.chunks * p.work);
    if (grad) {
      w.dstates = c.take<float>(kept_states(p));
      w.xs = c.take<float>(kept_rows(p));
    }
  }
  w.bytes = c.used;
  return w;
}

bool words(const Walk& w, const void* p) { return w.b % 8 == 0 && w.t % 8 == 0 && w.h % 8 == 0 && (uintptr_t)p % 16 == 0; }

dim3 scan_grid(const Delta& p) { return dim3((unsigned)(up(p.a.batch * p.a.heads, 8) * p.blocks)); }

// -------------------------------------------------------------------- norm
struct Norm {
  NormArgs a;
  NormShape shape;
  int64_t channels, v;
};

static_assert(kNormRows % 4 == 0, "k_norm_team_grad has up to 4 rows on their way");
static_assert(MS_ACT_NONE == kActNone && MS_ACT_RELU == kActRelu && MS_ACT_SILU == kActSilu, "activations");

// v: values of a word, as sizes, strides and pointers allow (1 for workspaces, which hold for any).
Norm check_norm(const ms_group_norm_desc* d) {
  need(d != nullptr, "NULL descriptor");
  need(d->batch >= 0 && d->batch < ((int64_t)1 << 31), "batch must be in [0, 2^31)");
  need(d->positions >= 0 && d->positions < ((int64_t)1 << 31), "positions must be in [0, 2^31)");
  need(d->groups >= 1 && d->channels >= 1 && d->channels < (1 << 24) && d->channels % d->groups == 0,
       "channels must be in [1, 2^24), a multiple of groups");
  need_dtype(d->dtype);
  need(d->activation == MS_ACT_NONE || d->activation == MS_ACT_RELU || d->activation == MS_ACT_SILU, "unknown activation");
  need(d->eps >= 0 && std::isfinite((float)d->eps), "eps must be finite in 32 bits and not negative");
  need(d->batch * d->groups < ((int64_t)1 << 40) && d->batch * d->channels < ((int64_t)1 << 44), "batch * channels is too large");
  Norm p{};
  NormArgs& a = p.a;
  p.channels = d->channels;
  a.batch = d->batch, a.positions = d->positions;
  a.groups = (int32_t)d->groups, a.width = (int32_t)(d->channels / d->groups);
  const auto pair = [&](const int64_t* s, int64_t& b, int64_t& t) {
    const bool packed = s[0] == 0 && s[1] == 0;
    b = packed ? d->positions * d->channels : s[0], t = packed ? d->channels : s[1];
    need(b >= 0 && t >= 0 && b < kMaxStride && t < kMaxStride, "strides must be in [0, 2^40)");
  };
  pair(d->x_stride, a.xb, a.xt);
  pair(d->y_stride, a.yb, a.yt);
  a.eps = (float)d->eps, a.act = d->activation;
  return p;
}

void norm_choose(Norm& p, int64_t v, bool grad) {
  NormArgs& a = p.a;
  p.v = v;
  a.nw = (int32_t)(a.width / v);
  p.shape = norm_shape(a.batch, a.positions, a.groups, a.nw, grad);
  a.team = p.shape.team, a.lanes = p.shape.lanes, a.pieces = p.shape.pieces;
  a.runs = p.shape.runs, a.run = p.shape.run, a.wide = p.shape.wide;
}

// Scratch memory: parts, then mean and rstd where the caller keeps none (or the
// groups' sums of the gradient).  Without pointers: the most that any word takes.
struct NormWork {
  float *parts, *sums, *next;
  int64_t bytes;
};

NormWork norm_work(const Norm& p, bool grad, void* ws) {
  Carve c{(char*)ws};
  NormWork w{};
  const NormArgs& a = p.a;
  if (!grad && !a.team) {
    w.parts = c.take<float>(a.batch * a.runs * a.groups * a.nw * 2);
    w.sums = c.take<float>(a.batch * a.groups * 2);
  } else if (grad) {
    const int64_t rows = a.team ? (int64_t)a.lanes * a.pieces : a.batch * a.runs;
    w.parts = c.take<float>(rows * 2 * p.channels);
    int64_t joined = 0;   // rows of all later levels
    for (int64_t r = rows; r > kColumnRows;) joined += r = (r + kColumnRows - 1) / kColumnRows;
    w.next = c.take<float>(joined * 2 * p.channels);
    if (!a.team) w.sums = c.take<float>(a.batch * a.groups * 2);
  }
  w.bytes = c.used;
  return w;
}

int64_t norm_most(Norm p, int32_t dtype, bool grad) {
  int64_t most = 0;
  for (int64_t v = 16 / (int64_t)size_of(dtype); v >= 1; v /= 2) {
    if (p.a.width % v != 0) continue;
    norm_choose(p, v, grad);
    most = std::max(most, norm_work(p, grad, nullptr).bytes);
  }
  return most;
}

// Calls f with a team's words to a thread.
template <class F>
void with_words(int32_t words, F&& f) {
  if (words == 1) f(std::integral_constant<int, 1>{});
  else if (words == 2) f(std::integral_constant<int, 2>{});
  else f(std::integral_constant<int, 4>{});
}

unsigned norm_grid(const Norm& p) {
  const int64_t blocks = (p.a.groups * (int64_t)p.a.nw + p.a.wide - 1) / p.a.wide;
  return (unsigned)std::min(p.a.batch * p.a.runs * blocks, kMaxBlocks);
}

}  // namespace

extern "C" {

ms_status ms_gated_delta_kept(const ms_gated_delta_desc* d, int64_t* elements_out) {
  return guarded([&] {
    const Delta p = check_delta(d);
    need(elements_out != nullptr, "NULL output");
    *elements_out = kept_states(p) + kept_rows(p);
  });
}

ms_status ms_gated_delta_workspace(const ms_gated_delta_desc* d, int32_t grad, int64_t* bytes_out) {
  return guarded([&] {
    const Delta p = check_delta(d);
    need(bytes_out != nullptr, "NULL output");
    *bytes_out = delta_work(p, grad != 0, nullptr).bytes;
  });
}

ms_status ms_gated_delta(const ms_gated_delta_desc* d, const void* q, const void* k, const void* v, const float* decay,
                         const float* rate, const float* s0, const int32_t* lengths, void* y, float* last, float* kept,
                         void* workspace, int64_t workspace_bytes) {
  return guarded([&] {
    Delta p = check_delta(d);
    DeltaArgs& a = p.a;
    if (a.batch == 0) return;
    const size_t es = size_of(d->dtype);
    need(walk_apart(a.y, a.batch, a.steps, a.heads, a.dv), "rows, steps or heads of y overlap");
    need(a.steps == 0 || (q && k && v && decay && rate && y), "NULL array");
    for (const void* x : {q, k, v, (const void*)y}) need_aligned(x, es, "q, k, v or y");
    for (const void* x : {(const void*)decay, (const void*)rate, (const void*)s0, (const void*)lengths, (const void*)last,
                          (const void*)kept})
      need_aligned(x, 4, "decay, rate, s0, lengths, last or kept");
    need((uintptr_t)kept % 16 == 0, "kept must be 16-byte aligned");
    const DeltaWork w = delta_work(p, false, workspace);
    need_workspace(workspace, workspace_bytes, w.bytes);
    DeviceGuard dg(d->device);
    const hipStream_t st = (hipStream_t)d->stream;
    a.lengths = lengths;
    float* errors = kept ? kept + kept_states(p) : nullptr;
    with_value(d->dtype, [&](auto zero) {
      using T = decltype(zero);
      const bool wide = a.dk % 8 == 0 && a.dv % 8 == 0 && words(a.q, q) && words(a.k, k) && words(a.v, v) && words(a.y, y);
      with_flag(wide, [&](auto vec) {
        with_keys(a.dk, [&](auto keys) {
          constexpr int DK = decltype(keys)::value;
          constexpr bool VEC = decltype(vec)::value;
          if (p.chunks)
            hipLaunchKernelGGL(HIP_KERNEL_NAME(k_delta_chunk<T, VEC, DK, false>),
                               dim3((unsigned)std::min(p.chunks, kMaxBlocks)), dim3(kChunk<T> * 4), 0, st, a, (const T*)q,
                               (const T*)k, decay, rate, w.chunk);
          with_flag(kept != nullptr, [&](auto keep) {
            constexpr auto scan = k_delta_scan<T, VEC, DK, decltype(keep)::value>;
            constexpr size_t lds = ScanLds<T, DK, false>::all;
            static_assert(lds <= 160 * 1024, "LDS");
            allow_lds(scan, lds);
            hipLaunchKernelGGL(scan, scan_grid(p), dim3(512), lds, st, a, p.blocks, (const T*)q, (const T*)k, (const T*)v,
                               decay, s0, (const char*)w.chunk, (T*)y, last, kept, errors);
          });
        });
      });
    });
    HIPCHECK(hipGetLastError());
  });
}

ms_status ms_gated_delta_grad(const ms_gated_delta_desc* d, const void* q, const void* k, const void* v, const float* decay,
                              const float* rate, const float* kept, const int32_t* lengths, const void* dy,
                              const float* dlast, void* dq, void* dk, void* dv, float* ddecay, float* drate, float* ds0,
                              void* workspace, int64_t workspace_bytes) {
  return guarded([&] {
    Delta p = check_delta(d);
    DeltaArgs& a = p.a;
    if (a.batch == 0) return;
    const size_t es = size_of(d->dtype);
    need(a.steps == 0 || (q && k && v && decay && rate && kept && dy && dq && dk && dv && ddecay && drate), "NULL array");
    for (const void* x : {q, k, v, dy, (const void*)dq, (const void*)dk, (const void*)dv})
      need_aligned(x, es, "q, k, v, dy, dq, dk or dv");
    for (const void* x : {(const void*)decay, (const void*)rate, (const void*)kept, (const void*)lengths, (const void*)dlast,
                          (const void*)ddecay, (const void*)drate, (const void*)ds0})
      need_aligned(x, 4, "decay, rate, kept, lengths, dlast, ddecay, drate or ds0");
    need((uintptr_t)kept % 16 == 0, "kept must be 16-byte aligned");
    const DeltaWork w = delta_work(p, true, workspace);
    need_workspace(workspace, workspace_bytes, w.bytes);
    DeviceGuard dg(d->device);
    const hipStream_t st = (hipStream_t)d->stream;
    a.lengths = lengths;
    const int64_t cells = p.chunks / a.group;
    const bool vec = a.dk % 8 == 0 && a.dv % 8 == 0 && words(a.q, q) && words(a.k, k) && words(a.y, dy) &&
                     (uintptr_t)dv % 16 == 0;
    with_value(d->dtype, [&](auto zero) {
      using T = decltype(zero);
      with_flag(vec, [&](auto flag) {
        with_keys(a.dk, [&](auto keys) {
          constexpr int DK = decltype(keys)::value;
          constexpr bool VEC = decltype(flag)::value;
          if (p.chunks)
            hipLaunchKernelGGL(HIP_KERNEL_NAME(k_delta_chunk<T, VEC, DK, true>),
                               dim3((unsigned)std::min(p.chunks, kMaxBlocks)), dim3(kChunk<T> * 4), 0, st, a, (const T*)q,
                               (const T*)k, decay, rate, w.chunk);
          constexpr auto back = k_delta_back<T, VEC, DK>;
          constexpr size_t lds = ScanLds<T, DK, true>::all;
          static_assert(lds <= 160 * 1024, "LDS");
          allow_lds(back, lds);
          hipLaunchKernelGGL(back, scan_grid(p), dim3(512), lds, st, a, p.blocks, (const T*)q, (const T*)k, (const T*)dy,
                             dlast, (const char*)w.chunk, ds0, w.dstates, w.xs);
          if (!p.chunks) return;
          with_flag(a.group > 1, [&](auto group) {
            constexpr auto grad = k_delta_grad<T, VEC, DK, decltype(group)::value>;
            constexpr size_t more = GradLds<T, DK>::bytes;
            static_assert(more <= 160 * 1024, "LDS");
            allow_lds(grad, more);
            hipLaunchKernelGGL(grad, dim3((unsigned)std::min<int64_t>(cells, kCUs)), dim3(512), more, st, a, (const T*)q,
                               (const T*)k, (const T*)dy, decay, rate, kept, kept + kept_states(p), (const float*)w.dstates,
                               (const float*)w.xs, DeltaGradOut{dq, dk, dv, ddecay, drate});
          });
        });
      });
    });
    HIPCHECK(hipGetLastError());
  });
}

ms_status ms_gated_delta_step(const ms_gated_delta_step_desc* d, const void* q, const void* k, const void* v,
                              const float* decay, const float* rate, float* state, const int32_t* slots, void* y) {
  return guarded([&] {
    need(d != nullptr, "NULL descriptor");
    need(d->rows >= 0 && d->rows < ((int64_t)1 << 31) && d->n_slots >= 0 && d->n_slots < ((int64_t)1 << 31),
         "rows and n_slots must be in [0, 2^31)");
    need(d->key_heads >= 1 && d->heads >= 1 && d->heads <= 65536 && d->heads % d->key_heads == 0,
         "heads must be in [1, 65536], a multiple of key_heads");
    need(d->keys >= 1 && d->keys <= 128, "keys must be in [1, 128]");
    need(d->values >= 1 && d->values <= 65536, "values must be in [1, 65536]");
    need_dtype(d->dtype);
    need(std::isfinite((float)d->scale), "scale must be finite in 32 bits");
    DeltaStepArgs a{};
    const auto pair = [&](const int64_t* s, int64_t heads, int64_t dim, int64_t* to) {
      const bool packed = s[0] == 0 && s[1] == 0;
      to[0] = packed ? heads * dim : s[0], to[1] = packed ? dim : s[1];
      need(to[0] >= 0 && to[1] >= 0 && to[0] < kMaxStride && to[1] < kMaxStride, "strides must be in [0, 2^40)");
    };
    pair(d->q_stride, d->key_heads, d->keys, a.q);
    pair(d->k_stride, d->key_heads, d->keys, a.k);
    pair(d->v_stride, d->heads, d->values, a.v);
    pair(d->y_stride, d->heads, d->values, a.y);
    pair(d->decay_stride, d->heads, 1, a.decay);
    pair(d->rate_stride, d->heads, 1, a.rate);
    const int64_t matrices = d->heads * d->keys * d->values;
    a.state = d->state_stride ? d->state_stride : matrices;
    need(a.state >= matrices && a.state < kMaxStride, "strides between slots must be at least heads * keys * values");
    if (d->rows == 0) return;
    need(walk_apart({0, a.y[0], a.y[1]}, 1, d->rows, d->heads, d->values), "rows or heads of y overlap");
    need(q && k && v && decay && rate && y && (state || d->n_slots == 0), "NULL array");
    for (const void* x : {q, k, v, (const void*)y}) need_aligned(x, size_of(d->dtype), "q, k, v or y");
    for (const void* x : {(const void*)decay, (const void*)rate, (const void*)state, (const void*)slots})
      need_aligned(x, 4, "decay, rate, state or slots");
    const int64_t es = (int64_t)size_of(d->dtype);
    const auto runs = [&](const void* x, const int64_t* s, int64_t heads, int64_t dim, int64_t size) {
      Runs r{x, dim * size, {{s[0] * size, d->rows}, {s[1] * size, heads}}};
      if (d->rows > 1 && heads > 1 && s[0] < s[1]) std::swap(r.level[0], r.level[1]);
      return r;
    };
    const Runs to = runs(y, a.y, d->heads, d->values, es);
    const bool same = y == v && (d->rows == 1 || a.y[0] == a.v[0]) && (d->heads == 1 || a.y[1] == a.v[1]);
    need((same || !may_share(to, runs(v, a.v, d->heads, d->values, es))) &&
             !may_share(to, runs(q, a.q, d->key_heads, d->keys, es)) && !may_share(to, runs(k, a.k, d->key_heads, d->keys, es)) &&
             !may_share(to, runs(decay, a.decay, d->heads, 1, 4)) && !may_share(to, runs(rate, a.rate, d->heads, 1, 4)) &&
             (d->n_slots == 0 || !may_share(to, Runs{state, matrices * 4, {{a.state * 4, d->n_slots}, {0, 1}}})) &&
             (!slots || !may_share(to, Runs{slots, d->rows * 4, {{0, 1}, {0, 1}}})),
         "y overlaps another array (it may be v itself)");
    a.rows = d->rows, a.slots = d->n_slots, a.heads = (int32_t)d->heads, a.group = (int32_t)(d->heads / d->key_heads);
    a.dk = (int32_t)d->keys, a.dv = (int32_t)d->values, a.scale = (float)d->scale;
    DeviceGuard dg(d->device);
    const bool vec = a.dv % 4 == 0 && a.state % 4 == 0 && (uintptr_t)state % 16 == 0;
    const int width = vec ? 4 : 1;
    int32_t nl = 1;
    while (nl < 32 && nl * width < a.dv) nl *= 2;
    const int32_t tiles = (a.dv + nl * width - 1) / (nl * width);
    const int64_t all = d->rows * d->heads * tiles;
    with_value(d->dtype, [&](auto zero) {
      using T = decltype(zero);
      with_flag(vec, [&](auto flag) {
        constexpr int V = decltype(flag)::value ? 4 : 1;
        hipLaunchKernelGGL(HIP_KERNEL_NAME(k_delta_step<T, V>), dim3((unsigned)std::min(all, kMaxBlocks)), dim3(256), 0,
                           (hipStream_t)d->stream, a, nl, tiles, (const T*)q, (const T*)k, (const T*)v, decay, rate, state,
                           slots, (T*)y);
      });
    });
    HIPCHECK(hipGetLastError());
  });
}

ms_status ms_group_norm_workspace(const ms_group_norm_desc* d, int32_t grad, int64_t* bytes_out) {
  return guarded([&] {
    const Norm p = check_norm(d);
    need(bytes_out != nullptr, "NULL output");
    *bytes_out = norm_most(p, d->dtype, grad != 0);
  });
}

ms_status ms_group_norm(const ms_group_norm_desc* d, const void* x, const float* weight, const float* bias,
                        const int32_t* lengths, void* y, float* kept, void* workspace, int64_t workspace_bytes) {
  return guarded([&] {
    Norm p = check_norm(d);
    NormArgs& a = p.a;
    if (a.batch == 0 || a.positions == 0) return;
    const size_t es = size_of(d->dtype);
    need(walk_apart({0, a.yb, a.yt}, 1, a.batch, a.positions, p.channels), "rows or positions of y overlap");
    need(x && y, "NULL array");
    for (const void* q : {x, (const void*)y}) need_aligned(q, es, "x or y");
    for (const void* q : {(const void*)weight, (const void*)bias, (const void*)lengths, (const void*)kept})
      need_aligned(q, 4, "weight, bias, lengths or kept");
    need_workspace(workspace, workspace_bytes, norm_most(p, d->dtype, false));
    norm_choose(p, Wide(es).of(a.width).of(a.xb).of(a.xt).of(a.yb).of(a.yt).at(x, es).at(y, es).at(weight, 4).at(bias, 4).v,
                false);
    const NormWork w = norm_work(p, false, workspace);
    a.weight = weight, a.bias = bias, a.lengths = lengths, a.kept = kept;
    DeviceGuard dg(d->device);
    const hipStream_t st = (hipStream_t)d->stream;
    with_type<8, 4>(d->dtype, p.v, [&](auto zero, auto width) {
      using T = decltype(zero);
      constexpr int V = decltype(width)::value;
      if (a.team) {
        // groups are counted in 32 bits: as many rows at a time as that allows
        const int64_t most = std::max<int64_t>(1, ((int64_t)1 << 30) / a.groups), batch = a.batch;
        for (int64_t b0 = 0; b0 < batch; b0 += most) {
          NormArgs part = a;
          part.batch = std::min(most, batch - b0);
          if (a.lengths) part.lengths += b0;
          if (a.kept) part.kept += b0 * a.groups * 2;
          const int64_t blocks = (part.batch * a.groups * a.team + 255) / 256;
          with_words(p.shape.words, [&](auto each) {
            with_flag(a.team > 64, [&](auto many) {
              with_flag(a.positions == 1, [&](auto one) {
                hipLaunchKernelGGL(
                    HIP_KERNEL_NAME(k_norm_team<T, V, decltype(each)::value, decltype(many)::value, decltype(one)::value>),
                    dim3((unsigned)std::min(blocks, kMaxBlocks / 2)), dim3(256), 0, st, part, (const T*)x + b0 * a.xb,
                    (T*)y + b0 * a.yb);
              });
            });
          });
        }
        return;
      }
      if (!kept) a.kept = w.sums;
      hipLaunchKernelGGL(HIP_KERNEL_NAME(k_norm_sums<T, V>), dim3(norm_grid(p)), dim3(256), 0, st, a, (const T*)x, w.parts);
      hipLaunchKernelGGL(HIP_KERNEL_NAME(k_norm_join<V>), dim3((unsigned)std::min(a.batch * a.groups, kMaxBlocks)), dim3(256),
                         0, st, a, (const float*)w.parts);
      hipLaunchKernelGGL(HIP_KERNEL_NAME(k_norm_apply<T, V>), dim3(norm_grid(p)), dim3(256), 0, st, a, (const T*)x, (T*)y);
    });
    HIPCHECK(hipGetLastError());
  });
}

ms_status ms_group_norm_grad(const ms_group_norm_desc* d, const void* x, const float* weight, const float* bias,
                             const int32_t* lengths, const float* kept, const void* dy, void* dx, float* dweight,
                             float* dbias, void* workspace, int64_t workspace_bytes) {
  return guarded([&] {
    Norm p = check_norm(d);
    NormArgs& a = p.a;
    const bool none = a.batch == 0 || a.positions == 0;
    const size_t es = size_of(d->dtype);
    need(none || (x && kept && dy && dx), "NULL array");
    need(dweight && dbias, "NULL array");
    for (const void* q : {x, dy, (const void*)dx}) need_aligned(q, es, "x, dy or dx");
    for (const void* q : {(const void*)weight, (const void*)bias, (const void*)lengths, (const void*)kept, (const void*)dweight,
                          (const void*)dbias})
      need_aligned(q, 4, "weight, bias, lengths, kept, dweight or dbias");
    if (!none) need_workspace(workspace, workspace_bytes, norm_most(p, d->dtype, true));
    DeviceGuard dg(d->device);
    const hipStream_t st = (hipStream_t)d->stream;
    const auto columns = [&](const float* parts, int64_t rows, float* next) {
      const int64_t blocks = (2 * p.channels + 31) / 32;
      while (true) {
        const int64_t runs = std::max<int64_t>(1, (rows + kColumnRows - 1) / kColumnRows);
        hipLaunchKernelGGL(k_norm_columns, dim3((unsigned)std::min(blocks * runs, kMaxBlocks / 4)), dim3(1024), 0, st, parts, rows, p.channels,
                           runs > 1 ? next : nullptr, dweight, dbias);
        if (runs == 1) break;
        parts = next, rows = runs, next += runs * 2 * p.channels;
      }
      HIPCHECK(hipGetLastError());
    };
    if (none) return columns(nullptr, 0, nullptr);
    norm_choose(p, Wide(es).of(a.width).of(a.xb).of(a.xt).of(a.yb).of(a.yt).at(x, es).at(dy, es).at(dx, es).at(weight, 4)
                       .at(bias, 4).v, true);
    const NormWork w = norm_work(p, true, workspace);
    a.weight = weight, a.bias = bias, a.lengths = lengths, a.kept = (float*)kept;
    with_type<8, 4>(d->dtype, p.v, [&](auto zero, auto width) {
      using T = decltype(zero);
      constexpr int V = decltype(width)::value;
      if (a.team) {
        const int64_t blocks = ((int64_t)a.lanes * a.groups * a.team + 255) / 256;
        with_words(p.shape.words, [&](auto each) {
          with_flag(a.team > 64, [&](auto many) {
            hipLaunchKernelGGL(HIP_KERNEL_NAME(k_norm_team_grad<T, V, decltype(each)::value, decltype(many)::value>),
                               dim3((unsigned)blocks), dim3(256), 0, st, a, (const T*)x, (const T*)dy, (T*)dx, w.parts);
          });
        });
        return;
      }
      hipLaunchKernelGGL(HIP_KERNEL_NAME(k_norm_grad_sums<T, V>), dim3(norm_grid(p)), dim3(256), 0, st, a, (const T*)x,
                         (const T*)dy, w.parts);
      hipLaunchKernelGGL(k_norm_grad_join, dim3((unsigned)std::min(a.batch * a.groups, kMaxBlocks)), dim3(256), 0, st, a,
                         (const float*)w.parts, w.sums);
      hipLaunchKernelGGL(HIP_KERNEL_NAME(k_norm_grad_apply<T, V>), dim3(norm_grid(p)), dim3(256), 0, st, a, (const T*)x,
                         (const T*)dy, (const float*)w.sums, (T*)dx);
    });
    columns(w.parts, a.team ? (int64_t)a.lanes * a.pieces : a.batch * a.runs, w.next);
  });
}

}  // extern "C"
