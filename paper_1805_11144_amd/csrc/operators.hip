// The operators on device arrays of the C ABI: argument checks, workspace
// layouts and launches.  The kernels are in kernels_embed.hpp,
// kernels_gated.hpp, kernels_orth.hpp and kernels_orth_small.hpp.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <string>

#include "host.hpp"
#include "kernels_embed.hpp"
#include "kernels_gated.hpp"
#include "kernels_orth.hpp"
#include "kernels_orth_small.hpp"
#include "operators_host.hpp"
#include "operators_rules.hpp"

using namespace ms;

namespace {

// ------------------------------------------------------------------ tables
struct Embed {
  int64_t ts, os;
};

Embed check_embed(const ms_embed_desc* d) {
  need(d != nullptr, "NULL descriptor");
  need(d->n_tokens >= 0 && d->n_tokens < ((int64_t)1 << 29), "n_tokens must be in [0, 2^29)");
  need(d->vocab >= 1 && d->vocab < ((int64_t)1 << 31), "vocab must be in [1, 2^31)");
  need(d->dim >= 1 && d->dim < (1 << 24), "dim must be in [1, 2^24)");
  need_dtype(d->dtype);
  need_dtype(d->grad_dtype);
  need(d->ids == MS_IDS_I32 || d->ids == MS_IDS_I64, "unknown token type");
  need(std::isfinite((float)d->scale), "scale must be finite in 32 bits");
  Embed e{d->table_stride ? d->table_stride : d->dim, d->row_stride ? d->row_stride : d->dim};
  need(e.ts >= d->dim && e.ts < kMaxStride && e.os >= d->dim && e.os < kMaxStride,
       "row strides must be at least dim");
  return e;
}

struct EmbedWork {
  uint32_t *keys[2], *pos[2], *counts, *block, *start;
  float* part;
  int64_t bytes;
};

EmbedWork embed_work(const ms_embed_desc* d, void* ws) {
  Carve c{(char*)ws};
  EmbedWork w;
  for (int i = 0; i < 2; ++i) w.keys[i] = c.take<uint32_t>(d->n_tokens), w.pos[i] = c.take<uint32_t>(d->n_tokens);
  const int64_t tiles = sort_tiles(d->n_tokens);
  w.counts = c.take<uint32_t>(tiles << kSortBits);
  w.block = tiles > kSortAll ? c.take<uint32_t>((up(tiles, kSortBlock) / kSortBlock + 1) << kSortBits) : nullptr;
  w.start = c.take<uint32_t>(d->vocab + 1);
  w.part = c.take<float>((d->n_tokens + kRun - 1) / kRun * 2 * d->dim);
  w.bytes = c.used;
  return w;
}

template <class I, int N>
void sort_small(const ms_embed_desc* d, const I* tokens, EmbedWork& w, int key_bits, hipStream_t st) {
  constexpr size_t lds = 1024 * N * 6 + 16 * 256 * 4 + 16;
  const void* k = (const void*)k_sort_small<I, N>;
  if (lds > 65536) HIPCHECK(hipFuncSetAttribute(k, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
  hipLaunchKernelGGL(HIP_KERNEL_NAME(k_sort_small<I, N>), dim3(1), dim3(1024), lds, st, tokens, (int32_t)d->n_tokens,
                     d->vocab, (key_bits + 7) / 8, w.keys[0], w.pos[0]);
}

template <class I, int BITS, int N>
void sort_tiled(const ms_embed_desc* d, const I* tokens, EmbedWork& w, int key_bits, int& in, hipStream_t st) {
  const int64_t n = d->n_tokens;
  const unsigned tiles = (unsigned)sort_tiles(n);
  for (int p = 0; p * BITS < key_bits; ++p, in ^= 1) {
    const uint32_t *k = p ? w.keys[in] : nullptr, *q = p ? w.pos[in] : nullptr;
    hipLaunchKernelGGL(HIP_KERNEL_NAME(k_sort_count<I, BITS, N>), dim3(tiles), dim3(256), 0, st, tokens, k, n, d->vocab,
                       p * BITS, w.counts);
    if (tiles > kSortAll) {
      constexpr int digits = 1 << BITS;
      const unsigned blocks = (tiles + kSortBlock - 1) / kSortBlock;
      hipLaunchKernelGGL(k_sort_prefix, dim3(blocks * (digits / 256)), dim3(256), 0, st, w.counts, w.block, (int32_t)tiles,
                         digits);
      hipLaunchKernelGGL(k_sort_blocks, dim3(digits / 256), dim3(256), 0, st, w.block, (int32_t)blocks, digits);
    }
    hipLaunchKernelGGL(HIP_KERNEL_NAME(k_sort_move<I, BITS, N>), dim3(tiles), dim3(256), 0, st, tokens, k, q, n, d->vocab,
                       p * BITS, (const uint32_t*)w.counts, (const uint32_t*)(tiles > kSortAll ? w.block : nullptr),
                       w.keys[in ^ 1], w.pos[in ^ 1]);
  }
}

// Sorted pairs to keys[in], pos[in].
template <class I>
void sort_tokens(const ms_embed_desc* d, const I* tokens, EmbedWork& w, int& in, hipStream_t st) {
  const int64_t n = d->n_tokens;
  int key_bits;
  const int bits = sort_bits(d->vocab, &key_bits), small = sort_small_items(n);   // keys are in [0, vocab]
  in = 0;
  if (small == 1) return sort_small<I, 1>(d, tokens, w, key_bits, st);
  if (small == 4) return sort_small<I, 4>(d, tokens, w, key_bits, st);
  const auto with = [&](auto digit) {
    constexpr int BITS = decltype(digit)::value;
    switch (sort_items(n)) {
      case 4: return sort_tiled<I, BITS, 4>(d, tokens, w, key_bits, in, st);
      case 8: return sort_tiled<I, BITS, 8>(d, tokens, w, key_bits, in, st);
      default: return sort_tiled<I, BITS, 16>(d, tokens, w, key_bits, in, st);
    }
  };
  if (bits == 8) with(std::integral_constant<int, 8>{});
  else if (bits == 9) with(std::integral_constant<int, 9>{});
  else with(std::integral_constant<int, 10>{});
}

// ------------------------------------------------------------------ gated
struct Gated {
  GatedArgs a;
  int64_t keeps;
};

void stride_pair(const int64_t* s, int64_t steps, int64_t dim, int64_t& b, int64_t& t) {
  const bool packed = s[0] == 0 && s[1] == 0;
  t = packed ? dim : s[1];
  b = packed ? steps * dim : s[0];
  need(b >= 0 && t >= 0 && b < kMaxStride && t < kMaxStride, "strides must not be negative");
}

// Whether runs of `dim` values at i * si + j * sj, i < ni, j < nj, are apart: one
// stride steps over a run, the other over all that the first one reaches.
bool apart(int64_t si, int64_t ni, int64_t sj, int64_t nj, int64_t dim) {
  if (ni == 0 || nj == 0) return true;
  const auto within = [&](int64_t inner, int64_t n, int64_t outer, int64_t m) {
    return (n == 1 || inner >= dim) && (m == 1 || (__int128)outer >= (__int128)(n - 1) * inner + dim);
  };
  return within(sj, nj, si, ni) || within(si, ni, sj, nj);
}

Gated check_gated(const ms_gated_lowpass_desc* d) {
  need(d != nullptr, "NULL descriptor");
  need(d->steps >= 0 && d->steps < ((int64_t)1 << 31), "steps must be in [0, 2^31)");
  need(d->dim >= 1 && d->dim < (1 << 24), "dim must be in [1, 2^24)");
  need(d->batch >= 0 && d->batch < ((int64_t)1 << 31) && d->batch * d->dim < ((int64_t)1 << 31),
       "batch * dim must be below 2^31");
  need_dtype(d->dtype);
  Gated g{};
  GatedArgs& a = g.a;
  a.batch = d->batch, a.steps = d->steps, a.dim = d->dim;
  stride_pair(d->v_stride, d->steps, d->dim, a.vb, a.vt);
  stride_pair(d->g_stride, d->steps, d->dim, a.gb, a.gt);
  stride_pair(d->y_stride, d->steps, d->dim, a.yb, a.yt);
  g.keeps = (d->steps + kKeep - 1) / kKeep;
  return g;
}

// Scratch memory of chunks that run side by side: their maps and states, the
// ticket.
struct GatedWork {
  uint64_t* maps;
  uint32_t *states, *ticket;
  int64_t bytes;
};

GatedWork gated_work(const Gated& g, void* ws) {
  const int64_t channels = g.a.batch * g.a.dim, chunks = (g.keeps + kGatedWaves - 1) / kGatedWaves;
  Carve c{(char*)ws};
  GatedWork w{};
  if (chunks > 1) {
    w.maps = c.take<uint64_t>(chunks * channels);
    w.states = c.take<uint32_t>(chunks / kSpan * channels);
    w.ticket = c.take<uint32_t>(1);
  }
  w.bytes = c.used;
  return w;
}

// Calls f(args, link, span, grid) with the shape's choices as compile-time
// values: once, or for as many groups at a time as a grid holds (its threads fit
// 31 bits).
template <class F>
void gated_launch(const GatedShape& s, GatedArgs a, F&& f) {
  const auto with = [&](auto link) {
    const int64_t all = s.link ? a.nchunk * a.groups : a.groups, most = ((int64_t)1 << 31) / s.threads;
    for (a.first = 0; a.first < all; a.first += most) {
      const dim3 grid((unsigned)std::min(all - a.first, most));
      if (s.span) f(a, link, std::true_type{}, grid);
      else f(a, link, std::false_type{}, grid);
    }
  };
  if (s.link) with(std::true_type{});
  else with(std::false_type{});
}

void gated_clear(GatedArgs& a, const GatedWork& w, hipStream_t st) {
  a.maps = w.maps, a.states = w.states, a.ticket = w.ticket;
  const int64_t words = ((char*)w.ticket - (char*)w.maps) / 4;
  hipLaunchKernelGGL(k_gated_clear, dim3((unsigned)std::min<int64_t>((words + 255) / 256, 2048)), dim3(256), 0, st,
                     (uint32_t*)w.maps, words, w.ticket);
}

// ------------------------------------------------------------------- orth
struct Orth {
  int64_t n, m;
  OrthShape shape;        // tiled
  double sx, sa, sq;      // scales of X, A and Q
  int grown[101];         // log2 of what the steps before a step, at most, multiply an iterate's norm by
  int64_t xm, xr, om, orow;
  int small;              // row tiles of 16 where a matrix fits into one workgroup's LDS, else 0
  int64_t stride;         // of its rows there
};

constexpr int64_t kOrthLds = 156 * 1024;   // of 160 KB

Orth check_orth(const ms_orth_desc* d) {
  need(d != nullptr, "NULL descriptor");
  need(d->rows >= 1 && d->rows <= 65536 && d->cols >= 1 && d->cols <= 65536, "rows and cols must be in [1, 65536]");
  need(d->batch >= 0, "batch must not be negative");
  need(d->batch <= kMaxBlocks, "too many matrices of this size");
  need(d->steps >= 1 && d->steps <= 100, "steps must be in [1, 100]");
  need_dtype(d->dtype);
  need(d->eps >= 0 && std::isfinite(d->eps), "eps must be finite and not negative");
  Orth o;
  auto pair = [&](const int64_t* s, int64_t& mat, int64_t& row) {
    const bool packed = s[0] == 0 && s[1] == 0;
    row = packed ? d->cols : s[1];
    mat = packed ? d->rows * d->cols : s[0];
    need(row >= d->cols && row < kMaxStride && mat >= 0 && mat < kMaxStride, "strides must be at least a row");
  };
  pair(d->x_stride, o.xm, o.xr);
  pair(d->out_stride, o.om, o.orow);
  o.n = std::min(d->rows, d->cols), o.m = std::max(d->rows, d->cols);
  o.shape = orth_shape(d->batch, o.n, o.m);
  o.stride = up(o.m, 64) + 4;
  o.small = (int)up(o.n, 16) / 16;
  if (o.small > 4 || orth_small_floats(o.small, o.stride) * 4 > kOrthLds) o.small = 0;
  // workgroups of up to 512 threads
  const int64_t groups = o.small ? 1 : std::max<int64_t>(kOrthParts, (o.shape.np / 64) * (o.shape.mp / 64));
  need(d->batch <= kMaxBlocks / 2 / groups, "too many matrices of this size");
  // How large an iterate's singular values and the polynomial can get: the
  // first are at most 1, and f(s) = s (c0 + c1 s^2 + c2 s^4) takes its extremes
  // over [0, top] at the ends or where its derivative is 0.
  double top = 1.0, poly = 0.0;
  const double *c = d->coef;
  need(std::isfinite(c[0]) && std::isfinite(c[1]) && std::isfinite(c[2]), "coefficients must be finite");
  double bound = 1.0, grown = 0.0;
  for (int k = 0; k < d->steps; ++k) {
    o.grown[k] = (int)std::ceil(grown);
    const auto q = [&](double t) { return std::fabs(c[0] + c[1] * t + c[2] * t * t); };   // t = s^2
    double most_f = top * q(top * top), most_q = std::max(q(0.0), q(top * top));
    const auto at = [&](double t) {
      if (t > 0.0 && t < top * top) most_f = std::max(most_f, std::sqrt(t) * q(t)), most_q = std::max(most_q, q(t));
    };
    if (c[2] != 0.0) {
      at(-c[1] / (2.0 * c[2]));
      const double disc = 9.0 * c[1] * c[1] - 20.0 * c[0] * c[2];
      if (disc >= 0.0) at((-3.0 * c[1] + std::sqrt(disc)) / (10.0 * c[2])), at((-3.0 * c[1] - std::sqrt(disc)) / (10.0 * c[2]));
    } else if (c[1] != 0.0) {
      at(-c[0] / (3.0 * c[1]));
    }
    poly = std::max(poly, most_q);
    grown += std::log2(std::max(most_q, 1e-30));
    top = most_f;
    bound = std::max(bound, top);
    need(bound <= 1000.0 && poly <= 1000.0, "the coefficients let the iterates grow past 1000");
  }
  o.grown[d->steps] = (int)std::ceil(grown);
  // an entry is at most the largest singular value; a factor of two to spare
  const auto scale = [](double b) { return std::ldexp(1.0, (int)std::floor(std::log2(32768.0 / b))); };
  o.sx = scale(bound), o.sa = scale(bound * bound), o.sq = scale(std::max(poly, 1e-20));
  return o;
}

struct OrthWork {
  double* parts;
  int32_t* lift;
  half_t *x, *t[2], *a, *q;
  float* sums;
  int64_t bytes;
};

OrthWork orth_work(const ms_orth_desc* d, const Orth& o, void* ws) {
  Carve c{(char*)ws};
  OrthWork w{};
  if (o.small) return w;
  [[maybe_unused]] const auto [pad, np, mp, split] = o.shape;
  const int64_t big = d->batch * kPair * np * mp, small = d->batch * kPair * np * np;
  w.parts = c.take<double>(d->batch * kOrthParts);
  w.lift = c.take<int32_t>(d->batch);
  w.x = c.take<half_t>(big);
  w.t[0] = c.take<half_t>(big);
  w.t[1] = c.take<half_t>(big);
  w.a = c.take<half_t>(small);
  w.q = c.take<half_t>(small);
  w.sums = c.take<float>(split > 1 ? split * d->batch * np * np : 0);
  w.bytes = c.used;
  return w;
}

template <int END, class T, int TILE, int WC, int ST, int KG>
void orth_launch(OrthGemm g, const OrthTiles& t, hipStream_t st) {
  constexpr size_t lds = KG * ST * kPair * 2 * TILE * kOrthSlice * sizeof(half_t);
  static_assert(lds >= (KG - 1) * TILE * TILE * sizeof(float) && lds <= 160 * 1024, "LDS");
  g.per = (uint32_t)t.per, g.whole = (uint32_t)t.whole;
  constexpr auto k = k_orth_gemm<TILE, WC, kOrthSlice, ST, KG, END, T>;
  if (lds >= 65536) HIPCHECK(hipFuncSetAttribute((const void*)k, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
  hipLaunchKernelGGL(k, dim3((unsigned)(up(t.whole, 8) + 4 * t.over)), dim3(128 * WC * KG), lds, st, g);
}

template <int END, class T>
void orth_gemm(const OrthGemm& g, int64_t pad, int64_t batch, hipStream_t st) {
  constexpr bool SYM = END == kEndGram || END == kEndPoly;
  const OrthTile kind = orth_choose(pad, SYM, batch, g.M, g.N, nullptr);
  const OrthTiles t = orth_tiles(kind, SYM, batch, g.M, g.N);
  if (kind == kTile64) orth_launch<END, T, 64, 2, 3, 2>(g, t, st);
  else if (kind == kTile128) orth_launch<END, T, 128, 2, 2, 1>(g, t, st);
  else orth_launch<END, T, 256, 4, 2, 1>(g, t, st);
}

// T: type of x (or the gradient); UPDATE: with momentum, into a weight.
template <class T, bool UPDATE>
void orth_run(const ms_orth_desc* d, const Orth& o, const OrthSrc& src, OrthWork& w, OrthGemm out, hipStream_t st) {
  const auto [pad, np, mp, split] = o.shape;
  const int64_t blocks = d->batch * (np / 64) * (mp / 64);
  const dim3 norms((unsigned)(d->batch * kOrthParts));
  const auto norm = [&](auto width) {
    hipLaunchKernelGGL(HIP_KERNEL_NAME(k_orth_norm<T, UPDATE, decltype(width)::value>), norms, dim3(256), 0, st, src, w.parts);
  };
  // packed matrices as one run of values, four at a time where that is aligned
  if (src.row != src.cols) norm(std::integral_constant<int, 0>{});
  else if (src.rows * src.cols % 4 == 0 && src.mat % 4 == 0 && (uintptr_t)src.x % (4 * sizeof(T)) == 0 &&
           (uintptr_t)src.momentum % 16 == 0)
    norm(std::integral_constant<int, 4>{});
  else norm(std::integral_constant<int, 1>{});
  hipLaunchKernelGGL(HIP_KERNEL_NAME(k_orth_first<T, UPDATE, kOrthSlice>), dim3((unsigned)blocks), dim3(256), 0, st, src,
                     (const double*)w.parts, d->eps, o.sx, w.x, w.t[0], w.lift, (int32_t)np, (int32_t)mp);
  using R = std::conditional_t<UPDATE, float, T>;
  for (int k = 0; k < d->steps; ++k) {
    OrthGemm g{};
    g.batch = out.batch = (uint32_t)d->batch, g.parts = out.parts = 1;
    g.lift = out.lift = w.lift;
    g.grown = out.grown = o.grown[k], g.grows = out.grows = o.grown[k + 1];
    g.slices = out.slices = INT32_MAX / 2;
    g.l = g.r = w.x, g.M = g.N = (int32_t)np, g.K = (int32_t)mp, g.c = w.a;
    g.f = (float)(o.sa / (o.sx * o.sx));
    if (split > 1) {
      g.sums = w.sums, g.parts = split, g.slices = (int32_t)((mp / kOrthSlice + split - 1) / split);
      orth_launch<kEndPart, R, 64, 2, 3, 2>(g, orth_tiles(kTile64, true, d->batch * split, np, np), st);
      hipLaunchKernelGGL(HIP_KERNEL_NAME(k_orth_join<kOrthSlice>), dim3((unsigned)((d->batch * np * np + 255) / 256)), dim3(256),
                         0, st, g);
    } else {
      orth_gemm<kEndGram, R>(g, pad, d->batch, st);
    }
    g.parts = 1, g.slices = INT32_MAX / 2;
    g.l = g.r = w.a, g.K = (int32_t)np, g.c = w.q, g.a = w.a;
    g.f = (float)(d->coef[2] * o.sq / (o.sa * o.sa));
    g.c0 = (float)(d->coef[0] * o.sq), g.c1 = (float)(d->coef[1] * o.sq / o.sa);
    orth_gemm<kEndPoly, R>(g, pad, d->batch, st);
    OrthGemm x = out;
    x.l = w.q, x.r = w.t[k % 2], x.M = (int32_t)np, x.N = (int32_t)mp, x.K = (int32_t)np;
    if (k + 1 < d->steps) {
      x.c = w.x, x.ct = w.t[(k + 1) % 2], x.f = (float)(1.0 / o.sq);
      orth_gemm<kEndNext, R>(x, pad, d->batch, st);
    } else {
      x.f = (float)(1.0 / (o.sq * o.sx));
      orth_gemm<UPDATE ? kEndUpdate : kEndOut, R>(x, pad, d->batch, st);
    }
  }
  HIPCHECK(hipGetLastError());
}

template <class T, bool UPDATE>
void orth_small(const ms_orth_desc* d, const Orth& o, const OrthSrc& src, const OrthGemm& out, hipStream_t st) {
  OrthSmall p{};
  p.src = src, p.out = out.out, p.omat = out.mat, p.orow = out.row;
  p.n = (int32_t)o.n, p.m = (int32_t)o.m, p.stride = (int32_t)o.stride, p.steps = d->steps;
  p.c0 = (float)d->coef[0], p.c1 = (float)d->coef[1], p.c2 = (float)d->coef[2];
  p.keep = out.keep, p.rate = out.rate, p.eps = d->eps;
  const size_t lds = (size_t)orth_small_floats(o.small, o.stride) * 4;
  const auto go = [&](auto nt) {
    constexpr int NT = decltype(nt)::value;
    if (lds > 65536)
      HIPCHECK(hipFuncSetAttribute((const void*)k_orth_small<T, UPDATE, NT>, hipFuncAttributeMaxDynamicSharedMemorySize,
                                   (int)kOrthLds));
    hipLaunchKernelGGL(HIP_KERNEL_NAME(k_orth_small<T, UPDATE, NT>), dim3((unsigned)d->batch), dim3(64 * kOrthWaves), lds, st,
                       p);
  };
  switch (o.small) {
    case 1: go(std::integral_constant<int, 1>{}); break;
    case 2: go(std::integral_constant<int, 2>{}); break;
    case 3: go(std::integral_constant<int, 3>{}); break;
    default: go(std::integral_constant<int, 4>{});
  }
  HIPCHECK(hipGetLastError());
}

template <class T, bool UPDATE>
void orth(const ms_orth_desc* d, const Orth& o, const OrthSrc& src, OrthWork& w, const OrthGemm& out, hipStream_t st) {
  if (o.small) orth_small<T, UPDATE>(d, o, src, out, st);
  else orth_run<T, UPDATE>(d, o, src, w, out, st);
}

}  // namespace

extern "C" {

ms_status ms_embed(const ms_embed_desc* d, const void* tokens, const void* table, void* out) {
  return guarded([&] {
    const Embed e = check_embed(d);
    if (d->n_tokens == 0) return;
    need(tokens && table && out, "NULL array");
    const size_t es = size_of(d->dtype);
    need_aligned(tokens, d->ids == MS_IDS_I64 ? 8 : 4, "tokens");
    need_aligned(table, es, "table");
    need_aligned(out, es, "out");
    DeviceGuard dg(d->device);
    const hipStream_t st = (hipStream_t)d->stream;
    const int64_t v = Wide(es).of(d->dim).of(e.ts).of(e.os).at(table, es).at(out, es).v;
    const int32_t nv = (int32_t)(d->dim / v), tpr = threads_per_row(nv);
    constexpr int kLookupRows = 4;
    const int64_t lookups = (d->n_tokens + kLookupRows - 1) / kLookupRows;
    with_type<8, 4>(d->dtype, v, [&](auto zero, auto width) {
      using T = decltype(zero);
      constexpr int V = decltype(width)::value;
      auto go = [&](auto id) {
        using I = decltype(id);
        hipLaunchKernelGGL(HIP_KERNEL_NAME(k_embed<T, I, V, kLookupRows>), dim3(row_blocks(lookups, tpr)), dim3(256), 0, st,
                           (const I*)tokens, (const T*)table, (T*)out, d->n_tokens, d->vocab, nv, tpr, e.ts, e.os,
                           (float)d->scale);
      };
      if (d->ids == MS_IDS_I64) go((int64_t)0);
      else go((int32_t)0);
    });
    HIPCHECK(hipGetLastError());
  });
}

ms_status ms_embed_grad_workspace(const ms_embed_desc* d, int64_t* bytes_out) {
  return guarded([&] {
    check_embed(d);
    need(bytes_out != nullptr, "NULL output");
    *bytes_out = embed_work(d, nullptr).bytes;
  });
}

ms_status ms_embed_grad(const ms_embed_desc* d, const void* tokens, const void* drows, void* dtable, void* workspace,
                        int64_t workspace_bytes) {
  return guarded([&] {
    const Embed e = check_embed(d);
    need(dtable && (d->n_tokens == 0 || (tokens && drows)), "NULL array");
    const size_t es = size_of(d->dtype), gs = size_of(d->grad_dtype);
    need_aligned(tokens, d->ids == MS_IDS_I64 ? 8 : 4, "tokens");
    need_aligned(drows, es, "drows");
    need_aligned(dtable, gs, "dtable");
    EmbedWork w = embed_work(d, workspace);
    need_workspace(workspace, workspace_bytes, w.bytes);
    DeviceGuard dg(d->device);
    const hipStream_t st = (hipStream_t)d->stream;
    int in = 0;
    if (d->n_tokens > 0) {
      if (d->ids == MS_IDS_I64) sort_tokens(d, (const int64_t*)tokens, w, in, st);
      else sort_tokens(d, (const int32_t*)tokens, w, in, st);
    }
    const int64_t v = Wide(es).of(d->dim).of(e.ts).of(e.os).at(drows, es).at(dtable, gs).v;
    const int32_t nv = (int32_t)(d->dim / v), tpr = threads_per_row(nv);
    const int32_t tpc = std::max(tpr, 64);   // a chunk's threads: whole wavefronts
    const int64_t chunks = (d->n_tokens + kRun - 1) / kRun;
    const unsigned pieces = (unsigned)((chunks + 256 / tpc - 1) / (256 / tpc));
    const unsigned searches = (unsigned)std::min<int64_t>((d->vocab + 256) / 256, kMaxBlocks / 2);
    with_type<8, 4>(d->dtype, v, [&](auto zero, auto width) {
      using T = decltype(zero);
      constexpr int V = decltype(width)::value;
      hipLaunchKernelGGL(HIP_KERNEL_NAME(k_embed_pieces<T, V>), dim3(searches + pieces), dim3(256), 0, st,
                         (const uint32_t*)w.keys[in], (const uint32_t*)w.pos[in], d->n_tokens, d->vocab, (const T*)drows, nv,
                         tpc, e.os, searches, w.start, w.part);
      auto go = [&](auto gz, auto full) {
        using D = decltype(gz);
        constexpr bool FULL = decltype(full)::value;
        hipLaunchKernelGGL(HIP_KERNEL_NAME(k_embed_sum<T, D, V, FULL>), dim3(row_blocks(d->vocab, tpr)), dim3(256), 0, st,
                           (const uint32_t*)w.pos[in], (const uint32_t*)w.start, (const T*)drows, (const float*)w.part,
                           (D*)dtable, d->vocab, nv, tpr, e.os, e.ts, (float)d->scale, d->accumulate);
      };
      const auto out = [&](auto full) {
        if (d->grad_dtype == MS_DTYPE_BF16) go((__bf16)0.0f, full);
        else go(0.0f, full);
      };
      if (tpr >= 64) out(std::true_type{});
      else out(std::false_type{});
    });
    HIPCHECK(hipGetLastError());
  });
}

ms_status ms_gated_lowpass_kept(const ms_gated_lowpass_desc* d, int64_t* elements_out) {
  return guarded([&] {
    const Gated g = check_gated(d);
    need(elements_out != nullptr, "NULL output");
    *elements_out = g.a.batch * g.keeps * g.a.dim;
  });
}

ms_status ms_gated_lowpass_workspace(const ms_gated_lowpass_desc* d, int64_t* bytes_out) {
  return guarded([&] {
    const Gated g = check_gated(d);
    need(bytes_out != nullptr, "NULL output");
    *bytes_out = gated_work(g, nullptr).bytes;
  });
}

ms_status ms_gated_lowpass(const ms_gated_lowpass_desc* d, const void* v, const void* g, const float* y0,
                           const int32_t* lengths, void* y, float* last, float* kept, void* workspace,
                           int64_t workspace_bytes) {
  return guarded([&] {
    Gated p = check_gated(d);
    GatedArgs& a = p.a;
    if (a.batch == 0) return;
    const size_t es = size_of(d->dtype);
    need(apart(a.yb, a.batch, a.yt, a.steps, a.dim), "the rows or steps of y overlap");
    need(a.steps == 0 || (v && g && y), "NULL array");
    for (const void* q : {v, g, (const void*)y}) need_aligned(q, es, "v, g or y");
    for (const void* q : {(const void*)y0, (const void*)lengths, (const void*)last, (const void*)kept})
      need_aligned(q, 4, "y0, lengths, last or kept");
    const GatedWork work = gated_work(p, workspace);
    if (a.steps > 0) need_workspace(workspace, workspace_bytes, work.bytes);
    DeviceGuard dg(d->device);
    const hipStream_t st = (hipStream_t)d->stream;
    if (a.steps == 0) {
      if (last)
        hipLaunchKernelGGL(k_gated_none, dim3((unsigned)((a.batch * a.dim + 255) / 256)), dim3(256), 0, st, y0, last,
                           a.batch * a.dim);
      HIPCHECK(hipGetLastError());
      return;
    }
    a.lengths = lengths;
    Wide wide = Wide(es).of(a.dim).of(a.vb).of(a.vt).of(a.gb).of(a.gt).of(a.yb).of(a.yt).at(v, es).at(g, es).at(y, es);
    const int64_t w = std::min<int64_t>(4 / (int64_t)es, wide.at(kept, 4).v);   // a word of 4 bytes to a lane
    a.nv = a.dim / w;
    const GatedShape shape = gated_shape(a.batch, p.keeps, a.nv);
    a.nchunk = shape.nchunk, a.groups = shape.groups, a.per_row = shape.per_row;
    if (shape.link) gated_clear(a, work, st);
    with_type<2, 1>(d->dtype, w, [&](auto zero, auto width) {
      using T = decltype(zero);
      constexpr int V = decltype(width)::value;
      gated_launch(shape, a, [&](const GatedArgs& a, auto link, auto span, dim3 grid) {
        hipLaunchKernelGGL(HIP_KERNEL_NAME(k_gated<T, V, decltype(link)::value, decltype(span)::value>), grid,
                           dim3(shape.threads), 0, st, a, (const T*)v, (const T*)g, y0, (T*)y, last, kept);
      });
    });
    HIPCHECK(hipGetLastError());
  });
}

ms_status ms_gated_lowpass_grad(const ms_gated_lowpass_desc* d, const void* v, const void* g, const float* kept,
                                const int32_t* lengths, const void* dy, const float* dlast, void* dv, void* dg,
                                float* dy0, void* workspace, int64_t workspace_bytes) {
  return guarded([&] {
    Gated p = check_gated(d);
    GatedArgs& a = p.a;
    if (a.batch == 0) return;
    const size_t es = size_of(d->dtype);
    need(a.steps == 0 || (v && g && kept && dy && dv && dg), "NULL array");
    for (const void* q : {v, g, dy, (const void*)dv, (const void*)dg}) need_aligned(q, es, "v, g, dy, dv or dg");
    for (const void* q : {(const void*)kept, (const void*)lengths, (const void*)dlast, (const void*)dy0})
      need_aligned(q, 4, "kept, lengths, dlast or dy0");
    const GatedWork work = gated_work(p, workspace);
    if (a.steps > 0) need_workspace(workspace, workspace_bytes, work.bytes);
    DeviceGuard guard(d->device);
    const hipStream_t st = (hipStream_t)d->stream;
    if (a.steps == 0) {
      if (dy0)
        hipLaunchKernelGGL(k_gated_none, dim3((unsigned)((a.batch * a.dim + 255) / 256)), dim3(256), 0, st, dlast, dy0,
                           a.batch * a.dim);
      HIPCHECK(hipGetLastError());
      return;
    }
    a.lengths = lengths;
    const int64_t w = std::min<int64_t>(4 / (int64_t)es, Wide(es).of(a.dim).of(a.vb).of(a.vt).of(a.gb).of(a.gt).of(a.yb).of(a.yt).at(v, es)
                                               .at(g, es).at(dy, es).at(dv, es).at(dg, es).v);
    a.nv = a.dim / w;
    const GatedShape shape = gated_shape(a.batch, p.keeps, a.nv);
    a.nchunk = shape.nchunk, a.groups = shape.groups, a.per_row = shape.per_row;
    if (shape.link) gated_clear(a, work, st);
    with_type<2, 1>(d->dtype, w, [&](auto zero, auto width) {
      using T = decltype(zero);
      constexpr int V = decltype(width)::value;
      gated_launch(shape, a, [&](const GatedArgs& a, auto link, auto span, dim3 grid) {
        hipLaunchKernelGGL(HIP_KERNEL_NAME(k_gated_grad<T, V, decltype(link)::value, decltype(span)::value>), grid,
                           dim3(shape.threads), 0, st, a, (const T*)v, (const T*)g, kept, (const T*)dy, dlast, (T*)dv, (T*)dg,
                           dy0);
      });
    });
    HIPCHECK(hipGetLastError());
  });
}

ms_status ms_gated_lowpass_step(const ms_gated_step_desc* d, const void* v, const void* g, float* state,
                                const int32_t* slots, void* y) {
  return guarded([&] {
    need(d != nullptr, "NULL descriptor");
    need(d->rows >= 0 && d->rows < ((int64_t)1 << 31) && d->n_slots >= 0 && d->n_slots < ((int64_t)1 << 31),
         "rows and n_slots must be in [0, 2^31)");
    need(d->dim >= 1 && d->dim < (1 << 24), "dim must be in [1, 2^24)");
    need_dtype(d->dtype);
    const auto stride = [&](int64_t s) {
      const int64_t r = s ? s : d->dim;
      need(r >= d->dim && r < kMaxStride, "row strides must be at least dim");
      return r;
    };
    const int64_t vs = stride(d->v_stride), gs = stride(d->g_stride), ys = stride(d->y_stride),
                  ss = stride(d->state_stride);
    if (d->rows == 0) return;
    need(v && g && y && (state || d->n_slots == 0), "NULL array");
    const size_t es = size_of(d->dtype);
    for (const void* q : {v, g, (const void*)y}) need_aligned(q, es, "v, g or y");
    for (const void* q : {(const void*)state, (const void*)slots}) need_aligned(q, 4, "state or slots");
    DeviceGuard dg(d->device);
    const int64_t w = std::min<int64_t>(
        4, Wide(es).of(d->dim).of(vs).of(gs).of(ys).of(ss).at(v, es).at(g, es).at(y, es).at(state, 4).v);
    const int32_t nv = (int32_t)(d->dim / w), tpr = threads_per_row(nv);
    with_type<4, 4>(d->dtype, w, [&](auto zero, auto width) {
      using T = decltype(zero);
      constexpr int V = decltype(width)::value;
      hipLaunchKernelGGL(HIP_KERNEL_NAME(k_gated_served<T, V>), dim3(row_blocks(d->rows, tpr)), dim3(256), 0,
                         (hipStream_t)d->stream, (const T*)v, (const T*)g, state, slots, (T*)y, d->rows, d->n_slots, nv,
                         tpr, vs, gs, ys, ss);
    });
    HIPCHECK(hipGetLastError());
  });
}

ms_status ms_orth_workspace(const ms_orth_desc* d, int32_t update, int64_t* bytes_out) {
  return guarded([&] {
    const Orth o = check_orth(d);
    need(bytes_out != nullptr, "NULL output");
    *bytes_out = orth_work(d, o, nullptr).bytes;
  });
}

ms_status ms_orthogonalise(const ms_orth_desc* d, const void* x, void* out, void* workspace, int64_t workspace_bytes) {
  return guarded([&] {
    const Orth o = check_orth(d);
    if (d->batch == 0) return;
    need(x && out, "NULL array");
    need(o.om >= (d->rows - 1) * o.orow + d->cols || d->batch <= 1, "the matrices of out must not overlap");
    const size_t es = size_of(d->dtype);
    need_aligned(x, es, "x");
    need_aligned(out, es, "out");
    OrthWork w = orth_work(d, o, workspace);
    need_workspace(workspace, workspace_bytes, w.bytes);
    DeviceGuard dg(d->device);
    const hipStream_t st = (hipStream_t)d->stream;
    OrthSrc src{x, nullptr, o.xm, o.xr, d->rows, d->cols, 0.0f, 0};
    OrthGemm g{};
    g.out = out, g.mat = o.om, g.row = o.orow, g.rows = d->rows, g.cols = d->cols;
    if (d->dtype == MS_DTYPE_BF16) orth<__bf16, false>(d, o, src, w, g, st);
    else orth<float, false>(d, o, src, w, g, st);
  });
}

ms_status ms_orthogonal_update(const ms_orth_desc* d, const ms_orth_rule* rule, float* weight, float* momentum,
                               const void* grad, void* workspace, int64_t workspace_bytes) {
  return guarded([&] {
    const Orth o = check_orth(d);
    need(rule != nullptr, "NULL rule");
    const float rate = (float)rule->rate, decay = (float)rule->momentum_decay,
                keep = (float)(1.0 - rule->rate * rule->weight_decay);
    need(std::isfinite(rate) && std::isfinite(decay) && std::isfinite(keep), "rates must be finite in 32 bits");
    if (d->batch == 0) return;
    need(weight && momentum && grad, "NULL array");
    need_aligned(weight, 4, "weight");
    need_aligned(momentum, 4, "momentum");
    need_aligned(grad, size_of(d->dtype), "grad");
    OrthWork w = orth_work(d, o, workspace);
    need_workspace(workspace, workspace_bytes, w.bytes);
    DeviceGuard dg(d->device);
    const hipStream_t st = (hipStream_t)d->stream;
    OrthSrc src{grad, momentum, o.xm, o.xr, d->rows, d->cols, decay, rule->nesterov};
    OrthGemm g{};
    g.out = weight, g.mat = d->rows * d->cols, g.row = d->cols, g.rows = d->rows, g.cols = d->cols;
    g.keep = keep, g.rate = rate;
    if (d->dtype == MS_DTYPE_BF16) orth<__bf16, true>(d, o, src, w, g, st);
    else orth<float, true>(d, o, src, w, g, st);
  });
}

}  // extern "C"
