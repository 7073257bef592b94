// Table lookup and its gradient by sorted tokens.
//
// The lookup moves rows: out[i] = scale * table[token[i]].  It is bound by
// memory; a row is read and written in words of up to 16 bytes per lane.
//
// The gradient adds the rows of equal tokens.  Atomic additions would make
// their order, and so the last bits, depend on timing; here (token, position)
// pairs are brought into token order by a stable radix sort (least significant
// digit first, 8 bits a pass), so each table row is the sum of a run of
// positions in ascending order.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

template <class T, int V>
struct alignas(sizeof(T) * V) Words {
  T v[V];
};

template <class T>
__device__ __forceinline__ float as_f32(T x) {
  return (float)x;
}

// LDS accesses of one wavefront stay in the order written here.
__device__ __forceinline__ void wave_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Token i as a key: its row, or `vocab` for padding.
template <class I>
__device__ __forceinline__ uint32_t token_key(const I* tokens, int64_t i, int64_t vocab) {
  const I t = tokens[i];
  return t >= 0 && (int64_t)t < vocab ? (uint32_t)t : (uint32_t)vocab;
}

// `tpr` (a power of two, at most 256) threads per row, 256 / tpr rows per
// workgroup; nv vectors of V values per row.
template <class T, class I, int V>
__global__ void __launch_bounds__(256) k_embed(const I* tokens, const T* table, T* out, int64_t n, int64_t vocab,
                                               int32_t nv, int32_t tpr, int64_t ts, int64_t os, float scale) {
  const int32_t rows = 256 / tpr;
  for (int64_t i = (int64_t)blockIdx.x * rows + threadIdx.x / tpr; i < n; i += (int64_t)gridDim.x * rows) {
    const uint32_t key = token_key(tokens, i, vocab);
    const bool pad = key == (uint32_t)vocab;
    const T* src = table + (int64_t)(pad ? 0 : key) * ts;
    T* dst = out + i * os;
    for (int32_t c = threadIdx.x % tpr; c < nv; c += tpr) {
      Words<T, V> w;
      if (!pad) w = *(const Words<T, V>*)(src + (int64_t)c * V);
#pragma unroll
      for (int e = 0; e < V; ++e) w.v[e] = pad ? (T)0.0f : (T)(scale * as_f32(w.v[e]));
      *(Words<T, V>*)(dst + (int64_t)c * V) = w;
    }
  }
}

// ------------------------------------------------------------------ sort
constexpr int kSortItems = 16;                     // per thread
constexpr int kSortTile = 256 * kSortItems;        // per workgroup
constexpr int kSortBits = 10;                      // of a digit, at most

// How many of a tile's keys have each digit (`bits` bits at `shift`), to
// counts[tile][digit].  The first pass reads the tokens (keys == NULL).
template <class I>
__global__ void __launch_bounds__(256) k_sort_count(const I* tokens, const uint32_t* keys, int64_t n, int64_t vocab,
                                                    int shift, int bits, uint32_t* counts) {
  __shared__ uint32_t hist[1 << kSortBits];
  const int digits = 1 << bits;
  for (int d = threadIdx.x; d < digits; d += 256) hist[d] = 0;
  __syncthreads();
  const int64_t base = (int64_t)blockIdx.x * kSortTile;
#pragma unroll
  for (int k = 0; k < kSortItems; ++k) {
    const int64_t i = base + k * 256 + threadIdx.x;
    if (i < n) {
      const uint32_t key = keys ? keys[i] : token_key(tokens, i, vocab);
      atomicAdd(&hist[(key >> shift) & (digits - 1)], 1u);
    }
  }
  __syncthreads();
  for (int d = threadIdx.x; d < digits; d += 256) counts[(int64_t)blockIdx.x * digits + d] = hist[d];
}

// The lanes of a wavefront that hold live keys of this lane's digit.
__device__ __forceinline__ uint64_t same_digit(uint32_t d, int bits, bool live) {
  uint64_t same = __ballot(live);
  for (int b = 0; b < bits; ++b) {
    const uint64_t set = __ballot((d >> b) & 1);
    same &= (d >> b) & 1 ? set : ~set;
  }
  return same;
}

// Ranks a wavefront's keys, item by item, among its earlier keys of the same
// digit; count[digit] ends as their number.
template <int N>
__device__ __forceinline__ void rank_keys(const uint32_t* key, uint32_t* rank, uint32_t* count, int64_t base, int64_t n,
                                          int shift, int bits) {
  const int lane = threadIdx.x % 64;
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const bool live = base + k * 64 + lane < n;
    const uint32_t d = (key[k] >> shift) & ((1u << bits) - 1);
    const uint64_t same = same_digit(d, bits, live), lower = same & ((1ull << lane) - 1);
    const uint32_t seen = count[d];   // every lane reads before the digit's first lane adds
    wave_order();
    rank[k] = seen + __popcll(lower);
    if (live && lower == 0) count[d] = seen + __popcll(same);
    wave_order();
  }
}

// Sum of x over the lanes up to this one.
__device__ __forceinline__ uint32_t wave_prefix(uint32_t x) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t y = __shfl_up(x, o, 64);
    if ((int)threadIdx.x % 64 >= o) x += y;
  }
  return x;
}

// Moves each pair to its place: behind the pairs of smaller digits, of earlier
// tiles and of earlier positions in the tile.  Wavefront w holds the tile's
// positions [w * 1024, (w + 1) * 1024) in order of (item, lane).
template <class I>
__global__ void __launch_bounds__(256) k_sort_move(const I* tokens, const uint32_t* keys, const uint32_t* pos,
                                                   int64_t n, int64_t vocab, int shift, int bits,
                                                   const uint32_t* counts, uint32_t* keys_out, uint32_t* pos_out) {
  constexpr int PER = (1 << kSortBits) / 256;   // digits of a thread: [tid * per, tid * per + per)
  __shared__ uint32_t part[4][1 << kSortBits];  // a wavefront's pairs of each digit, then where its first one goes
  __shared__ uint32_t sums[4];
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64, digits = 1 << bits;
  const int per = max(1, digits / 256);
  for (int d = tid; d < digits; d += 256)
#pragma unroll
    for (int w = 0; w < 4; ++w) part[w][d] = 0;
  uint32_t key[kSortItems], rank[kSortItems];
  const int64_t base = (int64_t)blockIdx.x * kSortTile + wave * 64 * kSortItems;
#pragma unroll
  for (int k = 0; k < kSortItems; ++k) {
    const int64_t i = base + k * 64 + lane;
    key[k] = i < n ? (keys ? keys[i] : token_key(tokens, i, vocab)) : 0;
  }
  // pairs of the thread's digits in all tiles, and in the earlier ones
  uint32_t before[PER] = {}, total[PER] = {}, all = 0;
  const bool has = tid * per < digits;
  if (has) {
#pragma unroll 8
    for (uint32_t t = 0; t < gridDim.x; ++t)
#pragma unroll
      for (int q = 0; q < PER; ++q)
        if (q < per) {
          const uint32_t c = counts[(int64_t)t * digits + tid * per + q];
          total[q] += c;
          before[q] += t < blockIdx.x ? c : 0;
        }
#pragma unroll
    for (int q = 0; q < PER; ++q) all += total[q];
  }
  const uint32_t incl = wave_prefix(all);
  if (lane == 63) sums[wave] = incl;
  __syncthreads();
  uint32_t lower = incl - all;
  for (int w = 0; w < wave; ++w) lower += sums[w];
  rank_keys<kSortItems>(key, rank, part[wave], base, n, shift, bits);
  __syncthreads();
  if (has) {
#pragma unroll
    for (int q = 0; q < PER; ++q)
      if (q < per) {
        uint32_t at = lower + before[q];
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const uint32_t c = part[w][tid * per + q];
          part[w][tid * per + q] = at;
          at += c;
        }
        lower += total[q];
      }
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kSortItems; ++k) {
    const int64_t i = base + k * 64 + lane;
    if (i < n) {
      const uint32_t at = part[wave][(key[k] >> shift) & (digits - 1)] + rank[k];
      keys_out[at] = key[k];
      pos_out[at] = pos ? pos[i] : (uint32_t)i;
    }
  }
}

// The whole sort in one workgroup, for at most 1024 N tokens: pairs in LDS
// between the passes, digits of at most 8 bits.
template <class I, int N>
__global__ void __launch_bounds__(1024) k_sort_small(const I* tokens, int32_t n, int64_t vocab, int passes, int bits,
                                                     uint32_t* keys_out, uint32_t* pos_out) {
  extern __shared__ uint32_t sort_lds[];
  uint32_t* keys = sort_lds;                                  // [1024 N]
  uint16_t* pos = (uint16_t*)(keys + 1024 * N);               // [1024 N]
  uint32_t(*part)[256] = (uint32_t(*)[256])(pos + 1024 * N);  // [16][256]
  uint32_t* sums = (uint32_t*)(part + 16);                    // [4]
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64, base = wave * 64 * N;
  uint32_t key[N], rank[N];
  uint16_t from[N];
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const int i = base + k * 64 + lane;
    key[k] = i < n ? token_key(tokens, i, vocab) : 0;
    from[k] = (uint16_t)i;
  }
  for (int p = 0; p < passes; ++p) {
    const int shift = p * bits;
    for (int d = lane; d < 256; d += 64) part[wave][d] = 0;
    __syncthreads();
    rank_keys<N>(key, rank, part[wave], base, n, shift, bits);
    __syncthreads();
    uint32_t all = 0, incl = 0;
    if (tid < 256) {
#pragma unroll
      for (int w = 0; w < 16; ++w) {
        const uint32_t c = part[w][tid];
        part[w][tid] = all;
        all += c;
      }
      incl = wave_prefix(all);
      if (lane == 63) sums[wave] = incl;
    }
    __syncthreads();
    if (tid < 256) {
      uint32_t lower = incl - all;
      for (int w = 0; w < wave; ++w) lower += sums[w];
#pragma unroll
      for (int w = 0; w < 16; ++w) part[w][tid] += lower;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (base + k * 64 + lane < n) {
        const uint32_t at = part[wave][(key[k] >> shift) & ((1u << bits) - 1)] + rank[k];
        keys[at] = key[k];
        pos[at] = from[k];
      }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int i = base + k * 64 + lane;
      if (i < n) key[k] = keys[i], from[k] = pos[i];
    }
  }
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const int i = base + k * 64 + lane;
    if (i < n) keys_out[i] = key[k], pos_out[i] = from[k];
  }
}

// ------------------------------------------------------------------- sums
// Runs of more than kRun positions are summed in pieces, so that a token that
// fills the batch does not wait for one workgroup: the sorted pairs are cut
// into chunks of kRun, a chunk holds pieces of at most two such runs (those of
// its first and of its last pair; a run between them would be shorter), and
// leaves their sums in part[chunk][2][dim].
constexpr int kRun = 64;

// Columns c, c + tpr.. of the sum of rows pos[s0] .. pos[s1 - 1], handed to put(c, sums).
template <class T, int V, class F>
__device__ __forceinline__ void sum_rows(const uint32_t* pos, uint32_t s0, uint32_t s1, const T* rows, int64_t rs,
                                         int32_t first, int32_t nv, int32_t tpr, F&& put) {
  for (int32_t c = first; c < nv; c += tpr) {
    float acc[V] = {};
    uint32_t s = s0;
    for (; s + 4 <= s1; s += 4) {
      Words<T, V> w[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) w[q] = *(const Words<T, V>*)(rows + (int64_t)pos[s + q] * rs + (int64_t)c * V);
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int e = 0; e < V; ++e) acc[e] += as_f32(w[q].v[e]);
    }
    for (; s < s1; ++s) {
      const Words<T, V> w = *(const Words<T, V>*)(rows + (int64_t)pos[s] * rs + (int64_t)c * V);
#pragma unroll
      for (int e = 0; e < V; ++e) acc[e] += as_f32(w.v[e]);
    }
    put(c, acc);
  }
}

// Workgroups [0, nchunk) sum the pieces of long runs; the others find
// start[v], v in [0, vocab]: the first sorted pair whose token is at least v.
template <class T, int V>
__global__ void __launch_bounds__(256) k_embed_pieces(const uint32_t* keys, const uint32_t* pos, int64_t n,
                                                      int64_t vocab, const T* rows, int32_t nv, int64_t rs,
                                                      uint32_t nchunk, uint32_t* start, float* part) {
  if (blockIdx.x >= nchunk) {
    const int64_t step = (int64_t)(gridDim.x - nchunk) * 256;
    for (int64_t v = (int64_t)(blockIdx.x - nchunk) * 256 + threadIdx.x; v <= vocab; v += step) {
      uint32_t lo = 0, hi = (uint32_t)n;
      while (lo < hi) {
        const uint32_t mid = lo + (hi - lo) / 2;
        if (keys[mid] < (uint32_t)v) lo = mid + 1;
        else hi = mid;
      }
      start[v] = lo;
    }
    return;
  }
  const uint32_t c0 = blockIdx.x * kRun, c1 = (uint32_t)min((int64_t)c0 + kRun, n);
  const int lane = threadIdx.x % 64;
  const uint32_t k0 = keys[c0], k1 = keys[c1 - 1];
#pragma unroll
  for (int side = 0; side < 2; ++side) {
    if (side == 1 && k1 == k0) return;
    const uint32_t k = side ? k1 : k0;
    if (k == (uint32_t)vocab) continue;   // padding
    // the run's pairs in this chunk and its neighbours: enough to tell whether it is long
    int seen = 0, here = 0;
#pragma unroll
    for (int w = -1; w <= 1; ++w) {
      const int64_t i = (int64_t)c0 + w * kRun + lane;
      const int same = __popcll(__ballot(i >= 0 && i < n && keys[i < 0 ? 0 : i < n ? i : n - 1] == k));
      seen += same;
      if (w == 0) here = same;
    }
    if (seen <= kRun) continue;
    const uint32_t s0 = side ? c1 - here : c0;
    float* o = part + ((int64_t)blockIdx.x * 2 + side) * nv * V;
    sum_rows<T, V>(pos, s0, s0 + here, rows, rs, threadIdx.x, nv, 256, [&](int32_t c, const float* acc) {
#pragma unroll
      for (int e = 0; e < V; ++e) o[(int64_t)c * V + e] = acc[e];
    });
  }
}

// dtable[v] = scale * sum of the rows at pos[start[v]] .. pos[start[v + 1] - 1].
template <class T, class D, int V>
__global__ void __launch_bounds__(256) k_embed_sum(const uint32_t* pos, const uint32_t* start, const T* rows,
                                                   const float* part, D* dtable, int64_t vocab, int32_t nv, int32_t tpr,
                                                   int64_t rs, int64_t gs, float scale, int accumulate) {
  const int32_t rpb = 256 / tpr;
  for (int64_t v = (int64_t)blockIdx.x * rpb + threadIdx.x / tpr; v < vocab; v += (int64_t)gridDim.x * rpb) {
    const uint32_t s0 = start[v], s1 = start[v + 1];
    if (accumulate && s0 == s1) continue;
    const auto put = [&](int32_t c, const float* acc) {
      D* dst = dtable + v * gs + (int64_t)c * V;
      Words<D, V> o;
      if (accumulate) o = *(const Words<D, V>*)dst;
#pragma unroll
      for (int e = 0; e < V; ++e) o.v[e] = (D)(scale * acc[e] + (accumulate ? as_f32(o.v[e]) : 0.0f));
      *(Words<D, V>*)dst = o;
    };
    if (s1 - s0 <= (uint32_t)kRun) {
      sum_rows<T, V>(pos, s0, s1, rows, rs, threadIdx.x % tpr, nv, tpr, put);
      continue;
    }
    // the pieces in order: its first chunk holds the run's beginning, as its first pair or up to its last
    const uint32_t b0 = s0 / kRun, b1 = (s1 - 1) / kRun;
    for (int32_t c = threadIdx.x % tpr; c < nv; c += tpr) {
      float acc[V];
      const float* q = part + ((int64_t)b0 * 2 + (s0 % kRun != 0)) * nv * V + (int64_t)c * V;
#pragma unroll
      for (int e = 0; e < V; ++e) acc[e] = q[e];
#pragma unroll 4
      for (uint32_t b = b0 + 1; b <= b1; ++b) {
        q = part + (int64_t)b * 2 * nv * V + (int64_t)c * V;
#pragma unroll
        for (int e = 0; e < V; ++e) acc[e] += q[e];
      }
      put(c, acc);
    }
  }
}
