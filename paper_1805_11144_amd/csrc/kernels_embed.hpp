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

// counts[tile][digit]: how many of the tile's keys have the digit at `shift`.
// The first pass reads the tokens (keys == NULL).
template <class I>
__global__ void __launch_bounds__(256) k_sort_count(const I* tokens, const uint32_t* keys, int64_t n, int64_t vocab,
                                                    int shift, uint32_t* counts) {
  __shared__ uint32_t hist[256];
  hist[threadIdx.x] = 0;
  __syncthreads();
  const int64_t base = (int64_t)blockIdx.x * kSortTile;
#pragma unroll 4
  for (int k = 0; k < kSortItems; ++k) {
    const int64_t i = base + k * 256 + threadIdx.x;
    if (i < n) {
      const uint32_t key = keys ? keys[i] : token_key(tokens, i, vocab);
      atomicAdd(&hist[(key >> shift) & 255], 1u);
    }
  }
  __syncthreads();
  counts[(int64_t)blockIdx.x * 256 + threadIdx.x] = hist[threadIdx.x];
}

// Moves each pair to its place: behind the pairs of smaller digits, of earlier
// tiles and of earlier positions in the tile.  Wavefront w holds the tile's
// positions [w * 1024, (w + 1) * 1024) in order of (item, lane), and ranks the
// lanes of an item by ballots over the digit's bits.
template <class I>
__global__ void __launch_bounds__(256) k_sort_move(const I* tokens, const uint32_t* keys, const uint32_t* pos,
                                                   int64_t n, int64_t vocab, int shift, const uint32_t* counts,
                                                   uint32_t* keys_out, uint32_t* pos_out) {
  __shared__ uint32_t part[4][256];   // pairs of each digit in a wavefront, then those before it
  __shared__ uint32_t first[256];     // where the tile's first pair of each digit goes
  __shared__ uint32_t sums[4];
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  {
    // digit `tid`: pairs in all tiles, and in the earlier ones
    uint32_t before = 0, total = 0;
    for (uint32_t t = 0; t < gridDim.x; ++t) {
      const uint32_t c = counts[(int64_t)t * 256 + tid];
      total += c;
      before += t < blockIdx.x ? c : 0;
    }
    uint32_t incl = total;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t x = __shfl_up(incl, o, 64);
      if (lane >= o) incl += x;
    }
    if (lane == 63) sums[wave] = incl;
#pragma unroll
    for (int w = 0; w < 4; ++w) part[w][tid] = 0;
    __syncthreads();
    uint32_t lower = incl - total;
    for (int w = 0; w < wave; ++w) lower += sums[w];
    first[tid] = lower + before;
  }
  __syncthreads();
  uint32_t key[kSortItems], rank[kSortItems];
  const int64_t base = (int64_t)blockIdx.x * kSortTile + wave * 64 * kSortItems;
#pragma unroll
  for (int k = 0; k < kSortItems; ++k) {
    const int64_t i = base + k * 64 + lane;
    key[k] = i < n ? (keys ? keys[i] : token_key(tokens, i, vocab)) : 0;
  }
#pragma unroll
  for (int k = 0; k < kSortItems; ++k) {
    const bool live = base + k * 64 + lane < n;
    const uint32_t d = (key[k] >> shift) & 255;
    uint64_t same = __ballot(live);
#pragma unroll
    for (int b = 0; b < 8; ++b) {
      const uint64_t set = __ballot((d >> b) & 1);
      same &= (d >> b) & 1 ? set : ~set;
    }
    const uint64_t lower = same & ((1ull << lane) - 1);
    // a wavefront reads its own counters before its first lane of the digit adds to them
    const uint32_t seen = part[wave][d];
    wave_order();
    rank[k] = seen + __popcll(lower);
    if (live && lower == 0) part[wave][d] = seen + __popcll(same);
    wave_order();
  }
  __syncthreads();
  {
    uint32_t sum = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const uint32_t c = part[w][tid];
      part[w][tid] = sum;
      sum += c;
    }
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kSortItems; ++k) {
    const int64_t i = base + k * 64 + lane;
    if (i < n) {
      const uint32_t d = (key[k] >> shift) & 255;
      const uint32_t at = first[d] + part[wave][d] + rank[k];
      keys_out[at] = key[k];
      pos_out[at] = pos ? pos[i] : (uint32_t)i;
    }
  }
}

// start[v], v in [0, vocab]: the first sorted pair whose token is at least v.
__global__ void __launch_bounds__(256) k_sort_starts(const uint32_t* keys, int64_t n, int64_t vocab, uint32_t* start) {
  for (int64_t v = (int64_t)blockIdx.x * 256 + threadIdx.x; v <= vocab; v += (int64_t)gridDim.x * 256) {
    uint32_t lo = 0, hi = (uint32_t)n;
    while (lo < hi) {
      const uint32_t mid = lo + (hi - lo) / 2;
      if (keys[mid] < (uint32_t)v) lo = mid + 1;
      else hi = mid;
    }
    start[v] = lo;
  }
}

// dtable[v] = scale * sum of the rows at pos[start[v]] .. pos[start[v + 1] - 1].
template <class T, class D, int V>
__global__ void __launch_bounds__(256) k_embed_sum(const uint32_t* pos, const uint32_t* start, const T* rows, D* dtable,
                                                   int64_t vocab, int32_t nv, int32_t tpr, int64_t rs, int64_t gs,
                                                   float scale, int accumulate) {
  const int32_t rpb = 256 / tpr;
  for (int64_t v = (int64_t)blockIdx.x * rpb + threadIdx.x / tpr; v < vocab; v += (int64_t)gridDim.x * rpb) {
    const uint32_t s0 = start[v], s1 = start[v + 1];
    if (accumulate && s0 == s1) continue;
    for (int32_t c = threadIdx.x % tpr; c < nv; c += tpr) {
      float acc[V] = {};
      for (uint32_t s = s0; s < s1; ++s) {
        const Words<T, V> w = *(const Words<T, V>*)(rows + (int64_t)pos[s] * rs + (int64_t)c * V);
#pragma unroll
        for (int e = 0; e < V; ++e) acc[e] += as_f32(w.v[e]);
      }
      D* dst = dtable + v * gs + (int64_t)c * V;
      Words<D, V> o;
      if (accumulate) o = *(const Words<D, V>*)dst;
#pragma unroll
      for (int e = 0; e < V; ++e) o.v[e] = (D)(scale * acc[e] + (accumulate ? as_f32(o.v[e]) : 0.0f));
      *(Words<D, V>*)dst = o;
    }
  }
}
