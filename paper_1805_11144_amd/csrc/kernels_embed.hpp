// Table lookup and its gradient by sorted tokens.
//
// The lookup moves rows: out[i] = scale * table[token[i]].  Memory bounds it; a
// group of threads reads and writes rows in words of up to 16 bytes, four rows
// at a time.  131072 rows of 1024 bf16 from a table of 32768: 55 us, 6.1 TB/s of
// the 0.34 GB that have to move.
//
// The gradient adds the rows of equal tokens.  Atomic additions would make
// their order, and so the last bits, depend on timing; here (token, position)
// pairs are brought into token order by a stable radix sort (least significant
// digit first, 8 to 10 bits a pass), so each table row is the sum of a run of
// positions in ascending order.  A run of more than 64 is summed in pieces that
// are added in their order, since a token's frequency falls with its rank and
// the first ones fill whole batches: with one group of threads to every row
// 262144 rows took 12.8 ms, in pieces 0.29.
// Measured, 262144 rows of 1024 bf16 into 65536 x 1024 float32 (0.81 GB): sort
// 37 us, pieces (0.29 GB) 60, rows (0.52 GB) 95: 5.2 TB/s of the sums' bytes.
// 12800 x 784 float32 into 10007 rows (71 MB): sort 19 us, pieces and row
// beginnings 9, rows 17: launches that each wait for the one before.
#pragma once

#include "kernels_words.hpp"

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

// `tpr` (a power of two, at most 256) threads per row, nv vectors of V values
// per row; a group of threads has R rows in flight.
template <class T, class I, int V, int R>
__global__ void __launch_bounds__(256) k_embed(const I* tokens, const T* table, T* out, int64_t n, int64_t vocab,
                                               int32_t nv, int32_t tpr, int64_t ts, int64_t os, float scale) {
  const int32_t groups = 256 / tpr;
  const int64_t step = (int64_t)gridDim.x * groups * R;
  for (int64_t i = ((int64_t)blockIdx.x * R * groups) + threadIdx.x / tpr; i < n; i += step) {
    uint32_t key[R];
#pragma unroll
    for (int r = 0; r < R; ++r) key[r] = token_key(tokens, min(i + r * groups, n - 1), vocab);
    for (int32_t c = threadIdx.x % tpr; c < nv; c += tpr) {
      Words<T, V> w[R];
#pragma unroll
      for (int r = 0; r < R; ++r)
        w[r] = *(const Words<T, V>*)(table + (int64_t)(key[r] < vocab ? key[r] : 0) * ts + (int64_t)c * V);
#pragma unroll
      for (int r = 0; r < R; ++r) {
#pragma unroll
        for (int e = 0; e < V; ++e) w[r].v[e] = key[r] < vocab ? (T)(scale * as_f32(w[r].v[e])) : (T)0.0f;
        if (i + r * groups < n) put_once(out + (i + r * groups) * os + (int64_t)c * V, w[r]);
      }
    }
  }
}

// ------------------------------------------------------------------ sort
constexpr int kSortBlock = 64;  // tiles whose counts k_sort_prefix adds up together

// A digit has BITS bits, 8 to 10, and counters come in rows of 256 PER = 2^BITS.
// A tile is 256 N pairs.

// How many of a tile's keys have each digit at `shift`, to
// counts[tile][digit].  The first pass reads the tokens (keys == NULL).
template <class I, int BITS, int N>
__global__ void __launch_bounds__(256) k_sort_count(const I* tokens, const uint32_t* keys, int64_t n, int64_t vocab,
                                                    int shift, uint32_t* counts) {
  constexpr int PER = 1 << (BITS - 8);
  __shared__ uint32_t hist[256 * PER];
#pragma unroll
  for (int q = 0; q < PER; ++q) hist[q * 256 + threadIdx.x] = 0;
  __syncthreads();
  const int64_t base = (int64_t)blockIdx.x * 256 * N;
  uint32_t key[N];
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const int64_t i = base + k * 256 + threadIdx.x;
    key[k] = i < n ? (keys ? keys[i] : token_key(tokens, i, vocab)) : 0;
  }
#pragma unroll
  for (int k = 0; k < N; ++k)
    if (base + k * 256 + threadIdx.x < n) atomicAdd(&hist[(key[k] >> shift) & ((1u << BITS) - 1)], 1u);
  __syncthreads();
#pragma unroll
  for (int q = 0; q < PER; ++q)
    counts[((int64_t)blockIdx.x * PER + q) * 256 + threadIdx.x] = hist[q * 256 + threadIdx.x];
}

// Turns n rows of a column, `digits` apart, into the sums of the rows before;
// returns the sum of all.
__device__ __forceinline__ uint32_t column_prefix(uint32_t* c, int32_t n, int32_t digits) {
  constexpr int A = 32;   // rows in flight
  uint32_t sum = 0;
  for (int32_t t = 0; t < n; t += A) {
    uint32_t x[A];
#pragma unroll
    for (int u = 0; u < A; ++u) x[u] = t + u < n ? c[(int64_t)(t + u) * digits] : 0;
#pragma unroll
    for (int u = 0; u < A; ++u) {
      if (t + u < n) c[(int64_t)(t + u) * digits] = sum;
      sum += x[u];
    }
  }
  return sum;
}

// Counts of many tiles as sums over the tiles before, so that a tile reads its
// own and its block's and not all tiles' counts.  counts[tile][digit] becomes the
// digit's pairs in the earlier tiles of its block of kSortBlock, and
// block[b][digit] those of block b.  One thread to a column of a block.
__global__ void __launch_bounds__(256) k_sort_prefix(uint32_t* counts, uint32_t* block, int32_t tiles, int32_t digits) {
  const int64_t d = (int64_t)blockIdx.x % (digits / 256) * 256 + threadIdx.x, b = blockIdx.x / (digits / 256);
  const int32_t n = (int32_t)min((int64_t)kSortBlock, tiles - b * kSortBlock);
  block[b * digits + d] = column_prefix(counts + b * kSortBlock * digits + d, n, digits);
}

// The same over the blocks; block[blocks] ends as the digits' pairs in all.
__global__ void __launch_bounds__(256) k_sort_blocks(uint32_t* block, int32_t blocks, int32_t digits) {
  uint32_t* c = block + (int64_t)blockIdx.x * 256 + threadIdx.x;
  c[(int64_t)blocks * digits] = column_prefix(c, blocks, digits);
}

// The lanes of a wavefront that hold live keys of this lane's digit.
template <int BITS>
__device__ __forceinline__ uint64_t same_digit(uint32_t d, bool live) {
  uint64_t same = __ballot(live);
#pragma unroll
  for (int b = 0; b < BITS; ++b) {
    const uint64_t set = __ballot((d >> b) & 1);
    same &= (d >> b) & 1 ? set : ~set;
  }
  return same;
}

// Ranks a wavefront's keys, item by item, among its earlier keys of the same
// digit; count[digit] ends as their number.
template <int BITS, int N>
__device__ __forceinline__ void rank_keys(const uint32_t* key, uint32_t* rank, uint32_t* count, int64_t base, int64_t n,
                                          int shift) {
  const int lane = threadIdx.x % 64;
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const bool live = base + k * 64 + lane < n;
    const uint32_t d = (key[k] >> shift) & ((1u << BITS) - 1);
    const uint64_t same = same_digit<BITS>(d, live), lower = same & ((1ull << lane) - 1);
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
// positions [w * 64 N, (w + 1) * 64 N) in order of (item, lane).  `block`: the
// sums that k_sort_prefix and k_sort_blocks left; NULL: every tile adds up the
// counts of all.
template <class I, int BITS, int N>
__global__ void __launch_bounds__(256) k_sort_move(const I* tokens, const uint32_t* keys, const uint32_t* pos,
                                                   int64_t n, int64_t vocab, int shift, const uint32_t* counts,
                                                   const uint32_t* block, uint32_t* keys_out, uint32_t* pos_out) {
  constexpr int PER = 1 << (BITS - 8);
  __shared__ uint32_t part[4][256 * PER];   // a wavefront's pairs of each digit, then where its first one goes
  __shared__ uint32_t first[256 * PER];     // pairs of each digit in all tiles, then of smaller digits
  __shared__ uint32_t sums[4];
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  uint32_t key[N], rank[N], from[N];
  const int64_t base = (int64_t)blockIdx.x * 256 * N + wave * 64 * N;
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const int64_t i = base + k * 64 + lane;
    key[k] = i < n ? (keys ? keys[i] : token_key(tokens, i, vocab)) : 0;
    from[k] = i < n && pos ? pos[i] : (uint32_t)i;
  }
  // pairs of the thread's digits, q * 256 + tid, in all tiles and in the earlier ones
  uint32_t before[PER] = {}, total[PER] = {};
  const uint32_t* c = counts + tid;
  const uint32_t tiles = block ? 0 : gridDim.x;
  constexpr int A = 64 / PER;   // tiles in flight
  uint32_t t = 0;
  if (block) {
    const uint32_t own = blockIdx.x / kSortBlock, blocks = (gridDim.x + kSortBlock - 1) / kSortBlock;
#pragma unroll
    for (int q = 0; q < PER; ++q) {
      before[q] = c[((int64_t)blockIdx.x * PER + q) * 256] + block[((int64_t)own * PER + q) * 256 + tid];
      total[q] = block[((int64_t)blocks * PER + q) * 256 + tid];
    }
  }
  for (; t + A <= tiles; t += A) {
    uint32_t x[A][PER];
#pragma unroll
    for (int u = 0; u < A; ++u)
#pragma unroll
      for (int q = 0; q < PER; ++q) x[u][q] = c[((int64_t)(t + u) * PER + q) * 256];
#pragma unroll
    for (int u = 0; u < A; ++u)
#pragma unroll
      for (int q = 0; q < PER; ++q) {
        total[q] += x[u][q];
        before[q] += t + u < blockIdx.x ? x[u][q] : 0;
      }
  }
#pragma unroll 8
  for (; t < tiles; ++t)
#pragma unroll
    for (int q = 0; q < PER; ++q) {
      const uint32_t x = c[((int64_t)t * PER + q) * 256];
      total[q] += x;
      before[q] += t < blockIdx.x ? x : 0;
    }
#pragma unroll
  for (int q = 0; q < PER; ++q) {
    first[q * 256 + tid] = total[q];
#pragma unroll
    for (int w = 0; w < 4; ++w) part[w][q * 256 + tid] = 0;
  }
  __syncthreads();
  // pairs of smaller digits: thread tid adds up digits [tid * PER, tid * PER + PER)
  uint32_t own[PER], all = 0;
#pragma unroll
  for (int q = 0; q < PER; ++q) own[q] = first[tid * PER + q], all += own[q];
  const uint32_t incl = wave_prefix(all);
  if (lane == 63) sums[wave] = incl;
  rank_keys<BITS, N>(key, rank, part[wave], base, n, shift);
  __syncthreads();
  uint32_t lower = incl - all;
  for (int w = 0; w < wave; ++w) lower += sums[w];
#pragma unroll
  for (int q = 0; q < PER; ++q) {
    first[tid * PER + q] = lower;
    lower += own[q];
  }
  __syncthreads();
#pragma unroll
  for (int q = 0; q < PER; ++q) {
    const int d = q * 256 + tid;
    uint32_t at = first[d] + before[q];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const uint32_t x = part[w][d];
      part[w][d] = at;
      at += x;
    }
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < N; ++k)
    if (base + k * 64 + lane < n) {
      const uint32_t at = part[wave][(key[k] >> shift) & ((1u << BITS) - 1)] + rank[k];
      keys_out[at] = key[k];
      pos_out[at] = from[k];
    }
}

// The whole sort in one workgroup, for at most 1024 N tokens: pairs in LDS
// between the passes, digits of 8 bits.
template <class I, int N>
__global__ void __launch_bounds__(1024) k_sort_small(const I* tokens, int32_t n, int64_t vocab, int passes,
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
    const int shift = p * 8;
    for (int d = lane; d < 256; d += 64) part[wave][d] = 0;
    __syncthreads();
    rank_keys<8, N>(key, rank, part[wave], base, n, shift);
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
        const uint32_t at = part[wave][(key[k] >> shift) & 255] + rank[k];
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

// Columns first, first + tpr.. of the sum of the rows at pos[s0] .. pos[s1 - 1]
// (at most kRun of them), handed to put(c, sums).  FULL: whole wavefronts work
// on one row, so its positions are fetched once, one to a lane, and a row's
// address is uniform; eight rows are in flight at a time.
template <class T, int V, bool FULL, class F>
__device__ __forceinline__ void sum_rows(const uint32_t* pos, uint32_t s0, uint32_t s1, const T* rows, int64_t rs,
                                         int32_t first, int32_t nv, int32_t tpr, F&& put) {
  constexpr int A = 8;
  const int n = (int)(s1 - s0);
  uint32_t mine = 0;
  if (FULL && (int)threadIdx.x % 64 < n) mine = pos[s0 + threadIdx.x % 64];
  const auto row = [&](int s) {
    const uint32_t p = FULL ? (uint32_t)__builtin_amdgcn_readlane((int)mine, s) : pos[s0 + s];
    return rows + (int64_t)p * rs;
  };
  for (int32_t c = first; c < nv; c += tpr) {
    float acc[V] = {};
    int s = 0;
    for (; s + A <= n; s += A) {
      Words<T, V> w[A];
#pragma unroll
      for (int q = 0; q < A; ++q) w[q] = take_once<T, V>(row(s + q) + (int64_t)c * V);
#pragma unroll
      for (int q = 0; q < A; ++q)
#pragma unroll
        for (int e = 0; e < V; ++e) acc[e] += as_f32(w[q].v[e]);
    }
    if (s + 4 <= n) {
      Words<T, V> w[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) w[q] = take_once<T, V>(row(s + q) + (int64_t)c * V);
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int e = 0; e < V; ++e) acc[e] += as_f32(w[q].v[e]);
      s += 4;
    }
    for (; s < n; ++s) {
      const Words<T, V> w = *(const Words<T, V>*)(row(s) + (int64_t)c * V);
#pragma unroll
      for (int e = 0; e < V; ++e) acc[e] += as_f32(w.v[e]);
    }
    put(c, acc);
  }
}

// The first `searches` workgroups find start[v], v in [0, vocab]: the first
// sorted pair whose token is at least v.  The others sum the pieces of long
// runs, `tpc` threads (a multiple of 64) to a chunk.
template <class T, int V>
__global__ void __launch_bounds__(256) k_embed_pieces(const uint32_t* keys, const uint32_t* pos, int64_t n,
                                                      int64_t vocab, const T* rows, int32_t nv, int32_t tpc, int64_t rs,
                                                      uint32_t searches, uint32_t* start, float* part) {
  if (blockIdx.x < searches) {
    const int64_t step = (int64_t)searches * 256;
    for (int64_t v = (int64_t)blockIdx.x * 256 + threadIdx.x; v <= vocab; v += step) {
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
  const int64_t chunk = __builtin_amdgcn_readfirstlane((blockIdx.x - searches) * (256 / tpc) + threadIdx.x / tpc);
  if (chunk * kRun >= n) return;
  const uint32_t c0 = (uint32_t)chunk * kRun, c1 = (uint32_t)min((int64_t)c0 + kRun, n);
  const int lane = threadIdx.x % 64;
  // the keys of this chunk and its neighbours: enough to tell whether its first and last runs are long
  uint32_t near[3];
#pragma unroll
  for (int w = 0; w < 3; ++w) {
    const int64_t i = (int64_t)c0 + (w - 1) * kRun + lane;
    near[w] = i >= 0 && i < n ? keys[i] : ~0u;   // no key
  }
  const uint32_t k0 = __builtin_amdgcn_readfirstlane(near[1]);
  const uint32_t k1 = __builtin_amdgcn_readlane(near[1], (int)(c1 - c0) - 1);
#pragma unroll
  for (int side = 0; side < 2; ++side) {
    if (side == 1 && k1 == k0) return;
    const uint32_t k = side ? k1 : k0;
    if (k == (uint32_t)vocab) continue;   // padding
    const int here = __popcll(__ballot(near[1] == k));
    if (here + __popcll(__ballot(near[0] == k)) + __popcll(__ballot(near[2] == k)) <= kRun) continue;
    const uint32_t s0 = side ? c1 - here : c0;
    float* o = part + (chunk * 2 + side) * nv * V;
    sum_rows<T, V, true>(pos, s0, s0 + here, rows, rs, threadIdx.x % tpc, nv, tpc, [&](int32_t c, const float* acc) {
      Words<float, V> x;
#pragma unroll
      for (int e = 0; e < V; ++e) x.v[e] = acc[e];
      *(Words<float, V>*)(o + (int64_t)c * V) = x;
    });
  }
}

// dtable[v] = scale * sum of the rows at pos[start[v]] .. pos[start[v + 1] - 1].
// FULL: tpr is a multiple of 64.
template <class T, class D, int V, bool FULL>
__global__ void __launch_bounds__(256) k_embed_sum(const uint32_t* pos, const uint32_t* start, const T* rows,
                                                   const float* part, D* dtable, int64_t vocab, int32_t nv, int32_t tpr,
                                                   int64_t rs, int64_t gs, float scale, int accumulate) {
  const int32_t rpb = 256 / tpr;
  for (int64_t v = (int64_t)blockIdx.x * rpb + threadIdx.x / tpr; v < vocab; v += (int64_t)gridDim.x * rpb) {
    uint32_t s0 = start[v], s1 = start[v + 1];
    if (FULL) s0 = __builtin_amdgcn_readfirstlane(s0), s1 = __builtin_amdgcn_readfirstlane(s1);
    if (accumulate && s0 == s1) continue;
    const auto put = [&](int32_t c, const float* acc) {
      D* dst = dtable + v * gs + (int64_t)c * V;
      Words<D, V> o;
      if (accumulate) o = *(const Words<D, V>*)dst;
#pragma unroll
      for (int e = 0; e < V; ++e) o.v[e] = (D)(scale * acc[e] + (accumulate ? as_f32(o.v[e]) : 0.0f));
      put_once(dst, o);
    };
    if (s1 - s0 <= (uint32_t)kRun) {
      sum_rows<T, V, FULL>(pos, s0, s1, rows, rs, threadIdx.x % tpr, nv, tpr, put);
      continue;
    }
    // the pieces in order: its first chunk holds the run's beginning, as its first pair or up to its last
    const uint32_t b0 = s0 / kRun, b1 = (s1 - 1) / kRun;
    for (int32_t c = threadIdx.x % tpr; c < nv; c += tpr) {
      const float* q = part + ((int64_t)b0 * 2 + (s0 % kRun != 0)) * nv * V + (int64_t)c * V;
      Words<float, V> acc = *(const Words<float, V>*)q;
#pragma unroll 8
      for (uint32_t b = b0 + 1; b <= b1; ++b) {
        const Words<float, V> x = *(const Words<float, V>*)(part + (int64_t)b * 2 * nv * V + (int64_t)c * V);
#pragma unroll
        for (int e = 0; e < V; ++e) acc.v[e] += x.v[e];
      }
      put(c, acc.v);
    }
  }
}
