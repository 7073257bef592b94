// Which variant of a kernel a call takes: rules on sizes and types, without HIP.
#pragma once

#include <algorithm>
#include <cmath>
#include <cstdint>

namespace ms {

// ------------------------------------------------------------------ tables
constexpr int kSortBits = 10;   // of a digit, at most

// Bits of a digit of the sort: the fewest passes over keys in [0, vocab], and
// digits as short as they allow, eight bits at least.
inline int sort_bits(int64_t vocab, int* key_bits) {
  int bits = 1;
  while (vocab >> bits) ++bits;
  const int passes = (bits + kSortBits - 1) / kSortBits;
  if (key_bits) *key_bits = bits;
  return std::max((bits + passes - 1) / passes, 8);
}

// Items of a thread in the sort in one workgroup, and 0 where many share it: one
// launch in place of four or more, 1000 tokens 20 us in all, and 29; 4096 tokens
// 35, and 41.
inline int sort_small_items(int64_t n) { return n <= 1024 ? 1 : n <= 4096 ? 4 : 0; }

// Items of a thread in the sort: a tile holds 256 times as many pairs.  Up to
// kSortAll tiles each adds up the counts of all, so tiles grow where they become
// many.  Gradients in us with 4, 8 and 16 items: 40000 tokens 50, 56, 64; 100000
// 59, 62, 73; 262144 101, 98, 104; 524288 138, 112, 111; 1048576 290, 200, 176.
inline int sort_items(int64_t n) { return n <= (1 << 17) ? 4 : n <= (1 << 19) ? 8 : 16; }

// With more tiles two launches a digit add up their counts: 131072 tokens in 128
// tiles 62 us, every tile for itself 56; 1048576 in 256 tiles 175 and 187; 16777216
// in 4096 tiles 1.9 ms and 11.
constexpr int64_t kSortAll = 255;

inline int64_t sort_tiles(int64_t n) { return (n + 256 * sort_items(n) - 1) / (256 * sort_items(n)); }

// ------------------------------------------------------------------ gated
// Steps of a wavefront, and between the states that the forward pass leaves for
// the gradient, which computes the states between them again.
constexpr int kKeep = 16;
constexpr int kGatedWaves = 8;   // of a workgroup, at most

// Threads of a workgroup, whether chunks run side by side, and how channels are
// dealt to lanes.  One after the other, a chunk costs about 5 us (gradient 9)
// while its data is on the way; side by side there is a launch that clears what
// they publish, and their waits.  bf16, rows x steps x channels, forward and
// gradient in us, one after the other and side by side:
//   1 x 384 x 2048     19, 29    16, 21        16 x 512 x 2048     27, 44     31, 47
//   1 x 512 x 2048     24, 37    17, 21        16 x 1024 x 2048    53, 87     51, 80
//   1 x 1024 x 2048    43, 70    17, 21        128 x 1024 x 2048   321, 570   319, 518
// Five chunks are about even: 16 x 640 x 2048 34, 54 and 37, 56.
struct GatedShape {
  int32_t threads;
  int32_t nchunk;    // chunks of threads / 64 * kKeep steps
  int32_t per_row;   // workgroups to a batch row, where a wavefront stays in one
  int32_t groups;    // workgroups to a chunk
  bool link, span;
};

// keeps: runs of kKeep steps; nv: a row's words.
inline GatedShape gated_shape(int64_t batch, int64_t keeps, int64_t nv) {
  GatedShape s;
  int waves = 1;
  while (waves < kGatedWaves && waves < keeps) waves *= 2;
  s.threads = 64 * waves;
  s.nchunk = (int32_t)((keeps + waves - 1) / waves);
  s.per_row = (int32_t)((nv + 63) / 64);
  // lanes over the rows where over a fifth would idle: forward and gradient of 256 x 1000 x 16 float32 24 and 31 us, a
  // row each 37 and 49; of 64 x 1000 x 96 27 and 38, 30 and 42; of 64 x 1000 x 100, a fifth, 38 and 61, 37 and 58
  s.span = s.per_row * 64 > nv + nv / 4;
  s.groups = (int32_t)(s.span ? (batch * nv + 63) / 64 : batch * s.per_row);
  s.link = (s.nchunk > 4 || (s.nchunk > 2 && s.groups <= 64)) &&
           (int64_t)s.nchunk * s.groups < ((int64_t)1 << 22);   // tickets in the grid's 32 bits of threads
  return s;
}

// ------------------------------------------------------------------- orth
constexpr int kCUs = 256;
constexpr int kOrthSlice = 32;   // values of k in a slice

// Tiles that a product can take.
enum OrthTile { kTile64, kTile128, kTile256 };

// A launch's tiles: whole ones, and those computed in parts.  A few tiles more
// than the CUs hold in whole rounds would take a round for themselves: up to
// half a round of them is spread over the CUs in quarters.
struct OrthTiles {
  int64_t per, whole, over;
};

inline OrthTiles orth_tiles(OrthTile kind, bool sym, int64_t batch, int64_t rows, int64_t cols) {
  const int64_t side = 64 << kind, r = (rows + side - 1) / side, c = (cols + side - 1) / side;
  const int64_t per = sym ? r * (r + 1) / 2 : r * c, tiles = batch * per;
  const int64_t over = kind != kTile64 && tiles > kCUs && tiles % kCUs <= kCUs / 2 ? tiles % kCUs : 0;
  return {per, tiles - over, over};
}

// What a product takes with a kind of tile, in us for 4096 values of k: rounds
// of the CUs times what one took on this card.
inline double orth_cost(OrthTile kind, bool sym, int64_t batch, int64_t rows, int64_t cols) {
  constexpr double round[3] = {42, 112, 333};
  const OrthTiles t = orth_tiles(kind, sym, batch, rows, cols);
  return ((double)((t.whole + kCUs - 1) / kCUs) + (t.over ? 0.3 : 0.0)) * round[kind];
}

// The cheapest tile whose sides divide `pad`: large ones read less, small ones
// are more, for the CUs to share.
inline OrthTile orth_choose(int64_t pad, bool sym, int64_t batch, int64_t rows, int64_t cols, double* cost) {
  OrthTile best = kTile64;
  double least = orth_cost(best, sym, batch, rows, cols);
  const auto offer = [&](OrthTile k) {
    const double c = orth_cost(k, sym, batch, rows, cols);
    if (c < least) best = k, least = c;
  };
  if (pad >= 128) offer(kTile128);
  if (pad >= 256) offer(kTile256);
  if (cost) *cost = least;
  return best;
}

// How the tiled kernels take matrices of n x m, n <= m.
struct OrthShape {
  int64_t pad, np, mp;   // sides are padded to whole tiles of side `pad`
  int split;             // workgroups that share the sum over m of a tile of X X'
};

inline OrthShape orth_shape(int64_t batch, int64_t n, int64_t m) {
  OrthShape s{};
  double least = INFINITY;
  for (int64_t pad : {64, 128, 256}) {   // larger tiles pad more
    const int64_t np = (n + pad - 1) / pad * pad, mp = (m + pad - 1) / pad * pad;
    double square, next;
    orth_choose(pad, true, batch, np, np, &square);
    orth_choose(pad, false, batch, np, mp, &next);
    const double cost = square * (mp + np) + next * np;
    if (cost < least) least = cost, s.pad = pad, s.np = np, s.mp = mp;
  }
  // Few tiles and a long sum (16 x 9000: one tile, 282 slices): shared by so many workgroups that they fill half the
  // CUs, none with fewer than 16 slices, and added up by one more launch.
  const int64_t tiles = orth_tiles(kTile64, true, batch, s.np, s.np).per * std::max<int64_t>(batch, 1);
  s.split = (int)std::max<int64_t>(1, std::min(kCUs / 2 / tiles, s.mp / kOrthSlice / 16));
  return s;
}

}  // namespace ms
