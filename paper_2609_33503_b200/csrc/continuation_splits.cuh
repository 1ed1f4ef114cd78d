// Internal: how the attention over continuations cuts keys into pieces, and what its launches need (host only, no CUDA).
#pragma once
#include <algorithm>

namespace relaxkv {

// Pieces per row so that a launch of `items` (row, KV head) pairs fills the GPU with two blocks per SM, each piece at least two tiles long.
inline int paged_pieces(long long items, long long tiles, int sms, int most) {
  const long long want = std::max<long long>(1, 2LL * sms / std::max<long long>(1, items));
  return (int)std::max<long long>(1, std::min<long long>({want, (tiles + 1) / 2, (long long)most}));
}

// Pieces that merge among themselves as one cluster of blocks: no launch behind them and no way through memory.  Taken where `most` of
// them make the launch at least three quarters full, or all there are tiles for.  0: pieces for the merge are better.
inline int paged_cluster(long long items, long long tiles, int sms, int most) {
  const int want = paged_pieces(items, tiles, sms, 64);
  return want <= most ? want : 4 * items * most >= 3LL * 2 * sms ? most : 0;
}

// Consumer warps (and sixteenths of a tile's keys) of a block that streams a row's keys, listed and own, for launches of one piece per row.  A block
// takes some 7 us whatever it reads, so launches of several turns of them are better off with more and smaller ones: 6 blocks of one warp to an SM, 4
// of two or 2 of four.  (row, KV head) pairs, keys up to: 512, 16: 18.3 us with one warp, 18.5 two, 23.4 four; 512, 600: 43.8 / 35.5 / 38.7; 1024, 256:
// 38.7 / 39.5 / 46.3; 2048, 128: 48 / 54 / 69; 2048, 600: 89.3 / 87.7 / 96.2; 512, 1024: - / 81.5 / 81.1; 320, 256: 27.3 / 22.9 / 22.5; 320, 128: 21.5 / 19.7 / 21.1.  With listed blocks
// (selection included): 512, 164 34.4 / 32.7 / 36.0; 1200, 612 80.6 / 71.1 / 76.0; 1200, 2148 206 / 175 / 168.
inline int paged_warps(long long items, long long keys, int sms) {
  if (items > 6LL * sms && keys <= 256) return 1;
  return (items > 3LL * sms && keys <= 640) || (items > 2LL * sms && keys <= 128) ? 2 : 4;
}

// Scores that a block of the selection needs room for, contexts of blocks [blk_cu[b], blk_cu[b+1]) in one call: the longest context that competes (has
// more blocks than are selected) and whose scores are kept at all.  A longer one beside it takes none of that room, and must not take it away.
inline int kept_scores(const int* blk_cu, int n, int n_select, int most) {
  int kept = 0;
  for (int b = 0; b < n; ++b) {
    const int nb = blk_cu[b + 1] - blk_cu[b];
    if (nb > n_select && nb <= most) kept = std::max(kept, nb);
  }
  return kept;
}

constexpr double kPrefixStartTiles = 3.0;      // start and end of a block of the prefix kernel, in its 128-key tiles

// Key tiles per block for contexts of n_tiles[0 .. n) tiles and row_tiles[0 .. n) tiles of rows, each times `heads` KV heads, one block per SM.
// Each block takes start + its tiles; blocks that all run at once end with the longest one, more of them when the SMs have worked all of it off
// (and on average half a block later).  A piece of the longest context is one more slot for the merge: merge_tiles, in the time of a tile.
inline int prefix_tiles_per_block(const int* n_tiles, const int* row_tiles, int n, int heads, int sms, int most_pieces, double merge_tiles) {
  int longest = 1;
  for (int i = 0; i < n; ++i)
    if (row_tiles[i] > 0) longest = std::max(longest, n_tiles[i]);
  int best = longest;
  double best_cost = 0;
  for (int p = 1; p <= most_pieces && p <= std::max(1, longest / 2); ++p) {
    const int per = (longest + p - 1) / p;
    double blocks = 0, all = 0;
    for (int i = 0; i < n; ++i) {
      const double k = (double)row_tiles[i] * heads, pieces = (n_tiles[i] + per - 1) / per;
      blocks += k * pieces;
      all += k * (pieces * kPrefixStartTiles + n_tiles[i]);
    }
    const double block = kPrefixStartTiles + per;
    const double cost = (blocks <= sms ? block : std::max(block, all / sms + 0.5 * block)) + merge_tiles * (p > 1 ? p : 0);
    if (p == 1 || cost < best_cost) { best_cost = cost; best = per; }
  }
  return best;
}

}  // namespace relaxkv
