// How attention over the KV cache is cut into blocks (host code, without HIP).
#pragma once

#include <stdint.h>

#include <algorithm>

namespace lrqat {

constexpr int kKvRowTile = 16;
constexpr int kKvStep = 64;               // keys of a step; splits start at multiples of it
constexpr int kKvFewRows = 32;            // rows of a sequence and key/value head up to which the tiles of 16 run
constexpr int64_t kKvPartRows = 131072;   // of partial results, at most

struct KvSizes {
  int heads, d, hq;          // key/value heads, their width, query heads
  int seqs, max_new, max_cached;
  int64_t tokens, capacity;  // rows of the batch, positions that a page table holds
};
struct KvAttnPlan {
  int chunk, nsplit;      // keys of a split, and splits of the longest sequence
  int64_t tiles, blocks;  // row tiles of a sequence and key/value head; blocks of the launch
  int rows, waves;        // of a tile: 16, 128 or 256 rows
};

// Which tiles, and how a long axis is split, from the upper bounds that the host knows.
//
// Tiles of 16 rows stream the keys past few rows at the memory's rate, but again for every tile; tiles of 128 and
// 256 rows pay about 2 us a step of 64 keys however few blocks there are.  So 16 rows up to kKvFewRows, and as long as
// the tiles fit the chip at once and are 16384 steps in all at d = 128.  Measured, us, 16 rows against the better of
// the others (32 query and 8 key/value heads of 128): one sequence of 128 new tokens after 400 cached ones 12 and 22,
// after 1500 22 and 29, after 8000 75 and 56; eight of them after 400 52 and 26; eight of 32 after 1500 32 and 32,
// after 8000 134 and 74.
// 256 rows against 128, us, medians of 11 runs in turn (the same heads): prompts of 2000 tokens 77 and 70, 2500 96 and 89,
// 3000 113 and 108, 3500 137 and 149, 4000 170 and 188, 8192 626 and 662; 1000 after 1500 cached ones 72 and 77, after
// 3000 99 and 107; 2000 after 500 95 and 87, after 1000 113 and 105, after 2000 148 and 140, after 6000 285 and 295,
// after 16000 626 and 676.  At d = 64: 3000 79 and 76, 4000 116 and 111, 8192 428 and 403; 1000 after 3000 67 and 71; 2000
// after 2000 103 and 96, after 16000 421 and 453.  So how the blocks fill the chip decides as much as the keys do: the
// limit of 3000 has the larger gains on its side, and the sizes just above it where 128 rows are 4 to 9% faster.
inline KvAttnPlan kv_attn_plan(const KvSizes& z) {
  KvAttnPlan p{};
  const int64_t group = z.hq / z.heads, longest = std::max<int64_t>(1, std::min(int64_t(z.max_new) + z.max_cached, z.capacity));
  const int64_t most = z.max_new * group, heads = int64_t(z.seqs) * z.heads, steps = (longest + kKvStep - 1) / kKvStep;
  const auto units = [&](int64_t rows) { return std::max<int64_t>(1, heads * ((most + rows - 1) / rows)); };
  const int64_t u16 = units(kKvRowTile);
  if (most <= kKvFewRows || (u16 <= 512 && u16 * steps * z.d <= 16384 * 128)) {
    // eight waves fit a CU: blocks of eight where there are too few for two of four, and steps enough
    p.rows = kKvRowTile;
    p.waves = u16 <= 256 && z.d <= 128 && steps > 4 ? 8 : 4;
  } else {
    p.rows = most <= 128 || z.d > 128 || longest < 3000 ? 128 : 256;
    p.waves = p.rows / 32;
  }
  const int64_t u = units(p.rows);
  p.tiles = u / std::max<int64_t>(1, heads);
  // The number of splits whose rounds of blocks are shortest, by what a block's step takes where the memory is not the
  // limit, and a join's 4 us and traffic.  No split of fewer keys than 512, and at most kKvPartRows rows of partial results.
  // (One token, 8 key/value heads: 16000 keys 135 us in one split, 16 in 32; 64000 keys 33 us in 32 splits, 38 in 64.)
  const bool few = p.rows == kKvRowTile;
  const int64_t slots = few ? 2048 / p.waves : z.d > 128 || p.waves == 8 ? 256 : 512;
  const double step_us = !few ? 2.5 : p.waves == 8 ? 4.2 : 2.9, rows = double(z.tokens) * z.hq;
  const int64_t most_splits = std::min<int64_t>((longest + 511) / 512, rows > 0 ? std::max<int64_t>(1, int64_t(kKvPartRows / rows)) : 1);
  double best = 0;
  int64_t splits = 1;
  for (int64_t n = 1; n <= std::min<int64_t>(most_splits, 256); ++n) {
    const int64_t own = (steps + n - 1) / n, each = few ? (own + p.waves - 1) / p.waves : own;
    const double us = double((u * n + slots - 1) / slots * (each + (few ? 0 : 3))) * step_us + (n > 1 ? 4.0 + 3e-6 * rows * double(n * z.d) : 0.0);
    if (n == 1 || us < best) {
      best = us;
      splits = n;
    }
    if (u * n > 4 * slots) break;  // (more only add rounds)
  }
  const int64_t grain = splits * kKvStep * (few ? p.waves : 1);
  p.chunk = int((longest + grain - 1) / grain * (grain / splits));
  p.nsplit = int((longest + p.chunk - 1) / p.chunk);
  p.blocks = u * p.nsplit;
  return p;
}

// The keys of a split among the first `seen`: from split * chunk up to here (at or below that: none).  The last split
// has all that follow: the lengths are device memory, and a sequence longer than the plan was made for costs time but
// needs no split, and no partial results, that the workspace does not have.  Within the plan the sum stays below 2^31.
constexpr int kv_split_end(int split, int nsplit, int chunk, int seen) {
  return split + 1 < nsplit && (split + 1) * chunk < seen ? (split + 1) * chunk : seen;
}
// Whether the keys 0 .. last fall into more than one split, which are joined from partial results; and into how many (1
// where there are none).
constexpr bool kv_split_up(int64_t last, int chunk, int nsplit) { return nsplit > 1 && last >= chunk; }
constexpr int kv_splits(int64_t last, int chunk, int nsplit) {
  return last / chunk + 1 < nsplit ? int(last / chunk) + 1 : nsplit;
}

}  // namespace lrqat
