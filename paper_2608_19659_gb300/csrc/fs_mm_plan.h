// Which tiles, clusters and order the products take: estimates, on the host (no CUDA: compiled alone by a test).
#pragma once

#include <algorithm>

#ifdef __CUDACC__
#define FS_HOST_DEVICE __host__ __device__
#else
#define FS_HOST_DEVICE
#endif

namespace fs {

constexpr int kMmBlock = 128;  // bytes of a row in one block of a sum

// ---------------------------------------------------------------- few rows

constexpr int kFewStages = 12, kFewCluster = 8;  // (at most)

// A product for k_mm_few: sums over blocks_k blocks of x rows and W rows.
struct MmFewPlan {
  int w_rows;     // rows of W a tile: 32, 64 or 128 (gated: half of them gate's, half up's)
  int tokens;     // rows of x a tile: a multiple of 16, up to 128
  int token_tiles, w_tiles;
  int cluster;    // blocks that share a tile's sum
  int stages;
  float ns;       // what it takes, by estimate
};
// Tokens of a tile that a block of the cluster finishes: eights, as they come out of tensor memory, or all of fewer.
FS_HOST_DEVICE inline int tokens_each(int valid, int cluster) {
  return valid < 8 ? valid : ((valid + cluster - 1) / cluster + 7) / 8 * 8;
}

inline int ring_bytes(const MmFewPlan& p) {
  const int slot = (p.w_rows + p.tokens) * kMmBlock;
  // (the last stage's products read 128 rows, whatever a tile has)
  return std::max(p.stages * slot, (p.stages - 1) * slot + 128 * kMmBlock);
}
// A cluster's sums come while a block's own products may still read its ring; those of a single block do not.
inline int sums_bytes(const MmFewPlan& p, int rows) { return tokens_each(std::min(p.tokens, rows), p.cluster) * p.cluster * p.w_rows * 4; }
inline int sums_at(const MmFewPlan& p) { return p.cluster > 1 ? ring_bytes(p) : 0; }
inline int bars_at(const MmFewPlan& p, int rows) { return std::max(ring_bytes(p), sums_at(p) + sums_bytes(p, rows)); }

// The tile and the cluster by an estimate of the time. What it goes by, and what the other choice cost where it decides (us, in
// graphs): memory at 6.6 TB/s; a block takes 100 bytes a ns, half of that beside another on its SM, and 165 ns a step at
// least, more with fewer rows of W, 60 more for a gated one's three copies (one row of 1024 8-bit over 8192, tiles of 32 6.0, of
// 64 5.6, of 128 5.5; 64 rows of 8192 8-bit over 10240, 240 blocks 18.7, 160 21.0, 80 20.8; one row of 8192 over 2 x 1792 gated, tiles of
// 128 in clusters of 8 11.9, of 6 12.1, of 32 without 24.5); a quarter of the lesser of both, as they do not overlap in whole; a
// cluster's exchange 0.55 us and 50 bytes a ns (333 rows of 1001 over 777, tiles of 64 in clusters of three 5.8, of six 7.3); blocks
// beyond what is resident wait for a place (100 rows of 4096 over 2560, 120 blocks 9.8, 160 15.9).
inline MmFewPlan mm_few_plan(int rows, int cols, int blocks_k, bool gated, int sms) {
  MmFewPlan best{};
  for (int w_rows = 128; w_rows >= 32; w_rows /= 2)
    for (int cluster = std::min(kFewCluster, blocks_k); cluster >= 1; --cluster) {
      MmFewPlan p{};
      p.w_rows = w_rows, p.cluster = cluster;
      p.token_tiles = (rows + 127) / 128;
      p.tokens = ((rows + p.token_tiles - 1) / p.token_tiles + 15) / 16 * 16;
      const int width = gated ? w_rows / 2 : w_rows, slot = (w_rows + p.tokens) * kMmBlock, depth = (blocks_k + cluster - 1) / cluster;
      p.w_tiles = (cols + width - 1) / width;
      const int sums = cluster > 1 ? sums_bytes(p, rows) : 0;
      // one block an SM if all of them find a place so, else two where each has three stages of its own. Clusters find theirs
      // in groups of about 18 SMs, of which some are smaller (one row of 8192 over 2 x 1792 gated, tiles of 64, 280 blocks in clusters of 5: 14.4)
      const int groups = std::max(1, sms / 18);
      const long long blocks = (long long)p.w_tiles * p.token_tiles * cluster, one = cluster == 1 ? sms : 18 / cluster * cluster * groups;
      const int half = (111 * 1024 - sums) / slot;  // stages of half an SM's shared memory
      const bool two = blocks > one && half >= std::min(3, depth);
      // Half of an SM's shared memory for short sums, where that holds five stages: a block of the next kernel finds room beside this one.
      // Whole -> half (us, in graphs, weights beyond the L2, one row unless said). Up to 12 steps half is the faster in 19 of 26 shapes: 4096 8-bit over
      // 5120 7.43 -> 6.70, 8192 8-bit over 2560 7.46 -> 6.77, 64 rows of 8192 8-bit over 1280 7.19 -> 7.04; but 6000 bf16 over 1280 6.36 -> 6.68. At 14 to 22 steps
      // it is now the one, now the other: 12288 8-bit over 2560 9.18 -> 8.39, 8192 bf16 over 1280 7.15 -> 7.38, 64 rows of 8192 bf16 over 1280 8.56 -> 8.97. From 24
      // on whole is: 14336 bf16 over 1280 9.19 -> 10.13, 64 rows of 12288 bf16 over 1280 10.3 -> 11.3, 8192 bf16 over 5120 16.0 -> 16.5. (A one-token layer of 9 calls
      // on a rank of TP 8: 46.4 without, 46.1 with any bound of 8 to 24 steps.)
      const bool less = !two && half >= 5 && depth <= 12;
      p.stages = std::clamp(two || less ? half : (216 * 1024 - sums) / slot, 2, std::min(kFewStages, std::max(2, depth)));
      const long long places = !two ? one : cluster == 1 ? 2 * sms : 34 / cluster * cluster * groups;
      const float waves = (float)((blocks + places - 1) / places), rate = two ? 50.f : 100.f;
      const float step = std::max(slot / rate, (w_rows == 32 ? 230.f : w_rows == 64 ? 185.f : 165.f) + (gated ? 60.f : 0.f));
      const float memory = (float)blocks_k * kMmBlock * cols * (gated ? 2 : 1) / 6600.f, steps = waves * depth * step;
      const float read = std::max(memory, steps) + 0.25f * std::min(memory, steps);
      // what comes after the sums, a third longer beside another block: a cluster's exchange; 4 ns a token, 8 more for those that
      // go to other blocks, 15 for those that it finishes (of 128 rows of W). 150 ns for each further tile of tokens
      const float tokens = (float)std::min(rows, p.tokens), gone = (float)(cluster - 1) / cluster;
      const float after = (cluster > 1 ? 550.f : 0.f) + tokens * (4.f + gone * (8.f + w_rows / 12.5f)) + 15.f * tokens_each((int)tokens, cluster) * w_rows / 128;
      p.ns = 2600.f + 150.f * (p.token_tiles - 1) + read + waves * after * (two ? 1.3f : 1.f);
      if (best.w_rows == 0 || p.ns < 0.995f * best.ns) best = p;
    }
  return best;
}

// ---------------------------------------------------------------- many rows

constexpr int kWideTile = 256;  // rows of a tile; its columns at most

// What a block of 128 bytes of a sum takes over a tile of that width, in ns: the products of a wide one, one thread's wait, products
// and commit of a narrow one (8192 terms over one tile: 256 wide 42 us, 192 33.7, 160 29.3, 128 26.6, 96 25.7, 64 24.4).
inline float mm_wide_block(int tile) { return tile <= 128 ? 140.f + 0.22f * tile : 8.f + 1.13f * tile; }

// The width of a tile by an estimate of the time (in ns): of its sums, or of its end, 17 ns a column (with an activation; 10 without; a
// choice by 12 comes out the same), where that is longer (2048 rows of 512 over 512: 256 wide 9.6 us, 64 wide 5.3); and the longer the work the more what narrow tiles read again costs (8192 rows over
// 10240: 256 699 us, 192 816). W is read at 6.6 TB/s, and a quarter of the lesser of both comes on top (32 rows over 10240 of 8192, 160: 35.3).
inline int mm_wide_tile(int rows, int cols, int blocks, bool gated, int sms, float* ns) {
  int best = 0;
  for (int tile = kWideTile; tile >= 64; tile -= gated ? 64 : 32) {
    const int width = gated ? tile / 2 : tile;
    const long long tiles = (long long)((rows + kWideTile - 1) / kWideTile) * ((cols + width - 1) / width);
    const float waves = (float)((tiles + sms / 2 - 1) / std::max(1, sms / 2));
    const float again = 1.f + 0.08f * (256.f / tile - 1.f) * std::min(waves, 4.f);
    const float one = blocks * mm_wide_block(tile), end = 17.f * tile;
    const float sums = ((waves - 1.f) * std::max(one, end) + one) * again, memory = (float)blocks * kMmBlock * cols * (gated ? 2 : 1) / 6600.f;
    const float t = std::max(sums, memory) + 0.25f * std::min(sums, memory) + 2900.f + end;
    if (!best || t < *ns) best = tile, *ns = t;
  }
  return best;
}

// dg and du, rounded to operands of the gradients' products, are held in two terms each (a value, and what its rounding left) for results whose sums
// are a block long: dW with up to 64 rows, dx with up to 64 columns. In longer sums the roundings average out to 1.41 times the error that the
// results' own rounding makes, in these it came to 1.1 to 2.4 times; with two terms to 1.00. What it takes (us, one term -> two): 1 row of 520 over 1003 15.1 ->
// 15.9, 16 rows of 300 over 2000 20.7 -> 21.2, 1 row of 4096 over 7168 111 -> 113, 2300 rows of 256 over 64 13.3 -> 14.0, 4096 of 4096 over 64 38.5 -> 43.2. For all sums it
// would be twice the products of the second launch: 77 rows of 520 over 1003 15.8 -> 16.6 for dW alone, 4096 rows of 4096 over 512 64 -> 87 for dx.
constexpr int kTwoTermRows = 64, kTwoTermColumns = 64;
inline bool mm_two_terms_dw(int rows) { return rows <= kTwoTermRows; }
inline bool mm_two_terms_dx(int out) { return out <= kTwoTermColumns; }
// Elements of all terms: not fewer for larger sizes, as a workspace serves all up to its own.
inline long long mm_terms(int rows, int out) {
  auto both = [](long long r, long long n) { return 2 * r * ((n + 63) / 64 * 64); };
  return std::max({both(rows, out), 2 * both(std::min(rows, kTwoTermRows), out), 2 * both(rows, std::min(out, kTwoTermColumns))});
}

// The order of gradients, the product with the longest tiles first, and the width of all their tiles: few long ones set the pace
// (1362 rows, 704 and 3848, dx's 18 tiles of 121 blocks: 256 wide 69 us, 128 wide 52). Pairs that have one of those get others
// only when it is done. A tile's end is counted with 17 ns a column, as above, though gradients have no activation: by 10 some shapes come out
// wider and are up to 12 % faster (1338 rows, 1462 and 4147: 81 -> 71 us; 2102, 3287 and 577: 55 -> 49), others come out narrower and lose more (382 rows, 3819
// and 5690: 102 -> 128; 545, 2700 and 4571: 74 -> 96), and with the rounds alone changed times are the same (220, 1546 and 4401: 35.7).
struct MmGradPlan {
  bool dw_first;     // both dW ahead of dx
  int tile;
  int lead, rounds;  // pairs that start with one of the longest tiles (0: tiles in their order), and how many others that takes as long as
};
inline MmGradPlan mm_grad_plan(int rows, int in, int out, int sms) {
  const int pairs = std::max(1, sms / 2);
  const int dx_blocks = (mm_two_terms_dx(out) ? 4 : 2) * ((out + 63) / 64), dw_blocks = (mm_two_terms_dw(rows) ? 2 : 1) * ((rows + 63) / 64);
  MmGradPlan best{};
  best.dw_first = dx_blocks < dw_blocks;
  const int longest = best.dw_first ? dw_blocks : dx_blocks, shortest = best.dw_first ? dx_blocks : dw_blocks;
  float least = 0.f;
  for (int tile = kWideTile; tile >= 128; tile -= 128) {
    auto tiles = [&](int n) { return (long long)((n + kWideTile - 1) / kWideTile) * ((in + tile - 1) / tile); };
    auto ns = [&](int blocks) { return std::max(blocks * mm_wide_block(tile), 17.f * tile); };
    const long long dx = tiles(rows), dw = 2 * tiles(out), lead = best.dw_first ? dw : dx, rest = best.dw_first ? dx : dw;
    const float all = (lead * ns(longest) + rest * ns(shortest)) / pairs * (tile == kWideTile ? 1.f : 1.08f);
    const float t = std::max(ns(longest), all) + ns(shortest) + 17.f * tile;
    if (tile < kWideTile && t >= least) break;
    least = t;
    best.tile = tile;
    best.lead = lead < pairs && lead + rest > pairs ? (int)lead : 0;
    best.rounds = std::max(1, (int)(ns(longest) / ns(shortest) + 0.5f));
  }
  return best;
}

// The tile that a pair, the first-th of `step`, takes after tile i, its k-th.
FS_HOST_DEVICE inline int mm_next_tile(int i, int k, int first, int step, int lead, int rounds) {
  if (!lead) return i + step;
  const int mine = first < lead ? 1 : rounds, others = step - lead;
  if (k < mine) return lead + k * others + (first - lead);
  return lead + rounds * others + (k - mine) * step + first;
}

}  // namespace fs
