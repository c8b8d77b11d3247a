// Which kernels a call of attention over the 4-bit cache launches, how they cut it, and the workspace that this takes: host code.
#pragma once

#include <algorithm>

#include "kvq.hpp"

namespace rollpack {

// What a call of attention launches, from its bounds alone.  Times in microseconds, bf16; 7 query heads to each of 4
// KV heads of 128 dims where nothing else is said ("2 x 64" names KV heads and dims).
struct AttendPlan {
  KvqCut walk, prompt;              // k_kvq_attend's tiles and k_kvq_prompt's
  int64_t walk_tiles = 0, prompt_tiles = 0;  // at most; 0: not launched
  int waves = 4, prompt_waves = 4;  // of a block
};

// Whether k_kvq_prompt takes the sequences of more than 64 columns.  It shares a page's unpacking among 128 columns, but a
// block of it takes its pages in turn, at ~1.9 us each beside another block (1.4 at 64 dims) after a start of 8: a batch that
// does not fill the card several times takes as long as its longest tile.  k_kvq_attend splits a tile's pages among its waves and
// takes about 7 ns + 0.66 ns (0.34) a page for each 16 columns on the whole card; prompts see half of their pages on average.
// k_kvq_prompt | k_kvq_attend:
//   32 prompts of 128 tokens 27 | 34, 8 of 512 38 | 48, 4 of 2,000 147 | 261, one of 8,192 483 | 703, of 3,000 89 | 115, of 2,048
//     61 | 63, of 1,024 34 | 26, of 397 17 | 10; 2 x 64, 8 of 512 18 | 29, 2 of 2,500 59 | 63, one of 8,192 181 | 212, of 4,500 96 | 75,
//     of 2,400 50 | 28
//   32 times the last 64 rows of 1,000 keys 46 | 72, 8 times 512 of 6,000 349 | 518; 2 x 64, the latter 140 | 163
// Fewer tiles than fill the card once are split over the keys of a long context:
//   the last 512 rows of 14,000 keys 134 | 176, 128 of 14,000 52 | 54, 64 of 14,000 41 | 38, 128 of 3,000 29 | 16,
//     256 of 2,000 30 | 19; 2 x 64, 512 of 14,000 53 | 68
inline bool prompt_pays(const KvqCache& c, const KvqBatch& b, int64_t tiles, int64_t pages) {  // tiles of 16 columns, over all KV heads
  const bool whole = 2 * static_cast<int64_t>(kvq_max_rows(b)) > b.max_context;
  if (tiles < 2048) return !whole && tiles * pages * c.hd >= int64_t{1} << 22;
  const int64_t seen = whole ? pages : 2 * pages;  // in halves
  return c.hd == 128 ? tiles * (20 + seen) > 24000 + 5760 * pages : tiles * (42 + seen) > 47000 + 8100 * pages;
}

inline AttendPlan attend_plan(const KvqCache& c, const KvqBatch& b, int n_q, bool bf16) {
  const int G = n_q / c.n_kv;
  const int64_t most = static_cast<int64_t>(kvq_max_rows(b)) * G;  // columns of a sequence
  const int pages = std::max(1, kvq_pages(b.max_context));
  AttendPlan p;
  p.walk.find = most > p.walk.cols;
  if (bf16 && most > 64 && prompt_pays(c, b, kvq_tile_bound(b, G, p.walk) * c.n_kv, pages)) {
    p.prompt.find = 1;
    p.prompt.least = 8;
    if (static_cast<int64_t>(b.n_seqs) * kvq_max_rows(b) > b.n_rows) p.prompt.above = p.walk.upto = 64;  // else all have as many rows
    // Eight waves, 256 columns, halve the unpacking: 1,384 | 1,474 with four for one prompt of 14,500 tokens, 128 | 142 of
    // 4,096, 403 | 424 for the last 2,048 rows of 14,000 keys; with fewer pages the start of a block counts: 68 | 60 for 2,048
    // tokens, 122 | 112 for 20 prompts of 128 to 1,024.  At 64 dims a page is half the work: 198 | 185 for 8,192.
    p.prompt.cols = 256;
    p.prompt_tiles = kvq_tile_bound(b, G, p.prompt);
    p.prompt_waves = c.hd == 128 && pages >= 64 && p.prompt_tiles * c.n_kv >= 192 ? 8 : 4;
    p.prompt.cols = 32 * p.prompt_waves;
    p.prompt_tiles = kvq_tile_bound(b, G, p.prompt);
    // Up to 512 blocks, which the card holds at once: one more is another turn, and a split one writes 512 bytes of
    // partial output per column.  One item | two: 452 blocks, 2,048 tokens, 61 | 70; 112, the last 512 rows of 14,000
    // keys, 359 | 191, four 134, five 171.
    const int64_t blocks = std::max<int64_t>(1, p.prompt_tiles * c.n_kv);
    if (p.prompt_waves == 4 && blocks <= 256) p.prompt.items = static_cast<int>(std::min<int64_t>(kvq_items(pages, kKvqTileItems, p.prompt.least), 512 / blocks));
    p.prompt.longest = blocks > 256 && p.prompt.items == 1;
  }
  if (p.prompt_tiles && !p.prompt.above) return p;
  p.walk_tiles = kvq_tile_bound(b, G, p.walk);
  const int64_t blocks = std::max<int64_t>(1, p.walk_tiles * c.n_kv);
  p.walk.least = 4;
  // Few blocks of more than 16 pages are split into as many as run at once: one of eight waves to a compute unit where that
  // comes out nearly even, else three of four waves, two in fp32: what 128 dims' registers allow (154 and 188; at 64 dims, 111 and
  // 124, four would fit).  7 query heads to each of 4 KV heads, items of eight waves | of four: 16 tokens of 2,000 to 14,000 keys (64 blocks) 23.5 (4) | 24.5 (12), with 6 of eight
  // waves 31; 32 of 1,000 to 14,000 36 (2) | 35 (6); 48 of 1,000 to 9,000 (192 blocks) 38 (1) | 32 (4); 64 of 4,000 25 (1) | 31 (3).
  const bool few = blocks <= 256, even = few && 256 / blocks * blocks >= 224;
  if (few && pages > 16) p.walk.items = static_cast<int>(std::min<int64_t>(kvq_items(pages, kKvqTileItems, p.walk.least), (even ? 256 : bf16 ? 768 : 512) / blocks));
  // Fewer blocks start together; for a few split ones the search costs more than it gives: 8 x 16 rows of 2,000 keys 26 | 30.
  p.walk.longest = p.walk.find && blocks > 256 && p.walk.items == 1;
  const int64_t all = blocks * p.walk.items;
  const int per = kvq_item_pages(pages, p.walk.items);
  // One wave where the blocks are 512 to each page, which nothing has to join: 8 prompts of 128 tokens 13.8 | 21.8 with
  // four; 64 decoded tokens of 600 to 4,500 keys (256 blocks) 83 | 28.  Eight, where the split made room for them, for at least
  // two pages each: the latter 23 | 28, one token of 12,000 keys (64 items of 3 pages) 10.3 | 9.8.
  p.waves = all >= 512 * per ? 1 : even && per > 16 ? 8 : 4;
  return p;
}

inline size_t part_floats(const KvqCut& cut, int64_t tiles, int n_kv, int hd) {  // of the partial outputs; the maxima and sums are 2 / hd of them
  return cut.items > 1 ? static_cast<size_t>(tiles) * cut.items * n_kv * cut.cols * hd : 0;
}

// Bytes of the workspace of launch_kvq_attend.
inline size_t kvq_attend_bytes(const KvqCache& c, const KvqBatch& b, int n_q) {
  size_t most = 0;  // whatever the type
  for (const bool bf16 : {true, false}) {
    const AttendPlan p = attend_plan(c, b, n_q, bf16);
    const size_t n = part_floats(p.walk, p.walk_tiles, c.n_kv, c.hd) + part_floats(p.prompt, p.prompt_tiles, c.n_kv, c.hd);
    most = std::max(most, (n + n / c.hd * 2) * 4);
  }
  return most;
}

// The most that any batch of up to these sequences, rows and contexts asks for.
inline size_t kvq_attend_bytes_most(const KvqCache& c, int n_q, int64_t max_seqs, int64_t max_rows, int max_context) {
  // attend_plan splits up to 256 blocks of 16 columns to at most 768 items of at least 4 pages, and up to 256 of 128 to at
  // most 512 of 8; a call with both kinds has both
  const int64_t pages = kvq_pages(max_context), G = n_q / c.n_kv, rows = std::max(max_rows, max_seqs);
  auto most = [&](int64_t cols, int64_t blocks, int64_t most_items, int64_t least) {
    const int64_t per_tile = std::min<int64_t>(kKvqTileItems, (pages + least - 1) / least), tiles = rows * G / cols + max_seqs;
    const int64_t items = std::min(std::min(tiles * c.n_kv, blocks) * per_tile, most_items);
    return per_tile > 1 ? static_cast<size_t>(items) * cols * (c.hd + 2) * 4 : size_t{0};
  };
  return most(16, 256, 768, 4) + most(128, 256, 512, 8);
}

// Whether its launches are within a grid's limits.
inline bool kvq_attend_fits(const KvqCache& c, const KvqBatch& b, int n_q) {
  for (const bool bf16 : {true, false}) {
    const AttendPlan p = attend_plan(c, b, n_q, bf16);
    if (std::max(p.walk_tiles, p.prompt_tiles) * c.n_kv >= (1 << 22)) return false;  // blocks of up to 512 threads, 2^32 in a dimension
  }
  return true;
}

}  // namespace rollpack
