// Host checks of how scores and attention over picked pages are cut and launched (csrc/kvq_pages.hpp), built with the sanitizers; as
// a library, the plans of one call for tests that have to know which kernel takes it.
#include <cassert>
#include <cmath>
#include <cstdio>
#include <random>

#include "kvq_pages.hpp"

using namespace rollpack;

static KvqBatch bounds(int n_rows, int max_rows, int max_context) {
  static const int32_t some = 0;
  KvqBatch b;
  b.n_seqs = 1;
  b.n_rows = n_rows;
  b.max_rows = max_rows;
  b.max_context = max_context;
  b.row_off = &some;  // only whether there are any matters
  return b;
}

// out: of scores, rows and tiles of a wave, whether ranges are shared; of attention, items, waves, whether pages are shared.
extern "C" void kvq_pages_plan_of(int n_q, int n_kv, int hd, int bf16, int n_rows, int max_rows, int columns, int n, int* out) {
  KvqCache c;
  c.n_kv = n_kv;
  c.hd = hd;
  const KvqBatch b = bounds(n_rows, max_rows, columns * kKvqPage);
  const ScorePlan s = score_plan(c, b, columns, bf16 != 0);
  const PickedPlan p = picked_plan(c, b, n, n_q);
  out[0] = s.rows;
  out[1] = s.tiles;
  out[2] = s.shared;
  out[3] = p.items;
  out[4] = p.waves;
  out[5] = p.shared;
}

int main() {
  std::mt19937_64 rng(7);
  auto log_pick = [&](int64_t lo, int64_t hi) {
    const double x = std::uniform_real_distribution<double>(0, 1)(rng);
    return static_cast<int64_t>(lo * std::pow(static_cast<double>(hi) / lo, x));
  };
  int split = 0, waves[9] = {0}, tiles[5] = {0};
  for (int round = 0; round < 400000; ++round) {
    KvqCache c;
    c.hd = rng() % 2 ? 128 : 64;
    c.n_kv = static_cast<int>(log_pick(1, 65));
    const int group = static_cast<int>(log_pick(1, 41)), n_q = c.n_kv * group, n = static_cast<int>(log_pick(1, 5000));
    const int n_rows = static_cast<int>(log_pick(1, (1 << 22) / c.n_kv)), columns = static_cast<int>(log_pick(1, 1 << 21));
    const KvqBatch b = bounds(n_rows, rng() % 3 ? 1 : n_rows, 64);
    const PickedPlan p = picked_plan(c, b, n, n_q);
    // every column of a row is one block's
    assert(p.cols >= 1 && p.cols <= 16 && p.col_tiles * 16 >= group && (p.col_tiles - 1) * 16 < group);
    // items cover the list, none of less than four entries' share but the last; few blocks alone are split, into what the join holds
    const int per = (n + p.items - 1) / p.items;
    assert(p.items >= 1 && p.items <= kKvqTileItems && per * p.items >= n && (p.items == 1 || (per >= 4 && p.waves == 4)));
    assert(p.items == 1 || picked_blocks(c, b, p) * p.items <= 512);
    assert(p.waves == 4 || p.waves == 8 || (p.waves == 2 && p.shared));
    assert((p.items > 1) == (kvq_picked_bytes(c, b, n, n_q) > 0));
    assert(kvq_picked_bytes(c, b, n, n_q) <= size_t{512} * 16 * (c.hd + 2) * 4);
    const bool bf16 = rng() % 2;
    const ScorePlan s = score_plan(c, b, columns, bf16);
    assert(s.rows >= 1 && s.groups * s.rows >= n_rows && (s.groups - 1) * s.rows < n_rows);
    assert(s.shared ? s.tiles == 2 || (s.tiles == 4 && bf16) : (s.tiles == 1 || s.tiles == 4) && s.rows == 1);
    // a grid: 2^32 threads in the first dimension, 65,535 blocks in the second
    assert(s.groups * c.n_kv * 256 < (int64_t{1} << 32) && (columns + 64 * s.tiles - 1) / (64 * s.tiles) < 65536);
    if (picked_blocks(c, b, p) < (int64_t{1} << 22)) assert(picked_blocks(c, b, p) * 64 * p.waves < (int64_t{1} << 32));
    split += p.items > 1;
    ++waves[p.waves];
    ++tiles[s.tiles];
  }
  assert(split > 1000 && waves[2] > 1000 && waves[4] > 1000 && waves[8] > 1000 && tiles[1] > 1000 && tiles[2] > 1000 && tiles[4] > 1000);
  std::puts("page plan tests passed");
}
