// Which forms of the kernels for scores of pages and for attention over picked ones take a call (csrc/kvq_pages.hpp), for tests that
// have to reach every one.
#include <cmath>
#include <random>

#include "kvq_pages.hpp"

using namespace rollpack;

static KvqCache cache(int n_kv, int hd) {
  KvqCache c;
  c.n_kv = n_kv;
  c.hd = hd;
  return c;
}
static KvqBatch bounds(int n_rows, int max_rows) {
  static const int32_t some = 0;
  KvqBatch b;
  b.n_seqs = 1;
  b.n_rows = n_rows;
  b.max_rows = max_rows;
  b.max_context = 64;
  b.row_off = &some;  // only whether there are any matters
  return b;
}
static int form(int n_q, int n_kv, int hd, int n_rows, int max_rows, int n) {
  const PickedPlan p = picked_plan(cache(n_kv, hd), bounds(n_rows, max_rows), n, n_q);
  return p.waves * 8 + (p.items > 1) * 4 + (p.cols > 8) * 2 + p.shared;
}
static int score_form(int n_q, int n_kv, int hd, int bf16, int n_rows, int max_rows, int columns) {
  const ScorePlan p = score_plan(cache(n_kv, hd), bounds(n_rows, max_rows), columns, bf16 != 0);
  const bool many = !p.shared && n_q > 16 * n_kv;
  return (many ? 1 : p.tiles) * 4 + many * 2 + p.shared;
}

// waves * 8, and 4 for a split list, 2 for more than eight columns, 1 for rows that may share pages.
extern "C" int kvq_picked_form_of(int n_q, int n_kv, int hd, int n_rows, int max_rows, int n) { return form(n_q, n_kv, hd, n_rows, max_rows, n); }

// seen[form] = 1 for each that some call has, of many over the whole range.
extern "C" void kvq_picked_forms(int hd, unsigned char* seen) {
  std::mt19937_64 rng(11);
  auto log_pick = [&](double lo, double hi) { return static_cast<int>(lo * std::pow(hi / lo, std::uniform_real_distribution<double>(0, 1)(rng))); };
  for (int i = 0; i < 400000; ++i) {
    const int n_kv = log_pick(1, 65), group = log_pick(1, 41), n_rows = log_pick(1, (1 << 22) / n_kv);
    seen[form(n_kv * group, n_kv, hd, n_rows, rng() % 2 ? 1 : n_rows, log_pick(1, 5000))] = 1;
  }
}

// tiles (of 16 pages to a wave) * 4, and 2 for more heads than a product has rows, 1 for rows that share ranges.
extern "C" int kvq_score_form_of(int n_q, int n_kv, int hd, int bf16, int n_rows, int max_rows, int columns) {
  return score_form(n_q, n_kv, hd, bf16, n_rows, max_rows, columns);
}
extern "C" void kvq_score_forms(int hd, int bf16, unsigned char* seen) {
  std::mt19937_64 rng(13);
  auto log_pick = [&](double lo, double hi) { return static_cast<int>(lo * std::pow(hi / lo, std::uniform_real_distribution<double>(0, 1)(rng))); };
  for (int i = 0; i < 400000; ++i) {
    const int n_kv = log_pick(1, 65), group = log_pick(1, 41), n_rows = log_pick(1, (1 << 22) / n_kv);
    seen[score_form(n_kv * group, n_kv, hd, bf16, n_rows, rng() % 2 ? 1 : n_rows, log_pick(1, 1 << 21))] = 1;
  }
}
