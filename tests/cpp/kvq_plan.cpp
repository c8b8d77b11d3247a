// Host checks of how attention over the 4-bit cache is cut and launched (csrc/kvq_plan.hpp), built with the sanitizers; as a
// library, the plan of one call for tests that have to know which kernel takes it.
#include <cassert>
#include <cmath>
#include <cstdio>
#include <random>

#include "kvq_plan.hpp"

using namespace rollpack;

// out: prompt tiles, waves, items; walk tiles, waves, items.
extern "C" void kvq_plan_of(int n_q, int n_kv, int hd, int bf16, int n_seqs, int n_rows, int max_rows, int max_context, int offsets, int* out) {
  KvqCache c;
  c.n_kv = n_kv;
  c.hd = hd;
  KvqBatch b;
  b.n_seqs = n_seqs;
  b.n_rows = n_rows;
  b.max_rows = max_rows;
  b.max_context = max_context;
  const int32_t some = 0;
  b.row_off = offsets ? &some : nullptr;  // only whether there are any matters
  const AttendPlan p = attend_plan(c, b, n_q, bf16 != 0);
  out[0] = static_cast<int>(p.prompt_tiles);
  out[1] = p.prompt_waves;
  out[2] = p.prompt.items;
  out[3] = static_cast<int>(p.walk_tiles);
  out[4] = p.waves;
  out[5] = p.walk.items;
}

int main() {
  std::mt19937_64 rng(5);
  auto log_pick = [&](int64_t lo, int64_t hi) {
    const double x = std::uniform_real_distribution<double>(0, 1)(rng);
    return static_cast<int64_t>(lo * std::pow(static_cast<double>(hi) / lo, x));
  };
  int split[2] = {0, 0}, waves[9] = {0}, prompts[9] = {0};
  for (int round = 0; round < 400000; ++round) {
    KvqCache c;
    c.hd = rng() % 2 ? 128 : 64;
    c.n_kv = static_cast<int>(log_pick(1, 65));
    const int group = static_cast<int>(log_pick(1, 41)), n_q = c.n_kv * group;
    KvqBatch b;
    const int32_t some = 0;
    b.n_seqs = static_cast<int>(log_pick(1, 2000));
    b.n_rows = b.n_seqs + static_cast<int>(log_pick(1, 40000)) - 1;
    b.row_off = rng() % 4 ? &some : nullptr;
    b.max_rows = static_cast<int>(log_pick(1, b.n_rows + 1));
    b.max_context = static_cast<int>(log_pick(1, 200000)) - (round % 100 == 0);
    if (!kvq_attend_fits(c, b, n_q)) continue;
    // an engine sizes its workspace for the most that its limits allow
    const int64_t more_seqs = b.n_seqs + (rng() % 3 ? 0 : static_cast<int64_t>(rng() % 100));
    const int more_ctx = b.max_context + (rng() % 3 ? 0 : static_cast<int>(rng() % 5000));
    assert(kvq_attend_bytes(c, b, n_q) <= kvq_attend_bytes_most(c, n_q, more_seqs, b.n_rows, more_ctx));
    for (const bool bf16 : {true, false}) {
      const AttendPlan p = attend_plan(c, b, n_q, bf16);
      assert(p.walk_tiles > 0 || p.prompt_tiles > 0);
      assert(bf16 || p.prompt_tiles == 0);
      // every count of columns is one kernel's
      assert(p.prompt_tiles == 0 ? p.walk.above == 0 && p.walk.upto == 0x7fffffff
                                 : p.walk_tiles == 0 ? p.prompt.above == 0 : p.prompt.above == p.walk.upto);
      assert(p.walk.items >= 1 && p.walk.items <= kKvqTileItems && p.prompt.items >= 1 && p.prompt.items <= kKvqTileItems);
      assert(p.walk.items == 1 || p.walk_tiles * c.n_kv <= 256);
      assert(p.prompt.items == 1 || (p.prompt_tiles * c.n_kv <= 256 && p.prompt_waves == 4));
      assert(p.waves == 1 || p.waves == 4 || p.waves == 8);
      assert(p.prompt_waves == 4 || (p.prompt_waves == 8 && c.hd == 128));
      assert(p.walk.cols == 16 && (p.prompt_tiles == 0 || p.prompt.cols == 32 * p.prompt_waves));
      assert(p.waves != 1 || p.walk.items == 1);  // one wave's blocks are many
      // a grid: 2^32 threads in the first dimension, 65,535 blocks in the others
      assert(p.walk_tiles * c.n_kv * 64 * p.waves < (int64_t{1} << 32) && p.prompt_tiles * c.n_kv * 64 * p.prompt_waves < (int64_t{1} << 32));
      if (p.walk_tiles) ++waves[p.waves], split[0] += p.walk.items > 1;
      if (p.prompt_tiles) ++prompts[p.prompt_waves], split[1] += p.prompt.items > 1;
    }
  }
  assert(split[0] > 1000 && split[1] > 1000 && waves[1] > 1000 && waves[4] > 1000 && waves[8] > 1000 && prompts[4] > 1000 && prompts[8] > 1000);
  std::puts("4-bit cache plan tests passed");
}
