// Host checks of the 4-bit cache's format and plan (csrc/kvq.hpp), built with the sanitizers.
#include <cassert>
#include <cmath>
#include <cstdio>
#include <cstring>
#include <random>
#include <vector>

#include "kvq.hpp"

using namespace rollpack;

// Every nibble of a block's codes is one (token, dimension) of K or V, every scale byte one (token, block).
static void layout(int hd) {
  std::vector<int> used(kvq_block_bytes(hd), 0);
  for (int t = 0; t < kKvqPage; ++t) {
    for (int d = 0; d < hd; ++d) {
      const int k = kvq_k_code(t, d, hd), v = kvq_v_code(t, d, hd);
      assert(k >= 0 && k < 32 * hd && v >= 32 * hd && v < 64 * hd);
      used[k] += 1 << (4 * (d & 1));
      used[v] += 1 << (4 * (d & 1));
      // eight dimensions of K are a word; of V a word at 128, two halves of four at 64
      assert(kvq_k_code(t, d & ~7, hd) % 4 == 0 && k - kvq_k_code(t, d & ~7, hd) == (d & 7) / 2);
      const int per = hd == 128 ? 8 : 4;
      assert(kvq_v_code(t, d / per * per, hd) % (per / 2) == 0 && v - kvq_v_code(t, d / per * per, hd) == d % per / 2);
    }
    for (int i = 0; i < hd / kKvqBlock; ++i) {
      const int k = kvq_k_scale(t, i, hd), v = kvq_v_scale(t, i, hd);
      assert(k >= 64 * hd && k < 66 * hd && v >= 66 * hd && v < 68 * hd);
      used[k] += 17;
      used[v] += 17;
    }
  }
  for (int u : used) assert(u == 17);
}

static void scales() {
  std::mt19937 rng(7);
  auto check = [](float a) {
    uint32_t bits;
    std::memcpy(&bits, &a, 4);
    const int e = static_cast<int>(kvq_scale_byte(bits)) - 127;
    const double s = std::ldexp(1.0, e);
    assert(e >= -125 && e <= 125);
    assert(a <= 7 * s || e == 125);
    assert(e == -125 || a > 7 * std::ldexp(1.0, e - 1));
  };
  for (int e = -149; e <= 127; ++e)
    for (float m : {1.f, 1.5f, 1.75f, std::nextafterf(1.75f, 2.f), std::nextafterf(1.75f, 1.f), std::nextafterf(2.f, 1.f)})
      check(std::ldexp(m, e));
  for (int i = 0; i < 100000; ++i) {
    uint32_t bits = rng() & 0x7fffffffu;
    if (bits >= 0x7f800000u) {
      assert(kvq_scale_byte(bits) == 255);
      continue;
    }
    float a;
    std::memcpy(&a, &bits, 4);
    check(a);
  }
  assert(kvq_scale_byte(0) == 2 && kvq_scale_byte(0x7f800000u) == 255 && kvq_scale_byte(0x7fc00000u) == 255);
}

// Device values out of bounds are neither followed nor counted; the items of every size that the plan may choose fit the
// bound that the launch and the workspace are made for.
static void batches() {
  std::mt19937 rng(11);
  auto pick = [&](int lo, int hi) { return lo + static_cast<int>(rng() % static_cast<uint32_t>(hi - lo + 1)); };
  KvqCache c;
  c.n_pages = 10;
  assert(!kvq_page_ok(c, -1) && kvq_page_ok(c, 0) && kvq_page_ok(c, 9) && !kvq_page_ok(c, 10) && !kvq_page_ok(c, 0x7fffffff));
  for (int round = 0; round < 4000; ++round) {
    const int n = pick(1, round % 3 ? 12 : 300), group = pick(1, 40), n_kv = pick(1, 9) * (round % 7 ? 1 : 100);
    const bool wild = round % 5 == 0;
    std::vector<int32_t> off(n + 1), ctx(n);
    KvqBatch b;
    b.n_seqs = n;
    b.max_context = pick(0, round % 4 ? 3000 : 60000);
    b.max_rows = round % 2 ? pick(0, 40) : 1;
    off[0] = pick(0, 3);
    for (int i = 0; i < n; ++i) {
      off[i + 1] = off[i] + (b.max_rows ? pick(0, b.max_rows) : 0);
      ctx[i] = pick(0, b.max_context);
      if (wild && rng() % 3 == 0) ctx[i] = static_cast<int32_t>(rng());
    }
    b.n_rows = off[n] + pick(0, 5);
    if (wild)
      for (int i = 0; i <= n; ++i)
        if (rng() % 4 == 0) off[i] = static_cast<int32_t>(rng());
    b.row_off = round % 2 ? off.data() : nullptr;
    if (!b.row_off) b.n_rows = std::max(b.n_rows, n);
    b.context = ctx.data();
    bool ascending = true;
    for (int i = 0; i < n; ++i) ascending = ascending && off[i] >= 0 && off[i + 1] >= off[i] && off[i + 1] <= b.n_rows;
    KvqPlanInput in;
    std::vector<int> pages(n), tiles(n);
    for (int i = 0; i < n; ++i) {
      const KvqSeq s = kvq_seq(b, i);
      assert(s.r0 >= 0 && s.n >= 0 && s.r0 + s.n <= b.n_rows);
      assert(s.n <= kvq_max_rows(b) && (!s.ok || (s.ctx >= 0 && s.ctx <= b.max_context)));
      pages[i] = kvq_pages(s);
      assert(pages[i] >= 0 && static_cast<int64_t>(pages[i]) * kKvqPage < b.max_context + int64_t{kKvqPage});
      tiles[i] = kvq_tiles(s, group, 16);
      if (!tiles[i]) pages[i] = 0;
      in.tile_pages += static_cast<int64_t>(tiles[i]) * pages[i];
      in.tiles += tiles[i];
      in.max_pages = std::max(in.max_pages, pages[i]);
    }
    const int64_t items = kvq_item_bound(b, n_kv, group, 16), most_tiles = kvq_tile_bound(b, group, 16);
    assert(items >= most_tiles || b.max_context <= kKvqPage);
    if (!ascending && b.row_off) continue;
    assert(in.tiles <= most_tiles);
    const int least = kvq_least_ppi(in, n_kv), most = std::max(1, in.max_pages);
    assert(least >= 1 && least <= most);
    for (int ppi = least;; ppi += std::max(1, (most - least) / 20)) {
      ppi = std::min(ppi, most);
      int64_t sum = 0;
      for (int i = 0; i < n; ++i) {
        const int k = kvq_items(pages[i], ppi);
        assert(k >= 1 && k <= kKvqTileItems && (pages[i] <= ppi) == (k == 1));
        sum += static_cast<int64_t>(tiles[i]) * k;
      }
      assert(sum <= items);
      if (ppi == most) break;
    }
  }
}

int main() {
  layout(64);
  layout(128);
  scales();
  batches();
  std::puts("4-bit cache host tests passed");
}
