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
  assert(kvq_scale_byte(0) == 127 && kvq_scale_byte(1) == 2 && kvq_scale_byte(0x7f800000u) == 255 && kvq_scale_byte(0x7fc00000u) == 255);
}

// Device values out of bounds are not followed; tiles fit the bound that the launch and the workspace are made for, and
// a tile's items have each of its pages once.
static void batches() {
  std::mt19937 rng(11);
  auto pick = [&](int lo, int hi) { return lo + static_cast<int>(rng() % static_cast<uint32_t>(hi - lo + 1)); };
  KvqCache c;
  c.n_pages = 10;
  assert(!kvq_page_ok(c, -1) && kvq_page_ok(c, 0) && kvq_page_ok(c, 9) && !kvq_page_ok(c, 10) && !kvq_page_ok(c, 0x7fffffff));
  for (int round = 0; round < 4000; ++round) {
    const int n = pick(1, round % 3 ? 12 : 300), group = pick(1, 40);
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
    const int most = pick(1, kKvqTileItems), least = pick(1, 20), above = pick(0, 100);
    KvqCut small, large;  // the classes that two launches share
    small.find = large.find = 1;
    large.cols = 128;
    small.upto = large.above = above;
    int64_t tiles[2] = {0, 0};
    for (int i = 0; i < n; ++i) {
      const KvqSeq s = kvq_seq(b, i);
      assert(s.r0 >= 0 && s.n >= 0 && s.r0 + s.n <= b.n_rows);
      assert(s.n <= kvq_max_rows(b) && (!s.ok || (s.ctx >= 0 && s.ctx <= b.max_context)));
      assert(!(kvq_tiles(s, group, small) && kvq_tiles(s, group, large)) &&
             (kvq_tiles(s, group, small) || kvq_tiles(s, group, large)) == (s.n > 0));
      for (int k = 0; k < 2; ++k) {
        const KvqCut& cut = k ? large : small;
        const int nt = kvq_tiles(s, group, cut);
        int covered = 0;
        for (int t = 0; t < nt; ++t) {
          const KvqTile tl = kvq_tile(s, group, t, cut.cols);
          assert(tl.cols >= 1 && tl.cols <= cut.cols && t * cut.cols == covered);
          covered += tl.cols;
          assert(tl.end >= 0 && tl.end <= b.max_context && (s.ok || tl.end == 0) && (!s.ok || tl.end <= s.ctx));
          if (t + 1 == nt && s.ok) assert(tl.end == s.ctx);
          const int pages = kvq_pages(tl.end), items = kvq_items(pages, most, least), per = kvq_item_pages(pages, items);
          assert(items >= 1 && items <= most && (items == 1 || pages > least));
          int sum = 0;
          for (int j = 0; j < items; ++j) sum += std::max(0, std::min(per, pages - j * per));
          assert(sum == pages);
        }
        assert(nt == 0 || covered == s.n * group);
        for (int p = -1; p <= kvq_pages(b.max_context); p += 1 + (round % 4 ? 0 : p / 8)) {
          int more = 0;
          for (int t = 0; t < nt; ++t) more += kvq_pages(kvq_tile(s, group, t, cut.cols).end) > p;
          assert(kvq_tiles_above(s, group, cut.cols, nt, p) == more);
        }
        assert(kvq_tiles_above(s, group, cut.cols, nt, kvq_pages(b.max_context)) == 0);
        tiles[k] += nt;
      }
    }
    if (ascending || !b.row_off) assert(tiles[0] <= kvq_tile_bound(b, group, small) && tiles[1] <= kvq_tile_bound(b, group, large));
  }
}

int main() {
  layout(64);
  layout(128);
  scales();
  batches();
  std::puts("4-bit cache host tests passed");
}
