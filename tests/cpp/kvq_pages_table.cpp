// Host checks of which entries of the page table a call of scores reads (csrc/kvq_pages.hpp), built with the sanitizers: none past a
// sequence's context, all of pages that a row sees.
#include <cassert>
#include <cstdio>
#include <vector>

#include "kvq_pages.hpp"

using namespace rollpack;

int main() {
  constexpr int kMost = 330;  // tokens, in pages of 64 with lanes far past the last
  int read = 0, bad = 0;
  for (int ctx = -3; ctx <= kMost + 3; ++ctx) {
    const std::vector<int32_t> table(ctx > 0 ? static_cast<size_t>(kvq_pages(ctx)) : 0, 7);  // as long as the context
    for (int n : {1, 2, 9, 64, 65, 400}) {
      const int32_t off[] = {0, n};
      KvqBatch b;
      b.n_seqs = 1;
      b.n_rows = b.max_rows = n;
      b.max_context = kMost;
      b.row_off = off;
      b.context = &ctx;
      const KvqSeq s = kvq_seq(b, 0);
      for (int i = 0; i < n; ++i) {
        const int seen = kvq_row_sees(s, i), pos = ctx - n + i;
        assert(s.ok == (ctx >= 0 && ctx <= kMost));
        assert(!s.ok ? seen < 0 : pos < 0 ? seen < 0 : seen == pos / kKvqPage);
        for (int p = 0; p < 600; ++p) {
          const int entry = kvq_seen_entry(p, seen);
          assert(entry == -1 || entry == p);
          if (entry >= 0) read += table.at(static_cast<size_t>(entry)) == 7;
          assert((entry >= 0) == (s.ok && pos >= 0 && p <= pos / kKvqPage));
        }
        bad += !s.ok;
      }
    }
  }
  assert(read > 100000 && bad > 1000);
  std::puts("page table tests passed");
}
