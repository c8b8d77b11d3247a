// Pages of the 4-bit KV cache as units of their own: handed out on the GPU from the sequences' lengths, bounded by the ranges
// of their keys, scored and picked for each query, and attended to.  Host code and device code share what is here.
//
// Ranges.  For a page and KV head, each dimension's smallest and largest key below its sequence's context, lo and hi, as
// the cache holds them: [page][KV head][lo, hi][hd] bf16, which holds every such value exactly.
//   sum_d max(q_d lo_d, q_d hi_d) = sum_d max(q_d, 0) hi_d + min(q_d, 0) lo_d  >=  q . k for every such key of the page,
// a product of [q+ | q-] with [hi | lo], 2 hd long: 4 hd bytes of a page in place of its 68 hd.
#pragma once

#include <algorithm>

#include "kvq.hpp"

namespace rollpack {

// ---- pages handed out ------------------------------------------------------------------

constexpr int kFitCounts = 16, kFitCountStride = 64, kFitWorkspace = kFitCountStride * (1 + kFitCounts);
static_assert(kFitWorkspace == 1088, "rp_kvq_pool's workspace");

// The pool (device memory): a list of free pages whose entries from n_free on are of no page, the sequences' contexts and tables.
struct KvqPool {
  int32_t* page_table = nullptr; int64_t table_stride = 0;
  int32_t* context = nullptr;   // [n_seqs]
  int32_t* free_pages = nullptr;  // [n_pages]
  int32_t* state = nullptr;     // [4]: n_free, error, rows of the last call, pages it was short of
  int32_t* workspace = nullptr;  // [kFitWorkspace]: counts of blocks, 0 between calls; [n_seqs + 1]: first_need
  int n_seqs = 0, n_pages = 0, max_context = 0;
#ifdef __HIPCC__
  __host__ __device__
#endif
  int32_t* first_need() const { return workspace + kFitWorkspace; }  // pages that the sequences before need
};
enum KvqFitError { kFitOk = 0, kFitPages = 1, kFitLength = 2, kFitRows = 3, kFitPool = 4, kFitSeqRows = 5 };

struct KvqFitArgs {
  KvqPool pool;
  const int32_t* length = nullptr;  // [n_seqs]
  int32_t* row_off = nullptr;       // [n_seqs + 1]
  int32_t* position = nullptr;      // [n_rows]
  int32_t* slot = nullptr;          // [n_rows]
  int n_rows = 0;
  int max_rows = 0, max_context = 0;  // of a sequence, in the batch that the call makes
};

// ---- ranges, scores, picks ---------------------------------------------------------------

struct KvqScoreArgs {
  KvqCache cache;
  KvqBatch batch;
  KvqTensor q;
  const uint16_t* ranges = nullptr;
  float* scores = nullptr;  // [n_rows][n_kv][columns]
  int n_q = 0, columns = 0;
};

// The last page that row i of a sequence sees; below 0: none, or its sequence is out of the batch's bounds.
RP_HD int kvq_row_sees(const KvqSeq& s, int i) { return s.ok ? (s.ctx - s.n + i) >> 6 : -1; }
// The entry of the page table that page p's id is read from, where rows see pages 0 .. `seen`: -1, none, past them.  What the table has
// behind a sequence's context is not read.
RP_HD int kvq_seen_entry(int p, int seen) { return p <= seen ? p : -1; }

// How a call of scores is cut where rows share ranges: `rows` consecutive rows and 16 `tiles` pages to a wave, more rows the more
// waves there are.
// 28/4 heads of 128, us, tiles/rows: 512 rows of 14,000 keys 1/1 42, 2/4 12.8, 2/8 10.0, 2/16 10.5, 4/16 14.2; 2,000 of 30,000
// 2/8 58, 2/16 52, 4/8 52, 4/32 33, 4/64 42; 9 rows each of 64 sequences in fp32 2/1 23, 2/4 16.7, 2/16 20.5.
//   Where each row is its sequence's only one a wave has 16 pages of it, or 64 once that leaves many waves: us, 16 | 64, 1 row of
// 30,000 keys 2.7 | 4.6, 32 of 20,000 to 30,000 7.2 | 7.9; 64 in fp32 12.4 | 11.1, 96 of up to 9,000 with 8 KV heads 8.6 | 8.3, 64 of up to
// 33,000 18.4 | 17.4.
struct ScorePlan {
  int rows = 1, tiles = 1;
  int64_t groups = 0;  // of rows
  int shared = 0;      // rows of a sequence read the same ranges
};
inline ScorePlan score_plan(const KvqCache& c, const KvqBatch& b, int columns, bool bf16) {
  ScorePlan p;
  p.shared = kvq_max_rows(b) > 1;
  auto waves = [&](int rows, int tiles) { return (static_cast<int64_t>(b.n_rows) + rows - 1) / rows * c.n_kv * ((columns + 16 * tiles - 1) / (16 * tiles)); };
  if (p.shared) {
    p.tiles = bf16 && waves(32, 4) >= 1600 ? 4 : 2;
    while (p.rows < 32 && waves(2 * p.rows, p.tiles) >= 1600) p.rows *= 2;
  } else if (waves(1, 1) >= 6144) {
    p.tiles = 4;
  }
  p.groups = (static_cast<int64_t>(b.n_rows) + p.rows - 1) / p.rows;
  return p;
}

struct KvqPickArgs {
  KvqBatch batch;
  const float* scores = nullptr;  // [n_rows][n_kv][columns]
  int32_t* picks = nullptr;       // [n_rows][n_kv][n]
  int n_kv = 0, columns = 0, first = 0, last = 0, n = 0;
};

// ---- attention over picked pages -----------------------------------------------------------

struct KvqPickedArgs {
  KvqCache cache;
  KvqBatch batch;
  KvqTensor q, out;
  const int32_t* picks = nullptr;  // [n_rows][n_kv][n]
  int n = 0, n_q = 0;
  float scale = 1.f;
  // workspace: per block and item [cols, hd] partial outputs, [2, cols] maxima and sums
  float* part_o = nullptr;
  float* part_ml = nullptr;
};

// What a call launches, from its bounds alone: a block has the up to 16 query heads (columns) of one row and KV head, and a
// share of the row's list, which `items` blocks split.
struct PickedPlan {
  int cols = 0, col_tiles = 0;  // columns of a block; blocks of a row and KV head, but for the items
  int items = 1, waves = 4;
  int shared = 0;  // rows of a sequence may read the same pages, which the caches then keep
};

// A wave takes 1 us a page, and the start and end of a block 6; a split's second launch and partial outputs take 4.5 and more.
// 7 query heads to each of 4 KV heads of 128 dims, us, whole with four waves | with eight | split: lists of 64 pages of 1 row (4
// blocks) 21.5 | 18.8 | 9.4, of 8 rows 28 | 22 | 12.3, of 16 rows 29 | 22 | 16.3; of 32 pages of 4 rows 13.4 | 12.0 | 9.8, of 16 rows 16.9 | 14.7 | 12.9,
// of 32 rows 17.6 | 15.7 | 17.0; of 16 pages of 8 rows 10.6 | 10.4 | 10.3; of 96 of 32 rows 42.6 | 34.1 | 28.7, of 64 rows 50.7 | 43.9 | 47.7; of 32
// of 96 rows (384 blocks) 25.0 | 31.8 | 33.  Many rows that share pages, with two waves | four: 200 of 8 pages 12.1 | 13.1, 512 of 32 53.8 |
// 53.5, 1,500 of 32 125 | 130; rows of their own of 48 pages (512 blocks) 50 | 45.
//   Pages that one row alone reads go past the caches; of 512 rows of 14,000 keys with 32 pages each 61 us with plain loads, 70
// so; of 64 rows of their own 43 so, 51 with plain loads (40/8 heads, 48 pages).
inline PickedPlan picked_plan(const KvqCache& c, const KvqBatch& b, int n, int n_q) {
  const int G = n_q / c.n_kv;
  PickedPlan p;
  p.cols = G < 16 ? G : 16;
  p.col_tiles = (G + 15) / 16;
  const int64_t blocks = std::max<int64_t>(1, static_cast<int64_t>(b.n_rows) * c.n_kv * p.col_tiles);
  p.shared = kvq_max_rows(b) > 1;
  if (blocks <= 128 && n >= 32 && 2 * n >= blocks) p.items = static_cast<int>(std::min<int64_t>(kvq_items(n, kKvqTileItems, 4), 512 / blocks));
  else if (blocks <= 256 && n > 16) p.waves = 8;
  else if (blocks >= 512 && p.shared) p.waves = 2;
  return p;
}

inline int64_t picked_blocks(const KvqCache& c, const KvqBatch& b, const PickedPlan& p) { return static_cast<int64_t>(b.n_rows) * c.n_kv * p.col_tiles; }

inline size_t picked_part_floats(const KvqCache& c, const KvqBatch& b, const PickedPlan& p) {  // of the partial outputs
  return p.items > 1 ? static_cast<size_t>(picked_blocks(c, b, p)) * p.items * p.cols * c.hd : 0;
}
// Bytes of the workspace of launch_kvq_attend_picked.
inline size_t kvq_picked_bytes(const KvqCache& c, const KvqBatch& b, int n, int n_q) {
  const size_t o = picked_part_floats(c, b, picked_plan(c, b, n, n_q));
  return (o + o / c.hd * 2) * 4;
}

#ifdef __HIPCC__
hipError_t launch_kvq_fit(const KvqFitArgs& a, hipStream_t s);
hipError_t launch_kvq_ranges(const KvqCache& c, const KvqBatch& b, uint16_t* ranges, hipStream_t s);
hipError_t launch_kvq_scores(const KvqScoreArgs& a, hipStream_t s);
hipError_t launch_kvq_pick(const KvqPickArgs& a, hipStream_t s);
// ws: of kvq_picked_bytes bytes.
hipError_t launch_kvq_attend_picked(const KvqPickedArgs& a, void* ws, hipStream_t s);
#endif

}  // namespace rollpack
