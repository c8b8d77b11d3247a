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

// The pool (device memory): a list of free pages whose entries from n_free on are of no page, the sequences' contexts and tables.
struct KvqPool {
  int32_t* page_table = nullptr; int64_t table_stride = 0;
  int32_t* context = nullptr;   // [n_seqs]
  int32_t* free_pages = nullptr;  // [n_pages]
  int32_t* state = nullptr;     // [4]: n_free, error, rows of the last call, pages it was short of
  int32_t* first_need = nullptr;  // [n_seqs] workspace: pages that the sequences before took
  int n_seqs = 0, n_pages = 0, max_context = 0;
};
enum KvqFitError { kFitOk = 0, kFitPages = 1, kFitLength = 2, kFitRows = 3, kFitPool = 4 };

struct KvqFitArgs {
  KvqPool pool;
  const int32_t* length = nullptr;  // [n_seqs]
  int32_t* row_off = nullptr;       // [n_seqs + 1]
  int32_t* position = nullptr;      // [n_rows]
  int32_t* slot = nullptr;          // [n_rows]
  int n_rows = 0;
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
};

inline PickedPlan picked_plan(const KvqCache& c, int n_rows, int n, int n_q) {
  const int G = n_q / c.n_kv;
  PickedPlan p;
  p.cols = G < 16 ? G : 16;
  p.col_tiles = (G + 15) / 16;
  const int64_t blocks = std::max<int64_t>(1, static_cast<int64_t>(n_rows) * c.n_kv * p.col_tiles);
  if (blocks < 512) p.items = static_cast<int>(std::min<int64_t>(kvq_items(n, kKvqTileItems, 8), std::max<int64_t>(1, 768 / blocks)));
  return p;
}

inline int64_t picked_blocks(const KvqCache& c, int n_rows, const PickedPlan& p) { return static_cast<int64_t>(n_rows) * c.n_kv * p.col_tiles; }

inline size_t picked_part_floats(const KvqCache& c, int n_rows, const PickedPlan& p) {  // of the partial outputs
  return p.items > 1 ? static_cast<size_t>(picked_blocks(c, n_rows, p)) * p.items * p.cols * c.hd : 0;
}
// Bytes of the workspace of launch_kvq_attend_picked.
inline size_t kvq_picked_bytes(const KvqCache& c, int n_rows, int n, int n_q) {
  const size_t o = picked_part_floats(c, n_rows, picked_plan(c, n_rows, n, n_q));
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
