// The KV cache held in 4 bits: its format, the batch that its calls take, and the plan that cuts attention
// into work items.  Host code and device code share what is here.
//
// Format.  The hd dimensions of one token and KV head are cut into blocks of 32.  A block is one scale
// byte b, the power of two s = 2^(b - 127), and 32 codes of four bits, the sign over an index into
// 0, 0.5, 1, 1.5, 2, 3, 4, 6 (e2m1): the value is s times the code's.  These are the operands of gfx950's
// v_cvt_scalef32_pk_bf16_fp4, which turns two codes and a scale into two bf16 in one instruction; bf16 holds
// every such value exactly.  4.25 bits per element: a token takes 17/64 of its bf16 size.
//   s is the least power of two with amax <= 7 s: up to 7 s the code 6 is at most s off, which is also the half
//   step of the codes below it, so a larger scale would lose more in the small elements than it gains in the largest.
//   2^-125 <= s <= 2^125 keeps every value a normal bf16 number (or zero); amax above 7 * 2^125 saturates at 6 * 2^125.
//   A block of zeros has s = 1.
//   A block that holds an infinity or a NaN gets b = 255 and reads as NaN.
//   A code is the nearest one, ties to the one with the even mantissa (v_cvt_scalef32_pk_fp4_f32's rounding).
//
// Layout.  Pages of 64 tokens, [page][KV head]: one block of 68 hd bytes
//   K codes [64 tokens x hd], V codes [64 tokens x hd], K scales [2 hd], V scales [2 hd]
// in the order in which the lanes of a wave (lane 16g + c) hold them as operands of v_mfma_f32_16x16x32_bf16, so that every load of codes is
// 16 bytes per lane and 1 KB per instruction without a gap:
//   K: MFMA row c of tile u is token 16u + c, and lane group g has dimensions hd/4 g .. hd/4 (g + 1) of it, for head
//      dimension 128 one scale block.  K scales: byte u of the lane's word is tile u's.
//   V: MFMA row c has dimensions hd/16 c .. hd/16 (c + 1) (one tile for each), and lane group g has tokens
//      16u + 4g .. 16u + 4g + 3 of tile u: those whose scores the lane gets from the K product, so that the
//      probabilities are the other operand without an exchange.  V scales: byte r of word u is token 16u + 4g + r's.
// A token's bytes are its own, so that appending never reads.
#pragma once

#include <cstddef>
#include <cstdint>

#ifndef __HIPCC__
#define RP_HD inline
#else
#include <hip/hip_runtime.h>
#define RP_HD __host__ __device__ __forceinline__
#endif

namespace rollpack {

constexpr int kKvqPage = 64;    // tokens of a page
constexpr int kKvqBlock = 32;   // dimensions that share a scale

RP_HD size_t kvq_block_bytes(int hd) { return static_cast<size_t>(68) * hd; }  // of one (page, KV head)

// Byte offsets in a (page, head) block.  Codes: of the byte that holds dimension d of token t, low half first.
RP_HD int kvq_k_code(int t, int d, int hd) {
  const int u = t >> 4, c = t & 15, g = d / (hd / 4), e = d % (hd / 4);
  return hd == 128 ? u * 1024 + (g * 16 + c) * 16 + e / 2 : (u >> 1) * 1024 + (g * 16 + c) * 16 + (u & 1) * 8 + e / 2;
}
RP_HD int kvq_v_code(int t, int d, int hd) {
  const int u = t >> 4, g = (t >> 2) & 3, r = t & 3, c = d / (hd / 16), e = d % (hd / 16);
  return 32 * hd + (hd == 128 ? u * 1024 + (g * 16 + c) * 16 + r * 4 + e / 2
                              : (u >> 1) * 1024 + (g * 16 + c) * 16 + ((u & 1) * 4 + r) * 2 + e / 2);
}
// Scales: of block i (dimensions 32i .. 32i + 31) of token t.
RP_HD int kvq_k_scale(int t, int i, int hd) { return 64 * hd + (i * 16 + (t & 15)) * 4 + (t >> 4); }
RP_HD int kvq_v_scale(int t, int i, int hd) {
  return 66 * hd + (i * 4 + ((t >> 2) & 3)) * 16 + (t >> 4) * 4 + (t & 3);
}

// The scale byte of a block whose largest magnitude has these fp32 bits (sign clear).
RP_HD uint32_t kvq_scale_byte(uint32_t amax_bits) {
  if (amax_bits >= 0x7f800000u) return 255;
  if (amax_bits == 0) return 127;
  // amax = m 2^e, 1 <= m < 2: the scale's exponent is e - 2 for m <= 1.75 and e - 1 above; the carry tells them apart
  const int b = static_cast<int>((amax_bits + 0x1fffffu) >> 23) - 2;
  return static_cast<uint32_t>(b < 2 ? 2 : b > 252 ? 252 : b);
}

// Which rows of a call belong to which sequence; pointers are device memory.
struct KvqBatch {
  int n_seqs = 0, n_rows = 0, max_rows = 1, max_context = 0;
  const int32_t* row_off = nullptr;    // [n_seqs + 1], or null: sequence b is row b
  const int32_t* context = nullptr;    // [n_seqs] with the call's rows
  const int32_t* page_table = nullptr; int64_t table_stride = 0;
  const int32_t* table_row = nullptr;  // [n_seqs] the sequence's row of the page table, or null: b
};

struct KvqCache {
  char* blocks = nullptr;
  int n_pages = 0, n_kv = 0, hd = 0;
};

// A strided [rows, heads, hd] tensor, hd contiguous; strides in elements.
struct KvqTensor {
  void* p = nullptr;
  int64_t row_stride = 0, head_stride = 0;
  int bf16 = 1;
  int vec = 0;  // pointer and strides allow accesses of 16 bytes (set by kvq_vec)
};
inline int kvq_vec(const KvqTensor& t) {
  const int64_t per = t.bf16 ? 8 : 4;
  return reinterpret_cast<uintptr_t>(t.p) % 16 == 0 && t.row_stride % per == 0 && t.head_stride % per == 0;
}

RP_HD bool kvq_page_ok(const KvqCache& c, int id) { return id >= 0 && id < c.n_pages; }

// A sequence of the batch: its rows of the call (max_rows at most), its context, and whether both are within the call's
// bounds.  Offsets outside the call's rows are taken as its ends, so that no row outside them is touched.
struct KvqSeq {
  int r0, n, ctx;
  bool ok;
};
RP_HD int kvq_clamp(int x, int lo, int hi) { return x < lo ? lo : x > hi ? hi : x; }
RP_HD int kvq_max_rows(const KvqBatch& bt) { return bt.row_off ? bt.max_rows : 1; }
RP_HD KvqSeq kvq_rows(const KvqBatch& bt, int b) {  // the rows alone
  KvqSeq s;
  if (bt.row_off) {
    s.r0 = kvq_clamp(bt.row_off[b], 0, bt.n_rows);
    s.n = kvq_clamp(bt.row_off[b + 1], s.r0, bt.n_rows) - s.r0;
  } else {
    s.r0 = b < bt.n_rows ? b : bt.n_rows;
    s.n = b < bt.n_rows ? 1 : 0;
  }
  s.ctx = 0;
  s.ok = s.n <= kvq_max_rows(bt);
  if (!s.ok) s.n = kvq_max_rows(bt);
  return s;
}
RP_HD KvqSeq kvq_seq(const KvqBatch& bt, int b) {
  KvqSeq s = kvq_rows(bt, b);
  s.ctx = bt.context[b];
  s.ok = s.ok && s.ctx >= 0 && s.ctx <= bt.max_context;
  return s;
}

// ---- how attention is cut --------------------------------------------------------------
//
// Work is counted in tiles: consecutive columns of a sequence and KV head, a column being one query head of one row (the
// G heads of a row side by side).  A tile's pages are cut into items, which blocks take; more than one item leaves partial
// outputs, which a second kernel joins.  Contexts are in device memory: the host bounds the items of a tile from the
// call's bounds, and a block counts its tile's from the context it finds, so that a captured graph follows them.

constexpr int kKvqTileItems = 64;  // items of one tile at most: the join holds one per lane

// Pages of `keys` keys; the items of a tile of so many pages, at most `most` of them and none below `least` pages unless
// it is the only one; the pages of an item.
RP_HD int kvq_pages(int keys) { return (keys + kKvqPage - 1) / kKvqPage; }
RP_HD int kvq_items(int pages, int most, int least) {
  const int n = (pages + least - 1) / least;
  return n < 1 ? 1 : n < most ? n : most;
}
RP_HD int kvq_item_pages(int pages, int items) { return items == 1 ? pages : (pages + items - 1) / items; }

// How a launch cuts a batch: tiles of `cols` columns of the sequences with more than `above` and up to `upto` columns.
struct KvqCut {
  int cols = 16;
  int find = 0;   // tiles are found by their sequences' rows (0: tile b is sequence b's only one)
  int longest = 0;  // with find: tiles of more pages come first
  int above = 0, upto = 0x7fffffff;
  int items = 1;  // of a tile at most
  int least = 1;  // pages of an item, unless it is its tile's only one
};

RP_HD int kvq_tiles(const KvqSeq& s, int group, const KvqCut& cut) {
  const int n = s.n * group;
  return n > cut.above && n <= cut.upto ? (n + cut.cols - 1) / cut.cols : 0;
}

// A tile of a sequence: its columns, the position of the sequence's first row, and the keys that some column sees.
struct KvqTile {
  int cols, first, end;
};
RP_HD KvqTile kvq_tile(const KvqSeq& s, int group, int tile, int cols) {
  KvqTile t;
  const int j0 = tile * cols, left = s.n * group - j0;
  t.cols = left < cols ? left : cols;
  t.first = s.ctx - s.n;
  const int end = t.first + (j0 + t.cols - 1) / group + 1;
  t.end = s.ok && end > 0 ? end : 0;
  return t;
}

// Of a sequence's `tiles` tiles of `cols` columns, a power of two, those that see more than `pages` pages: the last ones,
// since the keys that tile i sees, first + ((i + 1) cols - 1) / group + 1 (or all, the last), grow with i.
RP_HD int kvq_tiles_above(const KvqSeq& s, int group, int cols, int tiles, int pages) {
  if (pages < 0 || tiles == 0) return tiles;
  const int64_t keys = int64_t{kKvqPage} * pages;
  if (!s.ok || s.ctx <= keys) return 0;
  const int64_t rows = keys - (s.ctx - s.n);
  if (rows <= 0) return tiles;
  const int64_t i = (rows * group) >> __builtin_ctz(static_cast<unsigned>(cols));
  return i < tiles - 1 ? static_cast<int>(tiles - i) : 1;
}

struct KvqAttendArgs {
  KvqCache cache;
  KvqBatch batch;
  KvqTensor q, out;
  int n_q = 0;
  float scale = 1.f;
  // workspace: per item and KV head [cols, hd] partial outputs, [2, cols] maxima and sums
  float* part_o = nullptr;
  float* part_ml = nullptr;
};

// Tiles of a cut that a batch has at most (of one KV head).
inline int64_t kvq_tile_bound(const KvqBatch& b, int group, const KvqCut& cut) {
  if (!cut.find) return b.n_seqs;
  const int64_t most = static_cast<int64_t>(kvq_max_rows(b)) * group;
  const int64_t per_seq = ((most < cut.upto ? most : cut.upto) + cut.cols - 1) / cut.cols;
  const int64_t by_rows = static_cast<int64_t>(b.n_rows) * group / cut.cols + b.n_seqs, by_seqs = per_seq * b.n_seqs;
  return by_rows < by_seqs ? by_rows : by_seqs;
}

#ifdef __HIPCC__
hipError_t launch_kvq_append(const KvqCache& c, const KvqBatch& b, const KvqTensor& k, const KvqTensor& v, hipStream_t s);
struct RopeArgs;
// The engine's append: bias and RoPE on the q/k/v projection's partials, the queries out in bf16, K and V of token i
// into position a.pos[i] of page-table row a.slot[i].
hipError_t launch_kvq_rope_append(const KvqCache& c, const RopeArgs& a, hipStream_t s);
hipError_t launch_kvq_read(const KvqCache& c, const KvqBatch& b, const KvqTensor& k, const KvqTensor& v, hipStream_t s);
// ws: of kvq_attend_bytes bytes.
hipError_t launch_kvq_attend(const KvqAttendArgs& a, void* ws, hipStream_t s);
#endif

}  // namespace rollpack
