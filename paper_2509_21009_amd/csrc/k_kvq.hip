// The KV cache held in 4 bits (kvq.hpp has its format): quantising rows into it, reading them back, and
// causal GQA attention over it.
#include <algorithm>

#include "kernels.hpp"
#include "kvq_device.hpp"
#include "kvq_plan.hpp"

namespace rollpack {

namespace {

// ---- append and read -----------------------------------------------------------------
//
// A wave takes `rows` (4 .. 64) consecutive rows of one KV head.  Each lane first looks up one row's place: its sequence by
// binary search in the offsets, its context, its page, three dependent reads that would otherwise come before every row's 2 KB.
// Then hd / 8 lanes have a row, eight consecutive dimensions each, K and V: 16 bytes of bf16 on one side, a word of codes
// on the other; the four (eight) rows of a step are consecutive, so that the pieces touched in the cache are 64 bytes.
// U steps at a time have their loads in flight together: one where a wave has one, else four.

// The rows of the wave's step `it` as its lanes have them.
template <int HD>
struct RowStep {
  static constexpr int LPR = HD / 8, RPS = 64 / LPR;  // lanes of a row, rows of a step
  int row, state, t;
  char* block;
  __device__ __forceinline__ RowStep(const KvqCache& c, const RowPlace& p, int base, int kh, int it) {
    const int lane = threadIdx.x & 63, src = it * RPS + lane / LPR;
    const int st = __shfl(p.state | p.t << 2, src & 63, 64), page = __shfl(p.page, src & 63, 64);
    row = base + src;
    state = st & 3;
    t = st >> 2;
    block = c.blocks + (static_cast<size_t>(page) * c.n_kv + kh) * kvq_block_bytes(HD);
  }
};

// Eight values to a word of codes and the scale byte of their block, whose other values the neighbouring three lanes
// have (NaN and infinity order above every finite value by their bits, so the maximum finds them).
__device__ __forceinline__ uint32_t quantise8(const float (&f)[8], uint32_t& byte) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(f[i]) & 0x7fffffffu);
  top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 1, 64)));
  top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 2, 64)));
  byte = kvq_scale_byte(top);
  if (byte == 255) return 0;  // its codes say nothing
  const float s = __uint_as_float(byte << 23);
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[0], f[1], s, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[2], f[3], s, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[4], f[5], s, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[6], f[7], s, 3);
  return w;
}

__device__ __forceinline__ void dequantise8(uint32_t w, uint32_t byte, float (&f)[8]) {
  const float s = __uint_as_float(byte << 23);  // 255: the conversion gives NaN
  const uint32_t p[4] = {code_pair<0>(w, s), code_pair<1>(w, s), code_pair<2>(w, s), code_pair<3>(w, s)};
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(i & 1 ? p[i / 2] & 0xffff0000u : p[i / 2] << 16);
}

// Eight dimensions of V lie in a word at hd 128, in two halves of one at 64.
template <int HD>
__device__ __forceinline__ void put_values(char* block, int t, int d, uint32_t w) {
  if constexpr (HD == 128) {
    *reinterpret_cast<uint32_t*>(block + kvq_v_code(t, d, HD)) = w;
  } else {
    *reinterpret_cast<uint16_t*>(block + kvq_v_code(t, d, HD)) = static_cast<uint16_t>(w);
    *reinterpret_cast<uint16_t*>(block + kvq_v_code(t, d + 4, HD)) = static_cast<uint16_t>(w >> 16);
  }
}
template <int HD>
__device__ __forceinline__ uint32_t get_values(const unsigned char* block, int t, int d) {
  if constexpr (HD == 128) {
    return *reinterpret_cast<const uint32_t*>(block + kvq_v_code(t, d, HD));
  } else {
    return *reinterpret_cast<const uint16_t*>(block + kvq_v_code(t, d, HD)) |
           static_cast<uint32_t>(*reinterpret_cast<const uint16_t*>(block + kvq_v_code(t, d + 4, HD))) << 16;
  }
}

// 11,511 tokens of the 7B layer (4 KV heads of 128) 10.8 us, 2.8 TB/s in and out: the launch and the lookups (three to ten reads
// that wait for each other) are half of it; one token each of 64 sequences 4.1 us.  Values come with plain loads: rows that the
// projection has just written are in the caches (past them: 21.7 | 21.0 us with the read-back for the former, 151 | 164 for
// 67,000 tokens of 8 heads).
template <int HD, bool BF16, int U>
__global__ __launch_bounds__(256) void k_kvq_append(KvqCache c, KvqBatch bt, KvqTensor k, KvqTensor v, int rows) {
  const int lane = threadIdx.x & 63, d = lane % (HD / 8) * 8;
  const int wave = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = wave / c.n_kv, kh = wave - g * c.n_kv, base = g * rows;
  if (base >= bt.n_rows) return;
  const RowPlace place = lane < rows ? row_place(c, bt, base + lane) : RowPlace{0, 0, 0};
  for (int it = 0; it < rows / RowStep<HD>::RPS; it += U) {
    float kf[U][8], vf[U][8];
#pragma unroll
    for (int n = 0; n < U; ++n) {
      const RowStep<HD> p(c, place, base, kh, it + n);
#pragma unroll
      for (int e = 0; e < 8; ++e) kf[n][e] = vf[n][e] = 0.f;
      if (p.state == 1 && it + n < rows / RowStep<HD>::RPS) {
        load8<BF16>(k, p.row, kh, d, kf[n]);
        load8<BF16>(v, p.row, kh, d, vf[n]);
      }
    }
#pragma unroll
    for (int n = 0; n < U; ++n) {
      if (it + n >= rows / RowStep<HD>::RPS) break;
      const RowStep<HD> p(c, place, base, kh, it + n);
      uint32_t kb, vb;
      const uint32_t kw = quantise8(kf[n], kb), vw = quantise8(vf[n], vb);  // every lane: the maxima cross lanes
      if (p.state != 1) continue;
      *reinterpret_cast<uint32_t*>(p.block + kvq_k_code(p.t, d, HD)) = kw;
      put_values<HD>(p.block, p.t, d, vw);
      if (d % kKvqBlock == 0) {
        p.block[kvq_k_scale(p.t, d / kKvqBlock, HD)] = static_cast<char>(kb);
        p.block[kvq_v_scale(p.t, d / kKvqBlock, HD)] = static_cast<char>(vb);
      }
    }
  }
}

// HBM bounds it: 163,000 tokens of the 7B layer 73 us alone, 5.8 TB/s, 84 to 100 one after another.  What it writes goes past
// the caches; with plain stores it took 19 us more.
template <int HD, bool BF16, int U>
__global__ __launch_bounds__(256) void k_kvq_read(KvqCache c, KvqBatch bt, KvqTensor k, KvqTensor v, int rows) {
  const int lane = threadIdx.x & 63, d = lane % (HD / 8) * 8;
  const int wave = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = wave / c.n_kv, kh = wave - g * c.n_kv, base = g * rows;
  if (base >= bt.n_rows) return;
  const RowPlace place = lane < rows ? row_place(c, bt, base + lane) : RowPlace{0, 0, 0};
  for (int it = 0; it < rows / RowStep<HD>::RPS; it += U) {
    uint32_t kw[U], vw[U], kb[U], vb[U];
#pragma unroll
    for (int n = 0; n < U; ++n) {  // places without a position read page 0
      const RowStep<HD> p(c, place, base, kh, it + n);
      const unsigned char* u = reinterpret_cast<const unsigned char*>(p.block);
      kw[n] = *reinterpret_cast<const uint32_t*>(u + kvq_k_code(p.t, d, HD));
      vw[n] = get_values<HD>(u, p.t, d);
      kb[n] = u[kvq_k_scale(p.t, d / kKvqBlock, HD)];
      vb[n] = u[kvq_v_scale(p.t, d / kKvqBlock, HD)];
    }
#pragma unroll
    for (int n = 0; n < U; ++n) {
      const RowStep<HD> p(c, place, base, kh, it + n);
      if (p.state == 0 || it + n >= rows / RowStep<HD>::RPS) continue;
      float kf[8], vf[8];
      dequantise8(kw[n], kb[n], kf);
      dequantise8(vw[n], vb[n], vf);
      if (p.state != 1) {
        const float x = p.state == 2 ? 0.f : __builtin_nanf("");
#pragma unroll
        for (int e = 0; e < 8; ++e) kf[e] = vf[e] = x;
      }
      store8<BF16, true>(k, p.row, kh, d, kf);
      store8<BF16, true>(v, p.row, kh, d, vf);
    }
  }
}

// The engine's append.  A thread has eight rotated pairs of a query or key head (dimensions d .. d + 7 and d + hd/2 ..)
// or eight dimensions of a value head of one row; the four threads of a scale block are neighbours.  A decode step of 64 rows
// (7B layer) takes it 4.1 us, of 330 6.2; 16,384 prompt tokens 71 us, 4.6 TB/s: HBM, the partials.  The S partials are all
// loaded before the first is added.  Keys and values are quantised from fp32: one rounding.
template <int HD, int S>
__global__ __launch_bounds__(256) void k_kvq_rope_append(KvqCache c, RopeArgs a) {
  constexpr int HALF = HD / 2, PER = HALF / 8, VPER = HD / 8;
  const int nq_el = a.n_q * HD, nk_el = a.n_kv * HD, nqkv = nq_el + 2 * nk_el;
  const int units = (a.n_q + a.n_kv) * PER + a.n_kv * VPER;  // of a row, a multiple of four
  const int64_t idx = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  const int i = static_cast<int>(idx / units), u = static_cast<int>(idx - static_cast<int64_t>(i) * units);
  if (i >= a.M) return;
  const bool value = u >= (a.n_q + a.n_kv) * PER;
  const int uv = u - (a.n_q + a.n_kv) * PER;
  const int head = value ? uv / VPER : u / PER, d = value ? uv % VPER * 8 : u % PER * 8;
  const int n1 = value ? nq_el + nk_el + head * HD + d : head * HD + d;
  const size_t plane = static_cast<size_t>(a.M) * nqkv;
  const float* p = a.part + static_cast<size_t>(i) * nqkv + n1;
  const int second = value ? 0 : HALF;
  f32x4_t w[S][4];
#pragma unroll
  for (int s = 0; s < S; ++s)
#pragma unroll
    for (int k = 0; k < 4; ++k) w[s][k] = *reinterpret_cast<const f32x4_t*>(p + s * plane + (k >= 2 ? second : 0) + 4 * (k & 1));
  const int pos = a.pos[i], slot = a.slot[i];
  const bool isq = !value && head < a.n_q;
  const bf16_t* bias = value ? static_cast<const bf16_t*>(a.bv) + head * HD + d
                       : isq ? static_cast<const bf16_t*>(a.bq) + n1
                             : static_cast<const bf16_t*>(a.bk) + n1 - nq_el;
  const u32x4 b1 = *reinterpret_cast<const u32x4*>(bias), b2 = *reinterpret_cast<const u32x4*>(bias + second);
  const float* cs = a.rope_cos + static_cast<size_t>(pos) * HALF + (value ? 0 : d);
  const float* sn = a.rope_sin + static_cast<size_t>(pos) * HALF + (value ? 0 : d);
  float x[8], y[8];
#pragma unroll
  for (int s = 1; s < S; ++s)
#pragma unroll
    for (int k = 0; k < 4; ++k) w[0][k] += w[s][k];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    x[e] = w[0][e >> 2][e & 3] + __uint_as_float(e & 1 ? b1[e >> 1] & 0xffff0000u : b1[e >> 1] << 16);
    y[e] = w[0][2 + (e >> 2)][e & 3] + __uint_as_float(e & 1 ? b2[e >> 1] & 0xffff0000u : b2[e >> 1] << 16);
  }
  if (!value) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float r1 = x[e] * cs[e] - y[e] * sn[e], r2 = y[e] * cs[e] + x[e] * sn[e];
      x[e] = r1;
      y[e] = r2;
    }
    if (isq) {
      const KvqTensor q{a.q_out, nq_el, HD, 1, 1};
      store8<true>(q, i, head, d, x);
      store8<true>(q, i, head, d + HALF, y);
      return;
    }
  }
  const int kh = value ? head : head - a.n_q, t = pos % kKvqPage;
  const int page = a.page_table[static_cast<size_t>(slot) * a.pt_stride + pos / kKvqPage];
  char* block = c.blocks + (static_cast<size_t>(page) * c.n_kv + kh) * kvq_block_bytes(HD);
  uint32_t byte;
  const uint32_t c1 = quantise8(x, byte);
  if (value) {
    put_values<HD>(block, t, d, c1);
    if (d % kKvqBlock == 0) block[kvq_v_scale(t, d / kKvqBlock, HD)] = static_cast<char>(byte);
  } else {
    uint32_t byte2;
    const uint32_t c2 = quantise8(y, byte2);
    *reinterpret_cast<uint32_t*>(block + kvq_k_code(t, d, HD)) = c1;
    *reinterpret_cast<uint32_t*>(block + kvq_k_code(t, d + HALF, HD)) = c2;
    if (d % kKvqBlock == 0) {
      block[kvq_k_scale(t, d / kKvqBlock, HD)] = static_cast<char>(byte);
      block[kvq_k_scale(t, (d + HALF) / kKvqBlock, HD)] = static_cast<char>(byte2);
    }
  }
}

// ---- which tile a block has ------------------------------------------------------------

// Tile `index` of the cut: its sequence (-1 past the last) and which of the sequence's.  Each wave finds it for itself.
// Up to 64 sequences: a lane has one, context and all, so that nothing is read twice.  More: lane l counts the sequences
// l per .. (l + 1) per - 1 (no further than 2^24, should offsets that do not ascend say more).
__device__ __forceinline__ int find_tile(const KvqBatch& bt, int group, const KvqCut& cut, int index, int& tile, KvqSeq& sq) {
  const int lane = threadIdx.x & 63;
  if (bt.n_seqs <= 64) {
    const KvqSeq s = kvq_seq(bt, min(lane, bt.n_seqs - 1));
    const int mine = lane < bt.n_seqs ? min(kvq_tiles(s, group, cut), 1 << 24) : 0, scan = wave_scan(mine);
    const uint64_t past = __ballot(scan > index);
    if (!past) return -1;
    const int w = __ffsll(static_cast<unsigned long long>(past)) - 1;
    tile = index - __builtin_amdgcn_readlane(scan - mine, w);
    sq.r0 = __builtin_amdgcn_readlane(s.r0, w);
    sq.n = __builtin_amdgcn_readlane(s.n, w);
    sq.ctx = __builtin_amdgcn_readlane(s.ctx, w);
    sq.ok = __builtin_amdgcn_readlane(s.ok, w);
    return w;
  }
  const int per = (bt.n_seqs + 63) >> 6, b0 = lane * per, b1 = min(b0 + per, bt.n_seqs);
  int mine = 0;
#pragma unroll 4
  for (int b = b0; b < b1; ++b) mine = min(mine + min(kvq_tiles(kvq_rows(bt, b), group, cut), 1 << 24), 1 << 24);
  const int scan = wave_scan(mine);
  const uint64_t past = __ballot(scan > index);
  if (!past) return -1;
  const int w = __ffsll(static_cast<unsigned long long>(past)) - 1;
  tile = index - __builtin_amdgcn_readlane(scan - mine, w);
  for (int b = w * per;; ++b) {  // within that lane's sequences
    sq = kvq_seq(bt, b);
    const int t = kvq_tiles(sq, group, cut);
    if (tile < t) return b;
    tile -= t;
  }
}

// The same with each sequence's last tile first, which sees most keys.  cut.longest, up to 64 sequences: over all of them,
// a lane each, tiles of more pages first; the pages of tile `index` are the most of which so many tiles have more, found by
// halves.  The last blocks to start are then short ones, and neighbours have the KV heads of a tile.  20 prompts of 128 to
// 1,024 tokens 126 us sequence by sequence, 112 so; 32 sequences' last 20 rows of 1,000 keys 37 | 29 (k_kvq_attend).
__device__ __forceinline__ int find_longest(const KvqBatch& bt, int group, const KvqCut& cut, int index, int& tile, KvqSeq& sq) {
  if (!cut.longest || bt.n_seqs == 1 || bt.n_seqs > 64) {
    const int b = find_tile(bt, group, cut, index, tile, sq);
    if (b >= 0) tile = kvq_tiles(sq, group, cut) - 1 - tile;
    return b;
  }
  const int lane = threadIdx.x & 63;
  const KvqSeq s = kvq_seq(bt, min(lane, bt.n_seqs - 1));
  const int tiles = lane < bt.n_seqs ? min(kvq_tiles(s, group, cut), 1 << 24) : 0;
  auto above = [&](int pages) { return kvq_tiles_above(s, group, cut.cols, tiles, pages); };  // of the lane's, with more pages
  auto total = [&](int x) { return __builtin_amdgcn_readlane(wave_scan(x), 63); };
  if (index >= total(tiles)) return -1;
  int lo = -1, hi = kvq_pages(bt.max_context);  // more than `index` tiles have more pages than lo, no more than that than hi
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (total(above(mid)) > index) lo = mid; else hi = mid;
  }
  const int more = above(hi), mine = above(hi - 1) - more, scan = wave_scan(mine), left = index - total(more);
  const int w = __ffsll(static_cast<unsigned long long>(__ballot(scan > left))) - 1;
  tile = __builtin_amdgcn_readlane(tiles - 1 - more - (left - scan + mine), w);
  sq.r0 = __builtin_amdgcn_readlane(s.r0, w);
  sq.n = __builtin_amdgcn_readlane(s.n, w);
  sq.ctx = __builtin_amdgcn_readlane(s.ctx, w);
  sq.ok = __builtin_amdgcn_readlane(s.ok, w);
  return w;
}

// ---- attention, 16 columns a block ------------------------------------------------------

// One block of NW waves takes an item: 16 columns of a sequence and KV head (a column is a query head of a row, the
// G heads of a row side by side) over a range of pages, which the waves take in turn.  Per page a wave forms
// S^T = K Q^T, an online softmax in the log2 domain and O^T += V^T P^T with MFMA, straight from registers: no
// value of the cache is used by more than one wave, so nothing passes through LDS but the waves' results.  The next
// page's K is loaded when the scores are formed, its V when the outputs are.
//   P is an operand rounded to fp16 (2^-11 of it at most, and see Softmax), V exact in it: less than the output's own
// rounding to bf16, 2^-8, where P in bf16 would add as much again.  Pages with values that fp16 does not hold, and fp32, take
// bf16: P in two pieces, or three.
//   HBM bounds decoding of many keys: one token each of 64 sequences of 600 to 4,500 (7B layer, 163,000 keys) 23 us, 3.9 TB/s;
// of 330 of 200 to 1,700 38.5 us, 4.6; of 96 of 32B's layer, 442,000 keys, 96 us, 5.1, what a copy reaches.  Below that it is
// the way to the first page (context, table, page: reads that wait for each other), the launch and the join: 12,000 keys of one
// sequence 6.6 us and 4.2 for the join.
template <int HD, bool F32, int NW>
__global__ __launch_bounds__(64 * NW, F32 ? 2 : 3) void k_kvq_attend(KvqAttendArgs a, KvqCut cut) {
  constexpr int NT = HD / 16, OLD = HD + 4;
  __shared__ __attribute__((aligned(16))) float so[NW][16 * OLD];
  __shared__ float sm[NW][16], sl[NW][16];
  const KvqBatch& bt = a.batch;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 4, c = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n_kv = a.cache.n_kv, G = a.n_q / n_kv;
  const int split = blockIdx.z;
  int index = blockIdx.x, kh = blockIdx.y, tile = 0, b = index;
  KvqSeq sq;
  if (cut.find) {
    index = blockIdx.x / n_kv;
    kh = blockIdx.x - index * n_kv;
    b = find_longest(bt, G, cut, index, tile, sq);
  } else {
    sq = kvq_seq(bt, b);
  }
  if (b < 0) return;
  const KvqTile tl = kvq_tile(sq, G, tile, cut.cols);
  const int j0 = tile * 16, n_cols = tl.cols, first = tl.first;
  const int pages = kvq_pages(tl.end), items = kvq_items(pages, cut.items, cut.least);
  if (n_cols <= 0 || split >= items) return;
  const int per_item = kvq_item_pages(pages, items), p0 = split * per_item;
  const int np = max(0, min(per_item, pages - p0));
  const int nw = np > wave ? (np - wave + NW - 1) / NW : 0;  // this wave's pages: wave, wave + NW, ...
  const int open = first + j0 / G + 1;  // keys that every column sees

  // The column: its query, and the last key that it sees.
  const int cc = min(c, n_cols - 1), row = (j0 + cc) / G, head = kh * G + (j0 + cc) - row * G;
  const int lim = sq.ok ? first + row : -1;
  const float scale_log2 = a.scale * kLog2e;

  f32x4_t o[NT];
#pragma unroll
  for (int i = 0; i < NT; ++i) o[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  Softmax st;
  if (nw > 0) {
    const int32_t* pt = table_of(bt, b) + p0;
    const int ptv = lane < np ? pt[lane] : 0;  // lane i has page i of the item, the first 64
    const size_t bytes = kvq_block_bytes(HD);
    const char* base = a.cache.blocks + kh * bytes;
    bool lost = false, lost_next = false;  // the page's id is outside the cache: page 0 stands in, and its scores are NaN
    auto block_of = [&](int i) {
      const int q = min(wave + NW * i, np - 1);  // past the last page: the last again
      const int id = q < 64 ? __builtin_amdgcn_readlane(ptv, q) : pt[q];
      lost_next = !kvq_page_ok(a.cache, id);
      return base + static_cast<size_t>(lost_next ? 0 : id) * n_kv * bytes;
    };
    Query<HD, F32 ? 3 : 1> qf;
    qf.load(a.q, sq.r0 + row, head);
    auto rescale = [&](float alpha) {
#pragma unroll
      for (int t = 0; t < NT; ++t) o[t] *= alpha;
    };
    int i = 0;
    // The wave's pages from i on.  HALF: V and P in fp16, up to the first page that does not fit; else in bf16.
    auto walk = [&](auto half_tag) {
      constexpr bool HALF = half_tag.value;
      PageK<HD> pk;
      PageV<HD> pv;
      const char* at = block_of(i);
      lost = lost_next;
      pk.load(at);
      pv.load(at);
      for (; i < nw; ++i) {
        const int tok0 = (p0 + wave + NW * i) * kKvqPage;
        f32x4_t s[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) s[u] = qf.scores(pk, u);
        const char* next = block_of(i + 1);
        pk.load(next);
        const int held = lost ? tok0 : tl.end;  // what lies behind the last key, or in a page that stands in, may be anything
        if (tok0 + kKvqPage > held) {
#pragma unroll
          for (int u = 0; u < 4; ++u) pv.s[u] = scales_below(pv.s[u], tok0 + 16 * u + 4 * g, held);
        }
        if (HALF && !__all(fits_half(pv.s))) return;
        if (lost || tok0 + kKvqPage > open) {
          asm volatile("");  // a branch: as selects it would cost every page
#pragma unroll
          for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float v = lost ? __builtin_nanf("") : s[u][e];
              s[u][e] = tok0 + 16 * u + 4 * g + e > lim ? -INFINITY : v;
            }
        }
        float x[16];
        uint32_t w[8];
#pragma unroll
        for (int k = 0; k < 16; ++k) x[k] = s[k >> 2][k & 3];
        softmax_page<HALF>(st, x, w, scale_log2, rescale, [&](const uint32_t (&small)[8]) {
          if constexpr (HALF) {
            half_values<HD, true, 1>(pv, 0, x, small, o);
            half_values<HD, true, 1>(pv, 1, x, small, o);
          }
        }, 16, 32);
        if (!HALF && !__all(fits_half(pv.s))) nan_values<HD>(pv, at, tok0, lim, o);
        half_values<HD, HALF, F32 ? 3 : 2>(pv, 0, x, w, o);
        half_values<HD, HALF, F32 ? 3 : 2>(pv, 1, x, w, o);
        at = next;
        lost = lost_next;
        pv.load(at);
      }
    };
    if constexpr (!F32) {
      walk(std::true_type{});
      if (i < nw) leave_half(st, rescale);
    }
    if (F32 || i < nw) walk(std::false_type{});
    st.l += __shfl_xor(st.l, 16, 64);
    st.l += __shfl_xor(st.l, 32, 64);
  }

  // Combine the waves: one without a page has m = -inf, l = 0, o = 0.
  if (g == 0) {
    sm[wave][c] = st.m;
    sl[wave][c] = st.l;
  }
  __syncthreads();
  float mx = sm[0][c];
#pragma unroll
  for (int w = 1; w < NW; ++w) mx = fmaxf(mx, sm[w][c]);
  const float fac = st.m == -INFINITY ? (st.l == 0.f ? 0.f : 1.f) : __builtin_amdgcn_exp2f(st.m - mx);
  if (c < n_cols) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int i = 0; i < NT; i += 4)  // dimensions hd/16 (4g + e) + i ..
        *reinterpret_cast<f32x4_t*>(&so[wave][c * OLD + (4 * g + e) * NT + i]) =
            f32x4_t{o[i][e], o[i + 1][e], o[i + 2][e], o[i + 3][e]} * fac;
  }
  __syncthreads();
  const int64_t part = (static_cast<int64_t>(index) * cut.items + split) * n_kv + kh;
  for (int q = tid; q < n_cols * (HD / 8); q += 64 * NW) {
    const int col = q / (HD / 8), d = q % (HD / 8) * 8;
    float m4 = sm[0][col], den = 0.f, x[8];
#pragma unroll
    for (int w = 1; w < NW; ++w) m4 = fmaxf(m4, sm[w][col]);
#pragma unroll
    for (int w = 0; w < NW; ++w)
      den += sm[w][col] == -INFINITY ? sl[w][col] : sl[w][col] * __builtin_amdgcn_exp2f(sm[w][col] - m4);
    f32x4_t y[2]{};
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      y[0] += *reinterpret_cast<const f32x4_t*>(&so[w][col * OLD + d]);
      y[1] += *reinterpret_cast<const f32x4_t*>(&so[w][col * OLD + d + 4]);
    }
    if (items == 1) {
      const int r = (j0 + col) / G, h = kh * G + (j0 + col) - r * G;
      // a row before the sequence's first token sees no key: zeros; a sequence out of bounds: NaN
      const float inv = !sq.ok ? __builtin_nanf("") : first + r < 0 ? 0.f : 1.f / den;
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] = y[k >> 2][k & 3] * inv;
      store8<!F32>(a.out, sq.r0 + r, h, d, x);
    } else {
      float* po = a.part_o + (part * 16 + col) * HD + d;
      *reinterpret_cast<f32x4_t*>(po) = y[0];
      *reinterpret_cast<f32x4_t*>(po + 4) = y[1];
      if (d == 0) {
        a.part_ml[part * 32 + col] = m4;
        a.part_ml[part * 32 + 16 + col] = den;
      }
    }
  }
}

// ---- attention of many rows -------------------------------------------------------------
//
// A block of NW waves owns 32 NW columns of a sequence and KV head, 32 a wave, and walks the pages that they see.  A page
// is unpacked once per block, every thread a share of it, into LDS, from where the waves' 32x32x16 MFMAs take it: a wave
// alone would spend more instructions on unpacking a page than on its softmax.  Two stages of LDS: page p + 1 is unpacked
// from registers while the block's other waves compute page p, and page p + 2 is on its way to the registers.
//   S^T = K Q^T in two tiles of 32 tokens: lane 32h + c gets tokens 8i + 4h + 0..3 of each, for column c, which in pairs
// of i are the operand P^T of a 16-token step of O^T += V^T P^T; V's rows keep the cache's order of tokens, so that
// nothing moves between lanes.  V's row c + 16 i of tile t is dimension hd/16 c + 2 t + i: the two that one byte holds.
//   Bound by MFMA and the vector ALU together: of a long prompt's SIMD cycles the one takes about 40%, the other (unpacking,
// softmax) 45 to 50, hardly at the same time though a SIMD has two waves (of two blocks of four waves, or of one of eight: 240
// registers); products and softmax of neighbouring pages interleaved in one wave took more registers than that hid.  One prompt
// of 14,500 tokens (7B layer) 1,420 to 1,510 us from card to card, 1,000 to 1,060 TFLOP/s, with blocks of eight waves; 20 of 128 to
// 1,024 tokens 114 us, 510, where the way to a block's first page and the first unpacking, ~7 us, are as long as its five pages.

typedef __attribute__((__vector_size__(16 * sizeof(float)))) float f32x16;

// One thread's share of a page between its load and LDS.  256 threads unpack K, 32 codes each at hd 128 (16 at 64), and 256
// V, two dimension pairs (one) of eight tokens: the same ones in a block of four waves, waves 0-3 and 4-7 in one of eight.
template <int HD>
struct PageShare {
  static constexpr int KW = HD / 32, VB = HD / 64;  // words of K; bytes of V per token
  uint32_t k[KW], v[8], ks, vs[2];
  uint32_t all;  // four value scales of the page, a lane's share of all of them
  bool lost;
};

template <int HD>
__device__ __forceinline__ void share_load(PageShare<HD>& s, const char* block, int th, bool has_k, bool has_v) {
  if (has_k) {
    const int u = th >> 6, g = (th >> 4) & 3, c = th & 15;
    const char* p = block + kvq_k_code(16 * u + c, g * (HD / 4), HD);
    if constexpr (HD == 128) {
      const u32x4 w = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
      for (int i = 0; i < 4; ++i) s.k[i] = w[i];
    } else {
      const uint2 w = *reinterpret_cast<const uint2*>(p);
      s.k[0] = w.x;
      s.k[1] = w.y;
    }
    s.ks = static_cast<unsigned char>(block[kvq_k_scale(16 * u + c, g * (HD / 4) / kKvqBlock, HD)]);
  }
  if (has_v) {
    const int u = (th >> 5) & 3, h = (th >> 4) & 1, c = th & 15;
#pragma unroll
    for (int e = 0; e < 2; ++e) {  // token groups h and h + 2 of the tile
      const char* p = block + kvq_v_code(16 * u + 4 * (h + 2 * e), c * (HD / 16), HD);
      if constexpr (HD == 128) {
        const u32x4 w = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) s.v[4 * e + i] = w[i];
      } else {
        const uint2 w = *reinterpret_cast<const uint2*>(p);
        s.v[2 * e] = w.x;
        s.v[2 * e + 1] = w.y;
      }
      s.vs[e] = *reinterpret_cast<const uint32_t*>(block + kvq_v_scale(16 * u + 4 * (h + 2 * e), c * (HD / 16) / kKvqBlock, HD));
    }
  }
  s.all = *(reinterpret_cast<const uint32_t*>(block + 66 * HD) + (threadIdx.x & (HD / 2 - 1)));
}

// NaN scales as 2^-127, which a zero probability clears.
__device__ __forceinline__ uint32_t without_nan(uint32_t s) {
#pragma unroll
  for (int r = 0; r < 4; ++r)
    if (((s >> (8 * r)) & 255u) == 255u) s &= ~(255u << (8 * r));
  return s;
}

template <int HD, bool HALF>
__device__ __forceinline__ void share_values(const PageShare<HD>& s, const uint32_t (&vs)[2], int th, u32x4* lv) {
  const int half = th >> 7, u = (th >> 5) & 3, h = (th >> 4) & 1, c = th & 15;
#pragma unroll
  for (int b = 0; b < HD / 64; ++b) {
    const int t = HD == 128 ? 2 * half + b : half;  // the tile of dimensions, and the byte of a token's that holds its two
    uint32_t x[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float sc = scale_of(vs[k >> 2], k & 3);
      if constexpr (HD == 128) {
        const uint32_t w = half ? s.v[k] >> 16 : s.v[k];
        x[k] = value_pair<HALF>(w, sc, b);
      } else {
        const uint32_t w = half ? s.v[k >> 1] >> 8 : s.v[k >> 1];
        x[k] = value_pair<HALF>(w, sc, 2 * (k & 1));
      }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      u32x4 w;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = __builtin_amdgcn_perm(x[2 * e + 1], x[2 * e], i ? 0x07060302u : 0x05040100u);
      lv[(t * 4 + u) * 64 + h * 32 + i * 16 + c] = w;
    }
  }
}

// The share into LDS; half: V in fp16.
template <int HD>
__device__ __forceinline__ void share_store(const PageShare<HD>& s, int th, bool has_k, bool has_v, int tok0, int end, bool half, u32x4* lk,
                                            u32x4* lv) {
  if (has_k) {
    const int u = th >> 6, g = (th >> 4) & 3, c = th & 15, t = 16 * u + c;
    const float sc = scale_of(s.ks, 0);
#pragma unroll
    for (int v = 0; v < HD / 32; ++v) {
      const int d8 = g * (HD / 32) + v;  // eight dimensions
      const uint32_t w = s.k[v];
      lk[((t >> 5) * (HD / 16) + (d8 >> 1)) * 64 + (d8 & 1) * 32 + (t & 31)] =
          u32x4{code_pair<0>(w, sc), code_pair<1>(w, sc), code_pair<2>(w, sc), code_pair<3>(w, sc)};
    }
  }
  if (!has_v) return;
  const int u = (th >> 5) & 3, h = (th >> 4) & 1, t = tok0 + 16 * u + 4 * h;
  uint32_t vs[2] = {s.vs[0], s.vs[1]};
  if (tok0 + kKvqPage > end) {
    vs[0] = scales_below(vs[0], t, end);
    vs[1] = scales_below(vs[1], t + 8, end);
  }
  if (half) {
    share_values<HD, true>(s, vs, th, lv);
  } else {
    vs[0] = without_nan(vs[0]);
    vs[1] = without_nan(vs[1]);
    share_values<HD, false>(s, vs, th, lv);
  }
}

// Orders the N products before it, each of one 16-byte LDS read: six reads ahead of the first, then one to each.
template <int N>
__device__ __forceinline__ void reads_ahead() {
  constexpr int A = N < 6 ? N : 6;
  __builtin_amdgcn_sched_group_barrier(0x100, A, 0);  // LDS reads
#pragma unroll
  for (int i = 0; i < N - A; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // MFMA
    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
  }
  __builtin_amdgcn_sched_group_barrier(0x008, A, 0);
}

// O^T += V^T P^T for a page: the lane's 32 probabilities x in two pieces of bf16, or w in fp16.
template <int HD, bool HALF>
__device__ __forceinline__ void page_values(const u32x4* lv, const float (&x)[32], const uint32_t (&w16)[16], f32x16 (&o)[HD / 32]) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    f16x8 ph;
    bf16x8_t pf[2];
    if constexpr (HALF) {
      ph = __builtin_bit_cast(f16x8, u32x4{w16[4 * u], w16[4 * u + 1], w16[4 * u + 2], w16[4 * u + 3]});
    } else {
      float y[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) y[k] = x[8 * u + k];
      split8<2>(y, pf);
    }
#pragma unroll
    for (int t = 0; t < HD / 32; ++t) {
      const u32x4 v = lv[(t * 4 + u) * 64 + lane];
      if constexpr (HALF) {
        o[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, v), ph, o[t], 0, 0, 0);
      } else {
        o[t] = mfma32x32x16(__builtin_bit_cast(bf16x8_t, v), pf[0], o[t]);
        o[t] = mfma32x32x16(__builtin_bit_cast(bf16x8_t, v), pf[1], o[t]);
      }
    }
  }
  if constexpr (HALF) reads_ahead<HD / 8>();
}

template <int HD, int NW>
__global__ __launch_bounds__(64 * NW, 2) void k_kvq_prompt(KvqAttendArgs a, KvqCut cut) {
  constexpr int KS = HD / 16, NT = HD / 32, STAGE = 2 * 8 * HD;  // STAGE: 16-byte pieces of a page, K and V
  static_assert(NW == 4 || NW == 8, "256 threads unpack K, 256 V");
  __shared__ __attribute__((aligned(16))) u32x4 lds[2][STAGE];
  const KvqBatch& bt = a.batch;
  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, c = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n_kv = a.cache.n_kv, G = a.n_q / n_kv;
  const int index = blockIdx.x / n_kv, kh = blockIdx.x - index * n_kv, split = blockIdx.z;
  int tile = 0;
  KvqSeq sq;
  const int b = find_longest(bt, G, cut, index, tile, sq);
  if (b < 0) return;
  const KvqTile tl = kvq_tile(sq, G, tile, cut.cols);
  const int j0 = tile * cut.cols, first = tl.first;
  const int pages = kvq_pages(tl.end), items = kvq_items(pages, cut.items, cut.least);
  if (split >= items) return;
  const int per_item = kvq_item_pages(pages, items), p0 = split * per_item;
  const int np = max(0, min(per_item, pages - p0));

  // The column, its query, and the last key that it sees; columns past the tile's last repeat that.
  const int col = wave * 32 + c, cc = min(col, tl.cols - 1);
  const int row = (j0 + cc) / G, head = kh * G + (j0 + cc) - row * G;
  const int lim = sq.ok ? first + row : -1;
  const int w0 = min(wave * 32, tl.cols - 1), w1 = min(wave * 32 + 31, tl.cols - 1);
  const int open = first + (j0 + w0) / G + 1;                                       // keys that every column of the wave sees
  const int wave_end = wave * 32 < tl.cols && sq.ok ? first + (j0 + w1) / G + 1 : 0;  // that some column of it does
  const float scale_log2 = a.scale * kLog2e;
  bf16x8_t qf[KS];
  {
    const bf16_t* q = static_cast<const bf16_t*>(a.q.p) + (sq.r0 + row) * a.q.row_stride + head * a.q.head_stride + 8 * h;
    if (a.q.vec) {
#pragma unroll
      for (int j = 0; j < KS; ++j) qf[j] = load_bf16x8(q + 16 * j);
    } else {
#pragma unroll
      for (int j = 0; j < KS; ++j) {
        u32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          w[i] = static_cast<uint32_t>(q[16 * j + 2 * i]) | static_cast<uint32_t>(q[16 * j + 2 * i + 1]) << 16;
        qf[j] = __builtin_bit_cast(bf16x8_t, w);
      }
    }
  }
  f32x16 o[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[t][r] = 0.f;
  Softmax st;

  if (np > 0) {
    const int32_t* pt = table_of(bt, b) + p0;
    const size_t bytes = kvq_block_bytes(HD);
    const char* base = a.cache.blocks + kh * bytes;
    auto block_of = [&](int id, bool& lost) {  // page 0 stands in for an id outside the cache
      lost = !kvq_page_ok(a.cache, id);
      return base + static_cast<size_t>(lost ? 0 : id) * n_kv * bytes;
    };
    auto id_of = [&](int p) { return __builtin_amdgcn_readfirstlane(pt[min(p, np - 1)]); };
    // The end of the keys of page p0 + p, whose share is s: none where another page stands in.
    auto held = [&](const PageShare<HD>& s, int p) { return s.lost ? (p0 + p) * kKvqPage : tl.end; };
    // Whether page p0 + p, whose share is s, has values that fp16 holds: the same in every wave.
    auto fits = [&](const PageShare<HD>& s, int p) {
      const int i = lane & (HD / 2 - 1), t = 16 * (i & 3) + 4 * ((i >> 2) & 3), tok0 = (p0 + p) * kKvqPage, end = held(s, p);
      const uint32_t w = tok0 + kKvqPage > end ? scales_below(s.all, tok0 + t, end) : s.all;
      return static_cast<bool>(__all((((w + 0x18181818u) ^ 0x80808080u) & 0xe0e0e0e0u) == 0));
    };
    PageShare<HD> share;
    const int th = tid & 255;
    const bool has_k = NW == 4 || wave < 4, has_v = NW == 4 || wave >= 4;
    int id = id_of(1);
    share_load<HD>(share, block_of(id_of(0), share.lost), th, has_k, has_v);
    bool half = fits(share, 0), lost = share.lost;
    share_store<HD>(share, th, has_k, has_v, p0 * kKvqPage, held(share, 0), half, lds[0], lds[0] + 8 * HD);
    share_load<HD>(share, block_of(id, share.lost), th, has_k, has_v);
    id = id_of(2);
    auto rescale = [&](float alpha) {
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[t][r] *= alpha;
    };
    int p = 0;
    // Pages from p on.  HALF: V and P in fp16, up to the first page that does not fit; else in bf16.
    auto walk = [&](auto half_tag) {
      constexpr bool HALF = half_tag.value;
      for (; p < np && (!HALF || half); ++p) {
        __syncthreads();  // page p is in its stage, and nobody reads the other one
        const u32x4* lk = lds[p & 1];
        const u32x4* lv = lk + 8 * HD;
        const bool lost_now = lost;
        if (p + 1 < np) {
          half = HALF && fits(share, p + 1);
          lost = share.lost;
          share_store<HD>(share, th, has_k, has_v, (p0 + p + 1) * kKvqPage, held(share, p + 1), half, lds[(p + 1) & 1], lds[(p + 1) & 1] + 8 * HD);
          share_load<HD>(share, block_of(id, share.lost), th, has_k, has_v);
          id = id_of(p + 3);
        }
        const int tok0 = (p0 + p) * kKvqPage;
        if (tok0 >= wave_end) continue;
        f32x16 s[2];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int r = 0; r < 16; ++r) s[t][r] = 0.f;
#pragma unroll
        for (int j = 0; j < KS; ++j)
#pragma unroll
          for (int t = 0; t < 2; ++t) s[t] = mfma32x32x16(__builtin_bit_cast(bf16x8_t, lk[(t * KS + j) * 64 + lane]), qf[j], s[t]);
        reads_ahead<2 * KS>();
        if (lost_now || tok0 + kKvqPage > open) {
          asm volatile("");  // a branch: as selects it would cost every page
#pragma unroll
          for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              const float v = lost_now ? __builtin_nanf("") : s[t][r];
              s[t][r] = tok0 + 32 * t + 8 * (r >> 2) + 4 * h + (r & 3) > lim ? -INFINITY : v;
            }
        }
        float x[32];
        uint32_t w[16];
#pragma unroll
        for (int k = 0; k < 32; ++k) x[k] = s[k >> 4][k & 15];
        softmax_page<HALF>(st, x, w, scale_log2, rescale, [&](const uint32_t (&small)[16]) {
          if constexpr (HALF) page_values<HD, true>(lv, x, small, o);
        }, 32);
        if (!HALF) {  // NaN value blocks: the outputs that lie in one turn NaN if the column sees the token
          bool ig;
          const char* block = block_of(__builtin_amdgcn_readfirstlane(pt[p]), ig);
#pragma unroll
          for (int i = 0; i < 2; ++i) {  // rows 8 i + .. of each 16 are dimensions of this block
            bool bad = false;
            for (int t = 0; t < kKvqPage; ++t)
              bad |= tok0 + t <= lim && static_cast<unsigned char>(block[kvq_v_scale(t, HD == 128 ? h + 2 * i : i, HD)]) == 255;
            if (bad) {
#pragma unroll
              for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                  if (((r >> 2) & 1) == i) o[t][r] += __builtin_nanf("");
            }
          }
        }
        page_values<HD, HALF>(lv, x, w, o);
      }
    };
    walk(std::true_type{});
    if (p < np) {
      leave_half(st, rescale);
      walk(std::false_type{});
    }
    st.l += __shfl_xor(st.l, 32, 64);
  }

  if (col >= tl.cols) return;
  // The lane's rows 8 i + 4 h + e of each tile: dimensions hd/16 c' + 2 t + (row >= 16), c' = row mod 16.
  const float inv = !sq.ok ? __builtin_nanf("") : lim < 0 ? 0.f : 1.f / st.l;
  const int64_t part = (static_cast<int64_t>(index) * cut.items + split) * n_kv + kh;
#pragma unroll
  for (int q = 0; q < 2; ++q)
#pragma unroll
    for (int e = 0; e < 4; e += 8 / (HD / 16)) {  // eight dimensions: of one c' at hd 128, of two at 64
      const int cp = 8 * q + 4 * h + e;
      float x[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int t = HD == 128 ? k >> 1 : (k >> 1) & 1, i = k & 1, ee = HD == 128 ? e : e + (k >> 2);
        x[k] = o[t][8 * i + 4 * q + ee];
      }
      if (items == 1) {
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] *= inv;
        store8<true>(a.out, sq.r0 + row, head, cp * (HD / 16), x);
      } else {
        float* po = a.part_o + (part * cut.cols + col) * HD + cp * (HD / 16);
        *reinterpret_cast<f32x4_t*>(po) = f32x4_t{x[0], x[1], x[2], x[3]};
        *reinterpret_cast<f32x4_t*>(po + 4) = f32x4_t{x[4], x[5], x[6], x[7]};
      }
    }
  if (items > 1 && h == 0) {
    float* ml = a.part_ml + part * 2 * cut.cols + col;
    ml[0] = st.m;
    ml[cut.cols] = st.l;
  }
}

// Joins the items of a tile: one block per (tile, KV head, column).  Four dimensions to a thread, the items dealt out to
// groups of threads whose loads are all in flight at once: 4 us for 64 items of 7 columns and 4 KV heads, most of it the launch.
template <int HD, bool F32>
__global__ __launch_bounds__(256) void k_kvq_join(KvqAttendArgs a, KvqCut cut) {
  constexpr int LPC = HD / 4, NG = 256 / LPC, PER = kKvqTileItems / NG;
  __shared__ float sw[kKvqTileItems];
  __shared__ __attribute__((aligned(16))) f32x4_t sx[NG][LPC];
  const int n_kv = a.cache.n_kv, G = a.n_q / n_kv;
  const int kh = blockIdx.y, col = blockIdx.z;
  int tile = 0;
  KvqSeq sq;
  int b = blockIdx.x;
  if (cut.find) b = find_longest(a.batch, G, cut, blockIdx.x, tile, sq);
  else sq = kvq_seq(a.batch, b);
  if (b < 0) return;
  const KvqTile tl = kvq_tile(sq, G, tile, cut.cols);
  const int n = kvq_items(kvq_pages(tl.end), cut.items, cut.least);
  if (n == 1 || col >= tl.cols) return;  // one item has written the output itself
  const int j0 = tile * cut.cols;
  const int64_t part = static_cast<int64_t>(blockIdx.x) * cut.items * n_kv + kh;  // of item 0; n_kv between items
  const int grp = threadIdx.x / LPC, d = threadIdx.x % LPC * 4;
  const float* po = a.part_o + (part * cut.cols + col) * HD + d;
  const int64_t step = static_cast<int64_t>(n_kv) * cut.cols * HD;
  f32x4_t x[PER];
#pragma unroll
  for (int k = 0; k < PER; ++k) x[k] = *reinterpret_cast<const f32x4_t*>(po + min(grp + NG * k, n - 1) * step);
  float den = 0.f;
  if (threadIdx.x < 64) {
    const int lane = threadIdx.x;
    const float* ml = a.part_ml + (part + static_cast<int64_t>(min(lane, n - 1)) * n_kv) * 2 * cut.cols + col;
    const float m = lane < n ? ml[0] : -INFINITY, l = lane < n ? ml[cut.cols] : 0.f;
    const float mx = wave_max(m);
    const float w = m == -INFINITY ? (l == 0.f ? 0.f : 1.f) : __builtin_amdgcn_exp2f(m - mx);
    sw[lane] = w;
    den = wave_sum(w * l);
  }
  __syncthreads();
  f32x4_t sum{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int k = 0; k < PER; ++k)
    if (grp + NG * k < n) sum += x[k] * sw[grp + NG * k];
  sx[grp][threadIdx.x % LPC] = sum;
  __syncthreads();
  if (threadIdx.x < HD / 8) {
    const int r = (j0 + col) / G, h = kh * G + (j0 + col) - r * G;
    const float inv = tl.first + r < 0 ? 0.f : 1.f / den;
    f32x4_t y[2]{};
#pragma unroll
    for (int k = 0; k < NG; ++k) {
      y[0] += sx[k][2 * threadIdx.x];
      y[1] += sx[k][2 * threadIdx.x + 1];
    }
    float out[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) out[k] = y[k >> 2][k & 3] * inv;
    store8<!F32>(a.out, sq.r0 + r, h, threadIdx.x * 8, out);
  }
}

// The same for k_kvq_prompt's tiles, which have many columns and few items: HD / 4 lanes to a column.  (A block to a column, as
// above, made 29,000 blocks for a prompt of 1,024 tokens, 50 us.)
template <int HD>
__global__ __launch_bounds__(256) void k_kvq_join_prompt(KvqAttendArgs a, KvqCut cut) {
  constexpr int LPC = HD / 4, PER = kKvqTileItems / LPC;
  const int n_kv = a.cache.n_kv, G = a.n_q / n_kv;
  const int kh = blockIdx.y, d4 = threadIdx.x % LPC, col = blockIdx.z * (256 / LPC) + threadIdx.x / LPC;
  int tile = 0;
  KvqSeq sq;
  const int b = find_longest(a.batch, G, cut, blockIdx.x, tile, sq);
  if (b < 0) return;
  const KvqTile tl = kvq_tile(sq, G, tile, cut.cols);
  const int n = kvq_items(kvq_pages(tl.end), cut.items, cut.least);
  if (n == 1 || col >= tl.cols) return;  // one item has written the output itself
  const int64_t part = static_cast<int64_t>(blockIdx.x) * cut.items * n_kv + kh;  // of item 0; n_kv between items
  const float* ml = a.part_ml + part * 2 * cut.cols + col;
  float m[PER], l[PER], mx = -INFINITY, den = 0.f;
#pragma unroll
  for (int k = 0; k < PER; ++k) {  // items d4, d4 + LPC, ...
    const int i = d4 + LPC * k;
    const float* p = ml + static_cast<int64_t>(min(i, n - 1)) * n_kv * 2 * cut.cols;
    m[k] = i < n ? p[0] : -INFINITY;
    l[k] = i < n ? p[cut.cols] : 0.f;
    mx = fmaxf(mx, m[k]);
  }
#pragma unroll
  for (int x = 1; x < LPC; x *= 2) mx = fmaxf(mx, __shfl_xor(mx, x, 64));
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    m[k] = m[k] == -INFINITY ? (l[k] == 0.f ? 0.f : 1.f) : __builtin_amdgcn_exp2f(m[k] - mx);
    den += m[k] * l[k];
  }
#pragma unroll
  for (int x = 1; x < LPC; x *= 2) den += __shfl_xor(den, x, 64);
  const float* po = a.part_o + (part * cut.cols + col) * HD + 4 * d4;
  const int64_t step = static_cast<int64_t>(n_kv) * cut.cols * HD;
  f32x4_t sum{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int k = 0; k < PER; ++k)
    for (int i0 = LPC * k; i0 < min(n, LPC * (k + 1)); i0 += 4) {
      f32x4_t x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = *reinterpret_cast<const f32x4_t*>(po + min(i0 + i, n - 1) * step);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float w = __shfl(m[k], (i0 + i) % LPC, LPC);
        if (i0 + i < n) sum += x[i] * w;
      }
    }
  const int row = (tile * cut.cols + col) / G, head = kh * G + tile * cut.cols + col - row * G;
  const float inv = tl.first + row < 0 ? 0.f : 1.f / den;
  float out[8];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    out[e] = sum[e] * inv;
    out[4 + e] = __shfl_xor(out[e], 1, 64);
  }
  if (!(d4 & 1)) store8<true>(a.out, sq.r0 + row, head, 4 * d4, out);
}

template <int HD, bool F32>
hipError_t attend_launch(KvqAttendArgs a, const AttendPlan& p, float* ws, hipStream_t s) {
  const int n_kv = a.cache.n_kv;
  if (p.prompt_tiles) {
    const size_t n = part_floats(p.prompt, p.prompt_tiles, n_kv, HD);
    a.part_o = ws;
    a.part_ml = n ? ws + n : nullptr;
    ws = n ? ws + n + n / HD * 2 : ws;
    if constexpr (!F32) {
      const dim3 grid(static_cast<uint32_t>(p.prompt_tiles * n_kv), 1, p.prompt.items);
      if (p.prompt_waves == 4) launch_kernel((k_kvq_prompt<HD, 4>), grid, dim3(256), 0, s, a, p.prompt);
      else if constexpr (HD == 128) launch_kernel((k_kvq_prompt<HD, 8>), grid, dim3(512), 0, s, a, p.prompt);
      else return hipErrorInvalidValue;
      constexpr int kCols = 1024 / HD;  // of a block of k_kvq_join_prompt
      if (n) launch_kernel((k_kvq_join_prompt<HD>), dim3(static_cast<uint32_t>(p.prompt_tiles), n_kv, p.prompt.cols / kCols), dim3(256), 0, s, a, p.prompt);
    }
  }
  if (p.walk_tiles) {
    const size_t n = part_floats(p.walk, p.walk_tiles, n_kv, HD);
    a.part_o = ws;
    a.part_ml = n ? ws + n : nullptr;
    const dim3 grid(static_cast<uint32_t>(p.walk.find ? p.walk_tiles * n_kv : p.walk_tiles), p.walk.find ? 1 : n_kv, p.walk.items);
    switch (p.waves) {
      case 1: launch_kernel((k_kvq_attend<HD, F32, 1>), grid, dim3(64), 0, s, a, p.walk); break;
      case 4: launch_kernel((k_kvq_attend<HD, F32, 4>), grid, dim3(256), 0, s, a, p.walk); break;
      case 8: launch_kernel((k_kvq_attend<HD, F32, 8>), grid, dim3(512), 0, s, a, p.walk); break;
      default: return hipErrorInvalidValue;
    }
    const int64_t most = std::min<int64_t>(p.walk.upto, static_cast<int64_t>(kvq_max_rows(a.batch)) * (a.n_q / n_kv));
    if (n) launch_kernel((k_kvq_join<HD, F32>), dim3(static_cast<uint32_t>(p.walk_tiles), n_kv, static_cast<uint32_t>(std::min<int64_t>(p.walk.cols, most))), dim3(256), 0, s, a, p.walk);
  }
  return hipGetLastError();
}

// Rows of a wave of the row kernels: one step, or four to as many as a wave's lanes look up, while 2,048 waves are left.
// Append and read-back of 11,511 tokens of the 7B layer: 21.0 us, with 1,024 waves 27.1, with 4,096 22.6.
int rows_per_wave(const KvqCache& c, int n_rows) {
  const int step = 512 / c.hd;
  const int64_t want = static_cast<int64_t>(n_rows) * c.n_kv / 2048;
  int r = want >= 4 * step ? 4 * step : step;
  while (r > step && r < 64 && 2 * r <= want) r *= 2;
  return r;
}
dim3 row_grid(const KvqCache& c, int n_rows, int rows) {
  const int64_t waves = (static_cast<int64_t>(n_rows) + rows - 1) / rows * c.n_kv;
  return dim3(static_cast<uint32_t>((waves + 3) / 4));
}

}  // namespace

template <int HD>
static hipError_t rope_append_hd(const KvqCache& c, const RopeArgs& a, hipStream_t s) {
  const int64_t units = static_cast<int64_t>(a.n_q + a.n_kv) * (HD / 16) + static_cast<int64_t>(a.n_kv) * (HD / 8);
  const dim3 grid(static_cast<uint32_t>((a.M * units + 255) / 256));
  switch (a.splits) {
#define RP_ROPE(S) case S: launch_kernel((k_kvq_rope_append<HD, S>), grid, dim3(256), 0, s, c, a); break;
    RP_ROPE(1) RP_ROPE(2) RP_ROPE(3) RP_ROPE(4) RP_ROPE(5) RP_ROPE(6) RP_ROPE(7) RP_ROPE(8)
    RP_ROPE(9) RP_ROPE(10) RP_ROPE(11) RP_ROPE(12) RP_ROPE(13) RP_ROPE(14) RP_ROPE(15) RP_ROPE(16)
#undef RP_ROPE
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

hipError_t launch_kvq_rope_append(const KvqCache& c, const RopeArgs& a, hipStream_t s) {
  if (a.M <= 0) return hipSuccess;
  return c.hd == 128 ? rope_append_hd<128>(c, a, s) : rope_append_hd<64>(c, a, s);
}

hipError_t launch_kvq_append(const KvqCache& c, const KvqBatch& b, const KvqTensor& k, const KvqTensor& v, hipStream_t s) {
  const int rows = rows_per_wave(c, b.n_rows);
  const dim3 grid = row_grid(c, b.n_rows, rows), block(256);
#define RP_ROWS(HD, BF16)                                                                                    \
  if (c.hd == HD && static_cast<bool>(k.bf16) == BF16) {                                                     \
    if (rows == 512 / HD) launch_kernel((k_kvq_append<HD, BF16, 1>), grid, block, 0, s, c, b, k, v, rows);   \
    else launch_kernel((k_kvq_append<HD, BF16, 4>), grid, block, 0, s, c, b, k, v, rows);                    \
  }
  RP_ROWS(128, true) RP_ROWS(128, false) RP_ROWS(64, true) RP_ROWS(64, false)
#undef RP_ROWS
  return hipGetLastError();
}

hipError_t launch_kvq_read(const KvqCache& c, const KvqBatch& b, const KvqTensor& k, const KvqTensor& v, hipStream_t s) {
  const int rows = rows_per_wave(c, b.n_rows);
  const dim3 grid = row_grid(c, b.n_rows, rows), block(256);
#define RP_ROWS(HD, BF16)                                                                                    \
  if (c.hd == HD && static_cast<bool>(k.bf16) == BF16) {                                                     \
    if (rows == 512 / HD) launch_kernel((k_kvq_read<HD, BF16, 1>), grid, block, 0, s, c, b, k, v, rows);   \
    else launch_kernel((k_kvq_read<HD, BF16, 4>), grid, block, 0, s, c, b, k, v, rows);                    \
  }
  RP_ROWS(128, true) RP_ROWS(128, false) RP_ROWS(64, true) RP_ROWS(64, false)
#undef RP_ROWS
  return hipGetLastError();
}

hipError_t launch_kvq_attend(const KvqAttendArgs& a, void* ws, hipStream_t s) {
  const AttendPlan p = attend_plan(a.cache, a.batch, a.n_q, a.q.bf16);
  float* w = static_cast<float*>(ws);
  if (a.q.bf16) return a.cache.hd == 128 ? attend_launch<128, false>(a, p, w, s) : attend_launch<64, false>(a, p, w, s);
  return a.cache.hd == 128 ? attend_launch<128, true>(a, p, w, s) : attend_launch<64, true>(a, p, w, s);
}

}  // namespace rollpack
