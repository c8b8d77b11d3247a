// The KV cache held in 4 bits (kvq.hpp has its format): quantising rows into it, reading them back, and
// causal GQA attention over it.
#include <type_traits>

#include "device_common.hpp"
#include "kernels.hpp"
#include "kvq.hpp"

namespace rollpack {

namespace {

constexpr float kLog2e = 1.4426950408889634f;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// ---- the batch -----------------------------------------------------------------------

__device__ __forceinline__ const int32_t* table_of(const KvqBatch& bt, int b) {
  return bt.page_table + static_cast<int64_t>(bt.table_row ? bt.table_row[b] : b) * bt.table_stride;
}

// The sequence that row `row` belongs to, -1 for rows behind the last one: the last whose first row is not past it.
// The wave counts 64 offsets at a time, four rows (one per 16 lanes) at once.
__device__ __forceinline__ int seq_of_row(const KvqBatch& bt, int row) {
  if (!bt.row_off) return row < min(bt.n_seqs, bt.n_rows) ? row : -1;
  const int lane = threadIdx.x & 63;
  int cnt[4] = {0, 0, 0, 0};
  for (int o = 0; o <= bt.n_seqs; o += 64) {
    const int v = o + lane <= bt.n_seqs ? bt.row_off[o + lane] : 0x7fffffff;
#pragma unroll
    for (int k = 0; k < 4; ++k) cnt[k] += __popcll(__ballot(v <= __builtin_amdgcn_readlane(row, 16 * k)));
  }
  const int k = lane >> 4;
  const int c = k == 0 ? cnt[0] : k == 1 ? cnt[1] : k == 2 ? cnt[2] : cnt[3];
  return c > bt.n_seqs ? -1 : c - 1;  // every offset is <= row: behind the last sequence
}

// ---- append and read -----------------------------------------------------------------
//
// A lane has eight consecutive dimensions of one row and KV head, K and V: 16 bytes of bf16 in, one word of
// codes out.  hd / 8 lanes have a row, and a wave takes consecutive rows of one head (four at hd 128, eight at 64),
// so that the runs it writes are whole 64-byte pieces: the layout keeps four consecutive tokens side by side.

struct RowPlace {
  int row, d, kh, state;  // state: 0 nothing to do, 1 a position of the cache, 2 before the sequence's first token, 3 bad
  int t;                  // place in the page
  char* block;
};

template <int HD>
__device__ __forceinline__ RowPlace row_place(const KvqCache& c, const KvqBatch& bt) {
  constexpr int LPR = HD / 8, RPW = 64 / LPR;  // lanes per row, rows per wave
  const int lane = threadIdx.x & 63;
  const int wave = blockIdx.x * (blockDim.x / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  RowPlace p;
  const int g = wave / c.n_kv;  // group of RPW rows
  p.kh = wave - g * c.n_kv;
  p.row = g * RPW + lane / LPR;
  p.d = lane % LPR * 8;
  p.state = 0;
  p.t = 0;
  p.block = c.blocks;
  int b;
  if (RPW == 4 || !bt.row_off) {
    b = seq_of_row(bt, p.row);
  } else {  // eight rows: the even ones of each 16 lanes' two, then the odd ones
    const int even = seq_of_row(bt, p.row & ~1), odd = seq_of_row(bt, p.row | 1);
    b = p.row & 1 ? odd : even;
  }
  if (b < 0 || p.row >= bt.n_rows) return p;
  const KvqSeq s = kvq_seq(bt, b);
  const int i = p.row - s.r0, pos = s.ctx - s.n + i;
  if (i < 0 || i >= s.n) return p;  // offsets that do not ascend
  if (!s.ok) {
    p.state = 3;
  } else if (pos < 0) {
    p.state = 2;
  } else {
    const int pg = table_of(bt, b)[pos / kKvqPage];
    p.state = kvq_page_ok(c, pg) ? 1 : 3;
    p.t = pos % kKvqPage;
    p.block += (static_cast<size_t>(p.state == 1 ? pg : 0) * c.n_kv + p.kh) * kvq_block_bytes(HD);
  }
  return p;
}

__device__ __forceinline__ void load8(const KvqTensor& x, int row, int head, int d, float (&f)[8]) {
  const int64_t at = row * x.row_stride + head * x.head_stride + d;
  if (x.bf16) {
    const bf16_t* p = static_cast<const bf16_t*>(x.p) + at;
    if (x.vec) {
      const u32x4 w = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = bf16_to_f32(static_cast<bf16_t>(w[i / 2] >> (16 * (i & 1))));
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = bf16_to_f32(p[i]);
    }
  } else {
    const float* p = static_cast<const float*>(x.p) + at;
    if (x.vec) {
      const f32x4_t a = *reinterpret_cast<const f32x4_t*>(p), b = *reinterpret_cast<const f32x4_t*>(p + 4);
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = i < 4 ? a[i] : b[i - 4];
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = p[i];
    }
  }
}

__device__ __forceinline__ void store8(const KvqTensor& x, int row, int head, int d, const float (&f)[8]) {
  const int64_t at = row * x.row_stride + head * x.head_stride + d;
  if (x.bf16) {
    bf16_t* p = static_cast<bf16_t*>(x.p) + at;
    if (x.vec) {
      u32x4 w;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        w[i] = static_cast<uint32_t>(f32_to_bf16(f[2 * i])) | static_cast<uint32_t>(f32_to_bf16(f[2 * i + 1])) << 16;
      *reinterpret_cast<u32x4*>(p) = w;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) p[i] = f32_to_bf16(f[i]);
    }
  } else {
    float* p = static_cast<float*>(x.p) + at;
    if (x.vec) {
      *reinterpret_cast<f32x4_t*>(p) = f32x4_t{f[0], f[1], f[2], f[3]};
      *reinterpret_cast<f32x4_t*>(p + 4) = f32x4_t{f[4], f[5], f[6], f[7]};
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) p[i] = f[i];
    }
  }
}

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

// The two values of byte I of a word of codes, packed bf16 (exact).
template <int I>
__device__ __forceinline__ uint32_t code_pair(uint32_t w, float s) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, I));
}

__device__ __forceinline__ void dequantise8(uint32_t w, uint32_t byte, float (&f)[8]) {
  const float s = __uint_as_float(byte << 23);  // 255: the conversion gives NaN
  const uint32_t p[4] = {code_pair<0>(w, s), code_pair<1>(w, s), code_pair<2>(w, s), code_pair<3>(w, s)};
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(i & 1 ? p[i / 2] & 0xffff0000u : p[i / 2] << 16);
}

// Eight consecutive dimensions d.. of token t, as they lie in a block: one word at hd 128; for V at hd 64 two halves of one.
template <int HD>
__global__ __launch_bounds__(256) void k_kvq_append(KvqCache c, KvqBatch bt, KvqTensor k, KvqTensor v) {
  const RowPlace p = row_place<HD>(c, bt);
  float kf[8] = {}, vf[8] = {};
  if (p.state == 1) {
    load8(k, p.row, p.kh, p.d, kf);
    load8(v, p.row, p.kh, p.d, vf);
  }
  uint32_t kb, vb;
  const uint32_t kw = quantise8(kf, kb), vw = quantise8(vf, vb);  // every lane: the maxima cross lanes
  if (p.state != 1) return;
  *reinterpret_cast<uint32_t*>(p.block + kvq_k_code(p.t, p.d, HD)) = kw;
  if constexpr (HD == 128) {
    *reinterpret_cast<uint32_t*>(p.block + kvq_v_code(p.t, p.d, HD)) = vw;
  } else {
    *reinterpret_cast<uint16_t*>(p.block + kvq_v_code(p.t, p.d, HD)) = static_cast<uint16_t>(vw);
    *reinterpret_cast<uint16_t*>(p.block + kvq_v_code(p.t, p.d + 4, HD)) = static_cast<uint16_t>(vw >> 16);
  }
  if (p.d % kKvqBlock == 0) {
    p.block[kvq_k_scale(p.t, p.d / kKvqBlock, HD)] = static_cast<char>(kb);
    p.block[kvq_v_scale(p.t, p.d / kKvqBlock, HD)] = static_cast<char>(vb);
  }
}

template <int HD>
__global__ __launch_bounds__(256) void k_kvq_read(KvqCache c, KvqBatch bt, KvqTensor k, KvqTensor v) {
  const RowPlace p = row_place<HD>(c, bt);
  if (p.state == 0) return;
  float kf[8], vf[8];
  if (p.state == 1) {
    const unsigned char* u = reinterpret_cast<const unsigned char*>(p.block);
    const uint32_t kw = *reinterpret_cast<const uint32_t*>(u + kvq_k_code(p.t, p.d, HD));
    uint32_t vw;
    if constexpr (HD == 128) {
      vw = *reinterpret_cast<const uint32_t*>(u + kvq_v_code(p.t, p.d, HD));
    } else {
      vw = *reinterpret_cast<const uint16_t*>(u + kvq_v_code(p.t, p.d, HD)) |
           static_cast<uint32_t>(*reinterpret_cast<const uint16_t*>(u + kvq_v_code(p.t, p.d + 4, HD))) << 16;
    }
    dequantise8(kw, u[kvq_k_scale(p.t, p.d / kKvqBlock, HD)], kf);
    dequantise8(vw, u[kvq_v_scale(p.t, p.d / kKvqBlock, HD)], vf);
  } else {
    const float x = p.state == 2 ? 0.f : __builtin_nanf("");
#pragma unroll
    for (int i = 0; i < 8; ++i) kf[i] = vf[i] = x;
  }
  store8(k, p.row, p.kh, p.d, kf);
  store8(v, p.row, p.kh, p.d, vf);
}

// ---- the plan, computed by every wave for itself ---------------------------------------

struct PlanShape {
  int cols;                           // columns of a tile
  float page_us, ends_us, join_us;    // kvq_price
};

// Where an index falls: the sequence, the tiles and items before it (of one KV head), and what is left of the index.
struct Found {
  int b, tile0, item0, rest, ppi;
  KvqSeq s;
};

// Finds item `index` (by_tile: tile `index`) of the batch; b = -1 past the last.  Lanes take 64 sequences at a time.
__device__ Found plan_find(const KvqBatch& bt, int n_kv, int group, const PlanShape& sh, int index, bool by_tile) {
  const int lane = threadIdx.x & 63;
  KvqPlanInput in;
  int64_t tp = 0;
  int tiles = 0, mp = 0;
  for (int o = 0; o < bt.n_seqs; o += 64) {
    if (o + lane < bt.n_seqs) {
      const KvqSeq s = kvq_seq(bt, o + lane);
      const int t = kvq_tiles(s, group, sh.cols), p = t ? kvq_pages(s) : 0;
      tp += static_cast<int64_t>(t) * p;
      tiles += t;
      mp = max(mp, p);
    }
  }
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) {
    tp += __shfl_xor(static_cast<long long>(tp), m, 64);
    tiles += __shfl_xor(tiles, m, 64);
    mp = max(mp, __shfl_xor(mp, m, 64));
  }
  in.tile_pages = tp;
  in.tiles = tiles;
  in.max_pages = mp;
  const int least = kvq_least_ppi(in, n_kv), most = max(1, mp);
  int ppi = most;
  if (least < most) {
    const float l2 = log2f(static_cast<float>(most) / least);
    int cand = min(most, static_cast<int>(least * exp2f(l2 * lane * (1.f / 63.f)) + 0.5f));
    if (lane == 63) cand = most;
    const float us = kvq_price(in, n_kv, cand, sh.page_us, sh.ends_us, sh.join_us);
    float best = us;
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) best = fminf(best, __shfl_xor(best, m, 64));
    const int who = 63 - __clzll(__ballot(us == best));  // the largest of the cheapest
    ppi = __builtin_amdgcn_readlane(cand, who);
  }
  Found f;
  f.b = -1;
  f.ppi = ppi;
  f.tile0 = f.item0 = f.rest = 0;
  f.s = KvqSeq{0, 0, 0, false};
  int tile_base = 0, item_base = 0;
  for (int o = 0; o < bt.n_seqs; o += 64) {
    KvqSeq s{0, 0, 0, false};
    int t = 0, it = 0;
    if (o + lane < bt.n_seqs) {
      s = kvq_seq(bt, o + lane);
      t = kvq_tiles(s, group, sh.cols);
      it = t * kvq_items(kvq_pages(s), ppi);
    }
    int ts = t, is = it;  // inclusive sums
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
      const int a = __shfl_up(ts, m, 64), c = __shfl_up(is, m, 64);
      if (lane >= m) {
        ts += a;
        is += c;
      }
    }
    const int mine = by_tile ? tile_base + ts : item_base + is;
    const uint64_t past = __ballot(mine > index);
    if (past) {
      const int w = __ffsll(static_cast<unsigned long long>(past)) - 1;
      f.b = o + w;
      f.tile0 = tile_base + __builtin_amdgcn_readlane(ts - t, w);
      f.item0 = item_base + __builtin_amdgcn_readlane(is - it, w);
      f.rest = index - (by_tile ? f.tile0 : f.item0);
      f.s.r0 = __builtin_amdgcn_readlane(s.r0, w);
      f.s.n = __builtin_amdgcn_readlane(s.n, w);
      f.s.ctx = __builtin_amdgcn_readlane(s.ctx, w);
      f.s.ok = __builtin_amdgcn_readlane(static_cast<int>(s.ok), w);
      return f;
    }
    tile_base += __builtin_amdgcn_readlane(ts, 63);
    item_base += __builtin_amdgcn_readlane(is, 63);
  }
  return f;
}

// ---- attention, 16 columns a block ------------------------------------------------------

// Two fp32 to packed bf16, round to nearest even.
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
}

// N bf16 pieces whose sum is x to 8 N bits: each is the rounded rest.
template <int N>
__device__ __forceinline__ void split8(float (&x)[8], bf16x8_t (&out)[N]) {
#pragma unroll
  for (int n = 0; n < N; ++n) {
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w[i] = pack2(x[2 * i], x[2 * i + 1]);
      if (n + 1 < N) {
        x[2 * i] -= __uint_as_float(w[i] << 16);
        x[2 * i + 1] -= __uint_as_float(w[i] & 0xffff0000u);
      }
    }
    out[n] = __builtin_bit_cast(bf16x8_t, w);
  }
}

// A page of one head as a lane holds it.
template <int HD>
struct PageRegs {
  u32x4 k[HD / 32], v[HD / 32], vs;
  uint32_t ks;
  __device__ __forceinline__ void load(const char* block) {
    const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
    const u32x4* p = reinterpret_cast<const u32x4*>(block) + lane;
#pragma unroll
    for (int i = 0; i < HD / 32; ++i) k[i] = __builtin_nontemporal_load(p + 64 * i);
    ks = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(block + 64 * HD) + (g * HD / 128) * 16 + c);
#pragma unroll
    for (int i = 0; i < HD / 32; ++i) v[i] = __builtin_nontemporal_load(p + 2 * HD + 64 * i);
    vs = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(block + 66 * HD) + (c * HD / 512) * 4 + g);
  }
};

__device__ __forceinline__ float scale_of(uint32_t word, int byte) {
  return __uint_as_float(((word >> (8 * byte)) & 255u) << 23);
}

// S^T of tile u: rows are the tile's tokens, columns the 16 columns; NQ pieces of the query.
template <int HD, int NQ>
__device__ __forceinline__ f32x4_t tile_scores(const PageRegs<HD>& pg, int u, const bf16x8_t (&qf)[HD / 32][NQ]) {
  f32x4_t acc{0.f, 0.f, 0.f, 0.f};
  const float s = scale_of(pg.ks, u);
#pragma unroll
  for (int j = 0; j < HD / 32; ++j) {
    const uint32_t w = HD == 128 ? pg.k[u][j] : pg.k[u >> 1][2 * (u & 1) + j];
    const bf16x8_t kf = __builtin_bit_cast(bf16x8_t, u32x4{code_pair<0>(w, s), code_pair<1>(w, s), code_pair<2>(w, s), code_pair<3>(w, s)});
#pragma unroll
    for (int n = 0; n < NQ; ++n) acc = mfma16x16x32(kf, qf[j][n], acc);
  }
  return acc;
}

// O^T += V^T P^T over tokens 32h .. 32h + 31 of the page: accumulator i's rows are dimensions hd/16 c + i.
template <int HD, int NP>
__device__ __forceinline__ void half_values(const PageRegs<HD>& pg, int h, const bf16x8_t (&pf)[NP], f32x4_t (&o)[HD / 16]) {
  uint32_t x[HD / 32][8];  // [dimension pair][token]: two dimensions of a token
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const float s = scale_of(pg.vs[2 * h + (k >> 2)], k & 3);
    if constexpr (HD == 128) {
      const uint32_t w = pg.v[2 * h + (k >> 2)][k & 3];
      x[0][k] = code_pair<0>(w, s);
      x[1][k] = code_pair<1>(w, s);
      x[2][k] = code_pair<2>(w, s);
      x[3][k] = code_pair<3>(w, s);
    } else {
      const uint32_t w = pg.v[h][k >> 1];
      x[0][k] = k & 1 ? code_pair<2>(w, s) : code_pair<0>(w, s);
      x[1][k] = k & 1 ? code_pair<3>(w, s) : code_pair<1>(w, s);
    }
  }
#pragma unroll
  for (int i = 0; i < HD / 16; ++i) {  // eight tokens of one dimension: the low or high halves of neighbouring tokens' pairs
    u32x4 w;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      w[e] = __builtin_amdgcn_perm(x[i / 2][2 * e + 1], x[i / 2][2 * e], i & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
    for (int n = 0; n < NP; ++n) o[i] = mfma16x16x32(__builtin_bit_cast(bf16x8_t, w), pf[n], o[i]);
  }
}

// A page that holds a NaN value block (or, past the context, anything): the blocks' scales become 2^-127, which a zero
// probability clears, and the lane's outputs turn NaN if its column sees the token.  A lane's outputs all lie in one
// block of 32 dimensions.
template <int HD>
__device__ __forceinline__ void nan_values(PageRegs<HD>& pg, const char* block, int tok0, int lim, f32x4_t (&o)[HD / 16]) {
  const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
  for (int u = 0; u < 4; ++u)
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (((pg.vs[u] >> (8 * r)) & 255u) == 255u) pg.vs[u] &= ~(255u << (8 * r));
  bool bad = false;
  for (int t = 0; t < kKvqPage; ++t)
    bad |= tok0 + t <= lim && static_cast<unsigned char>(block[kvq_v_scale(t, g * HD / 128, HD)]) == 255;
  if (bad) {
#pragma unroll
    for (int i = 0; i < HD / 16; ++i) o[i] += __builtin_nanf("");
  }
}

__device__ __forceinline__ bool has_nan_scale(const u32x4& vs) {
  float top = 0.f;  // scales are positive: of valid blocks at most 2^125, of NaN blocks infinity
#pragma unroll
  for (int u = 0; u < 4; ++u)
#pragma unroll
    for (int r = 0; r < 4; ++r) top = fmaxf(top, scale_of(vs[u], r));
  return top > 8.5e37f;
}

// One block of NW waves takes an item: 16 columns of a sequence and KV head (a column is a query head of a row, the
// G heads of a row side by side) over a range of pages, which the waves take in turn.  Per page a wave forms
// S^T = K Q^T, an online softmax in the log2 domain and O^T += V^T P^T with MFMA, straight from registers: no
// value of the cache is used by more than one wave, so nothing passes through LDS but the waves' results.
//   Q and P are operands in bf16.  fp32 queries are three bf16 pieces (24 bits), and so are their probabilities; of
// bf16 queries the probabilities are two pieces, so that the output's own rounding is the only one that counts.
//   The running maximum moves only when a score passes it by more than 2^8: probabilities up to 256 lose nothing in
// fp32 or bf16, and the outputs need rescaling a few times per item instead of every page.
template <int HD, int NQ, int NP, int NW>
__global__ __launch_bounds__(64 * NW, 2) void k_kvq_attend(KvqAttendArgs a, PlanShape sh) {
  constexpr int NT = HD / 16, OLD = HD + 4;
  __shared__ __attribute__((aligned(16))) float so[NW][16 * OLD];
  __shared__ float sm[NW][16], sl[NW][16];
  const KvqBatch& bt = a.batch;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 4, c = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n_kv = a.cache.n_kv, G = a.n_q / n_kv;
  const int item = blockIdx.x / n_kv, kh = blockIdx.x - item * n_kv;
  const Found f = plan_find(bt, n_kv, G, sh, item, false);
  if (f.b < 0) return;
  const int n_pages = kvq_pages(f.s), splits = kvq_items(n_pages, f.ppi);
  const int tile = f.rest / splits, split = f.rest - tile * splits;
  const int j0 = tile * 16, n_cols = min(16, f.s.n * G - j0);
  const int first = f.s.ctx - f.s.n;  // position of the sequence's first row
  const int end = f.s.ok ? max(0, first + (j0 + n_cols - 1) / G + 1) : 0;  // keys that the tile sees
  const int p0 = split * f.ppi, p1 = min(p0 + f.ppi, (end + kKvqPage - 1) / kKvqPage);
  const int np = max(0, p1 - p0);
  const int nw = np > wave ? (np - wave + NW - 1) / NW : 0;  // this wave's pages: wave, wave + NW, ...
  const int open = first + j0 / G + 1;  // keys that every column sees

  // The column: its query, and the last key that it sees.
  const int cc = min(c, n_cols - 1), row = (j0 + cc) / G, head = kh * G + (j0 + cc) - row * G;
  const int lim = f.s.ok ? first + row : -1;
  const float scale_log2 = a.scale * kLog2e;

  const int32_t* pt = table_of(bt, f.b);
  const int ptv = lane < np ? pt[p0 + lane] : 0;  // lane i has page i of the item, the first 64
  const size_t bytes = kvq_block_bytes(HD);
  PageRegs<HD> pg[2];
  const char* at[2];
  bool lost[2];
  auto load = [&](int sl, int i) {
    const int q = min(wave + NW * i, max(np - 1, 0));  // past the last page: the last again
    int id = q < 64 ? __builtin_amdgcn_readlane(ptv, q) : pt[p0 + q];
    lost[sl] = !kvq_page_ok(a.cache, id);
    id = lost[sl] ? 0 : id;
    at[sl] = a.cache.blocks + (static_cast<size_t>(id) * n_kv + kh) * bytes;
    pg[sl].load(at[sl]);
  };
  f32x4_t o[NT];
#pragma unroll
  for (int i = 0; i < NT; ++i) o[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  float m_run = -INFINITY, l_run = 0.f;
  if (nw > 0) {
    bf16x8_t qf[HD / 32][NQ];
    {
      float x[HD / 32][8];
#pragma unroll
      for (int j = 0; j < HD / 32; ++j) load8(a.q, f.s.r0 + row, head, g * (HD / 4) + 8 * j, x[j]);
      load(0, 0);
      load(1, 1);
#pragma unroll
      for (int j = 0; j < HD / 32; ++j) split8<NQ>(x[j], qf[j]);
    }
    auto step = [&](int sl, int i) {
      const int tok0 = (p0 + wave + NW * i) * kKvqPage;
      float sv[16];
      float pmax = -INFINITY;
      const bool masked = tok0 + kKvqPage > open;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const f32x4_t s = tile_scores<HD, NQ>(pg[sl], u, qf);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float v = s[e];
          if (lost[sl]) v = __builtin_nanf("");
          if (masked && tok0 + 16 * u + 4 * g + e > lim) v = -INFINITY;
          sv[4 * u + e] = v;
          pmax = fmaxf(pmax, v);
        }
      }
      pmax = fmaxf(pmax, __shfl_xor(pmax, 16, 64));
      pmax = fmaxf(pmax, __shfl_xor(pmax, 32, 64));
      pmax *= scale_log2;
      if (__any(pmax > m_run + 8.f)) {
        const float m_new = pmax > m_run + 8.f ? pmax : m_run;
        const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run - m_new);
        l_run *= alpha;
        m_run = m_new;
#pragma unroll
        for (int t = 0; t < NT; ++t) o[t] *= alpha;
      }
      const float shift = m_run == -INFINITY ? 0.f : m_run;
      float sum = 0.f;
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        sv[k] = __builtin_amdgcn_exp2f(__builtin_fmaf(sv[k], scale_log2, -shift));
        sum += sv[k];
      }
      l_run += sum;  // of this lane's tokens; the lanes of a column add up at the end
      if (__any(has_nan_scale(pg[sl].vs))) nan_values<HD>(pg[sl], at[sl], tok0, lim, o);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float x[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = sv[8 * h + k];
        bf16x8_t pf[NP];
        split8<NP>(x, pf);
        half_values<HD, NP>(pg[sl], h, pf, o);
      }
    };
    for (int i = 0; i < nw; i += 2) {
      step(0, i);
      load(0, i + 2);
      if (i + 1 < nw) {
        step(1, i + 1);
        load(1, i + 3);
      }
    }
    l_run += __shfl_xor(l_run, 16, 64);
    l_run += __shfl_xor(l_run, 32, 64);
  }

  // Join the waves: one without a page has m = -inf, l = 0, o = 0.
  if (g == 0) {
    sm[wave][c] = m_run;
    sl[wave][c] = l_run;
  }
  __syncthreads();
  float mx = sm[0][c];
#pragma unroll
  for (int w = 1; w < NW; ++w) mx = fmaxf(mx, sm[w][c]);
  const float fac = m_run == -INFINITY ? (l_run == 0.f ? 0.f : 1.f) : __builtin_amdgcn_exp2f(m_run - mx);
#pragma unroll
  for (int e = 0; e < 4; ++e)
#pragma unroll
    for (int i = 0; i < NT; i += 4)  // dimensions hd/16 (4g + e) + i ..
      *reinterpret_cast<f32x4_t*>(&so[wave][c * OLD + (4 * g + e) * NT + i]) =
          f32x4_t{o[i][e], o[i + 1][e], o[i + 2][e], o[i + 3][e]} * fac;
  __syncthreads();
  const int64_t part = static_cast<int64_t>(f.item0 + f.rest) * n_kv + kh;
  for (int q = tid; q < n_cols * (HD / 8); q += 64 * NW) {
    const int col = q / (HD / 8), d = q % (HD / 8) * 8;
    float m4 = sm[0][col], den = 0.f, x[8];
#pragma unroll
    for (int w = 1; w < NW; ++w) m4 = fmaxf(m4, sm[w][col]);
#pragma unroll
    for (int w = 0; w < NW; ++w)
      den += sm[w][col] == -INFINITY ? sl[w][col] : sl[w][col] * __builtin_amdgcn_exp2f(sm[w][col] - m4);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      x[k] = so[0][col * OLD + d + k];
#pragma unroll
      for (int w = 1; w < NW; ++w) x[k] += so[w][col * OLD + d + k];
    }
    if (splits == 1) {
      const int r = (j0 + col) / G, h = kh * G + (j0 + col) - r * G;
      // a row before the sequence's first token sees no key: zeros; a sequence out of bounds: NaN
      const float inv = !f.s.ok ? __builtin_nanf("") : first + r < 0 ? 0.f : 1.f / den;
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] *= inv;
      store8(a.out, f.s.r0 + r, h, d, x);
    } else {
      float* po = a.part_o + (part * 16 + col) * HD + d;
      *reinterpret_cast<f32x4_t*>(po) = f32x4_t{x[0], x[1], x[2], x[3]};
      *reinterpret_cast<f32x4_t*>(po + 4) = f32x4_t{x[4], x[5], x[6], x[7]};
      if (d == 0) {
        a.part_ml[part * 32 + col] = m4;
        a.part_ml[part * 32 + 16 + col] = den;
      }
    }
  }
}

// Joins the items of a tile: one block per (tile, KV head), a thread per column and eight dimensions.
template <int HD>
__global__ __launch_bounds__(16 * HD / 8) void k_kvq_join(KvqAttendArgs a, PlanShape sh) {
  constexpr int NTH = 16 * HD / 8;
  __shared__ float sw[16][kKvqTileItems];
  __shared__ float sden[16];
  const int n_kv = a.cache.n_kv, G = a.n_q / n_kv;
  const int ti = blockIdx.x / n_kv, kh = blockIdx.x - ti * n_kv;
  const Found f = plan_find(a.batch, n_kv, G, sh, ti, true);
  if (f.b < 0) return;
  const int n = kvq_items(kvq_pages(f.s), f.ppi);
  if (n <= 1) return;  // written by its only item
  const int tile = f.rest, j0 = tile * 16, n_cols = min(16, f.s.n * G - j0);
  if (static_cast<int64_t>(f.item0) + (tile + 1) * n > a.items) return;  // offsets that do not ascend
  const int64_t part = (static_cast<int64_t>(f.item0) + tile * n) * n_kv + kh;  // of split 0; n_kv between splits
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int col = wave; col < n_cols; col += NTH / 64) {
    const float* ml = a.part_ml + (part + static_cast<int64_t>(min(lane, n - 1)) * n_kv) * 32 + col;
    const float m = lane < n ? ml[0] : -INFINITY, l = lane < n ? ml[16] : 0.f;
    const float mx = wave_max(m);
    const float w = m == -INFINITY ? (l == 0.f ? 0.f : 1.f) : __builtin_amdgcn_exp2f(m - mx);
    sw[col][lane] = w;
    const float den = wave_sum(w * l);
    if (lane == 0) sden[col] = den;
  }
  __syncthreads();
  const int col = threadIdx.x / (HD / 8), d = threadIdx.x % (HD / 8) * 8;
  if (col >= n_cols) return;
  const float* po = a.part_o + (part * 16 + col) * HD + d;
  const int64_t step = static_cast<int64_t>(n_kv) * 16 * HD;
  f32x4_t x0{0.f, 0.f, 0.f, 0.f}, x1 = x0;
#pragma unroll 8
  for (int s = 0; s < n; ++s) {
    x0 += *reinterpret_cast<const f32x4_t*>(po + s * step) * sw[col][s];
    x1 += *reinterpret_cast<const f32x4_t*>(po + s * step + 4) * sw[col][s];
  }
  const int r = (j0 + col) / G, h = kh * G + (j0 + col) - r * G;
  const float inv = !f.s.ok ? __builtin_nanf("") : f.s.ctx - f.s.n + r < 0 ? 0.f : 1.f / sden[col];
  float x[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) x[k] = (k < 4 ? x0[k] : x1[k - 4]) * inv;
  store8(a.out, f.s.r0 + r, h, d, x);
}

constexpr PlanShape kWalk{16, 0.4f, 2.5f, 4.5f};

template <int HD>
hipError_t attend_hd(const KvqAttendArgs& a, int64_t tiles, int64_t items, hipStream_t s) {
  const int n_kv = a.cache.n_kv;
  const dim3 grid(static_cast<uint32_t>(items * n_kv));
  if (a.q.bf16) launch_kernel((k_kvq_attend<HD, 1, 2, 4>), grid, dim3(256), 0, s, a, kWalk);
  else launch_kernel((k_kvq_attend<HD, 3, 3, 4>), grid, dim3(256), 0, s, a, kWalk);
  if (items > tiles) launch_kernel(k_kvq_join<HD>, dim3(static_cast<uint32_t>(tiles * n_kv)), dim3(16 * HD / 8), 0, s, a, kWalk);
  return hipGetLastError();
}

dim3 row_grid(const KvqCache& c, int n_rows) {
  const int64_t rpw = 512 / c.hd, waves = (n_rows + rpw - 1) / rpw * c.n_kv;
  return dim3(static_cast<uint32_t>((waves + 3) / 4));
}

}  // namespace

size_t kvq_attend_bytes(const KvqCache& c, const KvqBatch& b, int n_q) {
  const int G = n_q / c.n_kv;
  const int64_t tiles = kvq_tile_bound(b, G, 16), items = kvq_item_bound(b, c.n_kv, G, 16);
  if (items <= tiles) return 0;
  return static_cast<size_t>(items) * c.n_kv * (16 * c.hd + 32) * 4;
}

hipError_t launch_kvq_append(const KvqCache& c, const KvqBatch& b, const KvqTensor& k, const KvqTensor& v, hipStream_t s) {
  if (c.hd == 128) launch_kernel(k_kvq_append<128>, row_grid(c, b.n_rows), dim3(256), 0, s, c, b, k, v);
  else launch_kernel(k_kvq_append<64>, row_grid(c, b.n_rows), dim3(256), 0, s, c, b, k, v);
  return hipGetLastError();
}

hipError_t launch_kvq_read(const KvqCache& c, const KvqBatch& b, const KvqTensor& k, const KvqTensor& v, hipStream_t s) {
  if (c.hd == 128) launch_kernel(k_kvq_read<128>, row_grid(c, b.n_rows), dim3(256), 0, s, c, b, k, v);
  else launch_kernel(k_kvq_read<64>, row_grid(c, b.n_rows), dim3(256), 0, s, c, b, k, v);
  return hipGetLastError();
}

hipError_t launch_kvq_attend(KvqAttendArgs a, void* ws, hipStream_t s) {
  const int G = a.n_q / a.cache.n_kv;
  const int64_t tiles = kvq_tile_bound(a.batch, G, 16), items = kvq_item_bound(a.batch, a.cache.n_kv, G, 16);
  a.items = items;
  a.part_o = static_cast<float*>(ws);
  a.part_ml = a.part_o ? a.part_o + items * a.cache.n_kv * 16 * a.cache.hd : nullptr;
  return a.cache.hd == 128 ? attend_hd<128>(a, tiles, items, s) : attend_hd<64>(a, tiles, items, s);
}

}  // namespace rollpack
