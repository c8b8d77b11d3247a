// What the kernels over the 4-bit KV cache share on the device: rows and their places, strided tensors, a page as a wave's
// operands, and the page-wise softmax.
#pragma once

#include <type_traits>

#include "device_common.hpp"
#include "kvq.hpp"

namespace rollpack {

namespace {

constexpr float kLog2e = 1.4426950408889634f;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// ---- the batch -----------------------------------------------------------------------

__device__ __forceinline__ const int32_t* table_of(const KvqBatch& bt, int b) {
  return bt.page_table + static_cast<int64_t>(bt.table_row ? bt.table_row[b] : b) * bt.table_stride;
}

// ---- where a row is -------------------------------------------------------------------

struct RowPlace {
  int state, t, page;  // state: 0 nothing to do, 1 a position of the cache, 2 before the sequence's first token, 3 bad
};
struct PagePlace : RowPlace {
  int i, left;  // which of its sequence's rows; with state 1, tokens from its own to the context's end
};

template <typename Place = RowPlace>
__device__ __forceinline__ Place row_place(const KvqCache& c, const KvqBatch& bt, int row) {
  Place p{};
  if (row >= bt.n_rows) return p;
  int b = row;
  if (bt.row_off) {  // the last sequence whose first row is not past it
    int lo = 0, hi = bt.n_seqs;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (bt.row_off[mid] <= row) lo = mid; else hi = mid - 1;
    }
    b = lo;
  }
  if (b >= bt.n_seqs) return p;  // behind the last sequence
  const KvqSeq s = kvq_seq(bt, b);
  const int i = row - s.r0, pos = s.ctx - s.n + i;
  if (i < 0 || i >= s.n) return p;  // past max_rows, or offsets that do not ascend
  if (!s.ok) {
    p.state = 3;
  } else if (pos < 0) {
    p.state = 2;
  } else {
    const int id = table_of(bt, b)[pos / kKvqPage];
    p.state = kvq_page_ok(c, id) ? 1 : 3;
    p.t = pos % kKvqPage;
    p.page = p.state == 1 ? id : 0;
  }
  if constexpr (std::is_same_v<Place, PagePlace>) {
    p.i = i;
    p.left = s.ctx - pos;
  }
  return p;
}

// The sequence of a row that the whole wave looks up: the first that ends past it, 64 ends at a time; -1 if none does.
__device__ __forceinline__ int wave_find_seq(const KvqBatch& bt, int row) {
  if (!bt.row_off) return row < bt.n_seqs ? row : -1;
  const int lane = threadIdx.x & 63;
  int lo = 0, n = bt.n_seqs;
  for (;;) {
    const int step = (n + 63) >> 6, i = min((lane + 1) * step, n) - 1;
    const uint64_t past = __ballot(bt.row_off[lo + i + 1] > row);
    if (!past) return -1;
    const int w = __ffsll(static_cast<unsigned long long>(past)) - 1;
    lo += w * step;
    if (step == 1) return lo;
    n = min(step, n - w * step);
  }
}

// row_place for the wave's lanes: rows base .. base + rows - 1 (64 at most).  Offsets, contexts of up to 64 sequences from the first
// row's on are a lane's each, where the rows look theirs up: two or three reads that wait for each other in place of row_place's
// search through memory.  Up to 64 sequences are all there.
__device__ __forceinline__ PagePlace wave_places(const KvqCache& c, const KvqBatch& bt, int base, int rows) {
  const int lane = threadIdx.x & 63, row = base + lane;
  const bool mine = lane < rows;
  if (!bt.row_off) return mine ? row_place<PagePlace>(c, bt, row) : PagePlace{};
  const int lo = bt.n_seqs <= 64 ? 0 : wave_find_seq(bt, base);
  if (lo < 0) return PagePlace{};
  const int b0 = min(lo + lane, bt.n_seqs - 1), start = bt.row_off[b0];
  const KvqSeq s0 = kvq_seq(bt, b0);
  const int end = __builtin_amdgcn_readlane(bt.row_off[b0 + 1], 63);
  if (end < base + rows && lo + 63 < bt.n_seqs - 1) return mine ? row_place<PagePlace>(c, bt, row) : PagePlace{};
  int s = 0;  // the last whose first row is not past it
#pragma unroll
  for (int step = 32; step >= 1; step >>= 1)
    if (__shfl(start, s + step, 64) <= row && lo + s + step < bt.n_seqs) s += step;
  const int i = row - __shfl(s0.r0, s, 64), n = __shfl(s0.n, s, 64), ctx = __shfl(s0.ctx, s, 64);
  const bool ok = __shfl(static_cast<int>(s0.ok), s, 64);
  PagePlace p{};
  if (!mine || row >= bt.n_rows || i < 0 || i >= n) return p;
  const int pos = ctx - n + i;
  p.i = i;
  p.state = !ok ? 3 : pos < 0 ? 2 : 1;
  if (p.state == 1) {
    const int id = table_of(bt, lo + s)[pos / kKvqPage];
    p.state = kvq_page_ok(c, id) ? 1 : 3;
    p.t = pos % kKvqPage;
    p.left = ctx - pos;
    p.page = p.state == 1 ? id : 0;
  }
  return p;
}

// ---- tensors ---------------------------------------------------------------------------

template <bool BF16>
__device__ __forceinline__ void load8(const KvqTensor& x, int row, int head, int d, float (&f)[8]) {
  const int64_t at = row * x.row_stride + head * x.head_stride + d;
  if constexpr (BF16) {
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

// NT: not to be kept in the caches.
template <bool NT, typename T>
__device__ __forceinline__ void store16(T* p, T x) {
  if constexpr (NT) __builtin_nontemporal_store(x, p);
  else *p = x;
}
template <bool BF16, bool NT = false>
__device__ __forceinline__ void store8(const KvqTensor& x, int row, int head, int d, const float (&f)[8]) {
  const int64_t at = row * x.row_stride + head * x.head_stride + d;
  if constexpr (BF16) {
    bf16_t* p = static_cast<bf16_t*>(x.p) + at;
    if (x.vec) {
      u32x4 w;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        w[i] = static_cast<uint32_t>(f32_to_bf16(f[2 * i])) | static_cast<uint32_t>(f32_to_bf16(f[2 * i + 1])) << 16;
      store16<NT>(reinterpret_cast<u32x4*>(p), w);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) p[i] = f32_to_bf16(f[i]);
    }
  } else {
    float* p = static_cast<float*>(x.p) + at;
    if (x.vec) {
      store16<NT>(reinterpret_cast<f32x4_t*>(p), f32x4_t{f[0], f[1], f[2], f[3]});
      store16<NT>(reinterpret_cast<f32x4_t*>(p + 4), f32x4_t{f[4], f[5], f[6], f[7]});
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) p[i] = f[i];
    }
  }
}

// The two values of byte I of a word of codes, packed bf16 (exact).
template <int I>
__device__ __forceinline__ uint32_t code_pair(uint32_t w, float s) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, I));
}

// Sums over the wave's lanes up to each lane, in six additions across lanes.
__device__ __forceinline__ int wave_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);  // one lane up within 16
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // lane 15 of a row of 16 to the next
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // lane 31 to the upper half
  return x;
}

// ---- a page as operands, and its softmax ----------------------------------------------

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

// A page of one head as a lane holds it.  NT: not to be kept in the caches, what one wave alone reads.
template <bool NT, typename T>
__device__ __forceinline__ T load_page(const T* p) {
  if constexpr (NT) return __builtin_nontemporal_load(p);
  else return *p;
}
template <int HD>
struct PageK {
  u32x4 k[HD / 32];
  uint32_t s;
  template <bool NT = true>
  __device__ __forceinline__ void load(const char* block) {
    const int lane = threadIdx.x & 63;
    const u32x4* p = reinterpret_cast<const u32x4*>(block) + lane;
#pragma unroll
    for (int i = 0; i < HD / 32; ++i) k[i] = load_page<NT>(p + 64 * i);
    s = load_page<NT>(reinterpret_cast<const uint32_t*>(block + 64 * HD) + ((lane >> 4) * HD / 128) * 16 + (lane & 15));
  }
};
template <int HD>
struct PageV {
  u32x4 v[HD / 32], s;
  template <bool NT = true>
  __device__ __forceinline__ void load(const char* block) {
    const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
    const u32x4* p = reinterpret_cast<const u32x4*>(block + 32 * HD) + lane;
#pragma unroll
    for (int i = 0; i < HD / 32; ++i) v[i] = load_page<NT>(p + 64 * i);
    s = load_page<NT>(reinterpret_cast<const u32x4*>(block + 66 * HD) + (c * HD / 512) * 4 + g);
  }
};

// Byte `i` of a word as the scale of a four-bit conversion, which reads a float's exponent field and nothing else of it.
__device__ __forceinline__ float scale_of(uint32_t word, int i) {
  return __uint_as_float(i == 3 ? word >> 1 : word << (23 - 8 * i));
}

// The queries of the 16 columns, and S^T = K Q^T of a page's tile u: rows are the tile's tokens, columns the queries.
// Queries are NQ pieces of bf16, one, or three (24 bits) of fp32; K unpacked to bf16 is exact.
// (v_mfma_scale_f32_16x16x128_f8f6f4 would take K's codes as they are, with queries as two e4m3 pieces, but its sum keeps
// only about 11 bits below its largest product; scores are sums in fp32.)
template <int HD, int NQ>
struct Query {
  bf16x8_t q[HD / 32][NQ];
  __device__ __forceinline__ void load(const KvqTensor& t, int row, int head) {
    const int g = (threadIdx.x & 63) >> 4;
    float x[HD / 32][8];
#pragma unroll
    for (int j = 0; j < HD / 32; ++j) load8<NQ == 1>(t, row, head, g * (HD / 4) + 8 * j, x[j]);
#pragma unroll
    for (int j = 0; j < HD / 32; ++j) split8<NQ>(x[j], q[j]);
  }
  __device__ __forceinline__ f32x4_t scores(const PageK<HD>& pg, int u) const {
    f32x4_t acc{0.f, 0.f, 0.f, 0.f};
    const float s = scale_of(pg.s, u);
#pragma unroll
    for (int j = 0; j < HD / 32; ++j) {
      const uint32_t w = HD == 128 ? pg.k[u][j] : pg.k[u >> 1][2 * (u & 1) + j];
      const u32x4 k{code_pair<0>(w, s), code_pair<1>(w, s), code_pair<2>(w, s), code_pair<3>(w, s)};
#pragma unroll
      for (int n = 0; n < NQ; ++n) acc = mfma16x16x32(__builtin_bit_cast(bf16x8_t, k), q[j][n], acc);
    }
    return acc;
  }
};

// One page of an online softmax in the log2 domain, for a lane's N scores of one column.
//   The reference m moves only when the sum of a page's probabilities passes kSumMost (or there is none yet): up to that they
// lose nothing, the outputs need rescaling a few times per item instead of every page, and a page's own maximum is not
// formed at all: its sum tells.  l is the lane's part of the sum; the lanes of a column add theirs at the end.
//   In fp16 (HALF) the largest probability of a page that moves m is 2^7, and none passes 2^15: from 2^-14 on, 2^-21 of that
// largest one, each is rounded once, to 2^-11 of itself.  Smaller ones fp16 would hold with fewer bits or not at all, to 2^-25,
// and a row whose largest weights meet values of zero is made of them.  So
// - m also moves down, where a page's largest is below 2^-9 (2^kDrop below): the sums are in fp32 and hold 2^kDropMost more, and
//   pages of small weights, as behind one strong key, come to lie like any other;
// - in pages that have just moved m, or of which a lane's sum is below kSumLeast, small_page takes those below 2^-14 as a
//   second operand, 2^29 times as large and normal down to 2^-43, 2^-50 of the largest.  Elsewhere 2^-25 for each of the
//   lane's N keys is less than 2^-11 of their sum.
// Without all this | with it: a prompt of 14,500 tokens 1,400 | 1,421 us, 64 of 512 tokens with 64 dims 94 | 100 (every fifth page
// is a first one, whose look for small ones takes most of that), decoding 23.3 | 23.6. Every key 15 nats below the first: 1,372 |
// 1,395, with small_page in the place of moves down 2,550; with every page looked through for small ones 2,130 for any keys.
struct Softmax {
  float m = -INFINITY, l = 0.f;
  float high = -INFINITY;  // the highest m
};
constexpr float kLift = 7.f, kDrop = 16.f, kDropMost = 40.f;
constexpr float kSmallBelow = 0x1p-14f;
constexpr float kSumLeast = 0x1p-9f;
template <bool HALF> constexpr float kSumMost = HALF ? 0x1p15f : 0x1p8f;

// Two probabilities as fp16, rounded to nearest; sum: theirs as rounded, added to it.
__device__ __forceinline__ uint32_t half_pair(float a, float b, float& sum) {
  const f16x2 p = __builtin_convertvector(f32x2{a, b}, f16x2);
  sum = __builtin_amdgcn_fdot2(p, f16x2{1, 1}, sum, false);
  return __builtin_bit_cast(uint32_t, p);
}

// The small probabilities of a page of fp16 ones x, w: products(small) of the operand that holds them, between scalings of the
// outputs by 2^29 and back, which are exact.  w is left without them.  Returns the sum of all, as rounded.
template <int N, typename Rescale, typename Products>
__device__ __forceinline__ float small_page(const float (&x)[N], uint32_t (&w)[N / 2], float sum, Rescale rescale, Products products) {
  uint32_t least = ~0u;  // by their bits less one: zeros, of keys out of sight, come last
#pragma unroll
  for (int k = 0; k < N; ++k) least = min(least, __float_as_uint(x[k]) - 1);
  if (__builtin_expect(!__any(least < __builtin_bit_cast(uint32_t, kSmallBelow) - 1), 1)) return sum;
  uint32_t small[N / 2];
  float large_sum = 0.f, small_sum = 0.f;
#pragma unroll
  for (int k = 0; k < N / 2; ++k) {
    const bool a = x[2 * k] < kSmallBelow, b = x[2 * k + 1] < kSmallBelow;
    w[k] = half_pair(a ? 0.f : x[2 * k], b ? 0.f : x[2 * k + 1], large_sum);
    small[k] = half_pair(a ? x[2 * k] * 0x1p29f : 0.f, b ? x[2 * k + 1] * 0x1p29f : 0.f, small_sum);
  }
  rescale(0x1p29f);
  products(small);
  rescale(0x1p-29f);
  return __builtin_fmaf(small_sum, 0x1p-29f, large_sum);
}

// x: the scores, and then the probabilities; w: these as pairs of fp16 (HALF), whose own sum l takes.  rescale(alpha) scales
// the outputs, products(w) adds the page's products of such pairs to them (HALF: of small probabilities; those of w are the
// caller's); ACROSS are the lanes (besides the first, as xor masks) that share the column.
template <bool HALF, int N, typename Rescale, typename Products, typename... Across>
__device__ __forceinline__ void softmax_page(Softmax& st, float (&x)[N], uint32_t (&w)[N / 2], float scale_log2, Rescale rescale,
                                             Products products, Across... across) {
  float s[N], sum;
#pragma unroll
  for (int k = 0; k < N; ++k) s[k] = x[k];
  auto move = [&] {
    float top = -INFINITY;
#pragma unroll
    for (int k = 0; k < N; ++k) top = fmaxf(top, s[k]);
    ((top = fmaxf(top, __shfl_xor(top, across, 64))), ...);
    float m_new = fmaxf(st.m, top * scale_log2);
    if constexpr (HALF) {
      m_new = __builtin_fmaf(top, scale_log2, -kLift);
      if (!(m_new > st.m)) m_new = m_new < st.m - kDrop && top > -INFINITY ? fmaxf(m_new, st.high - kDropMost) : st.m;
      st.high = fmaxf(st.high, m_new);
    }
    const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(st.m - m_new);
    st.m = m_new;
    st.l *= alpha;
    rescale(alpha);
  };
  auto form = [&] {
    const float shift = st.m == -INFINITY ? 0.f : st.m;
#pragma unroll
    for (int k = 0; k < N; ++k) x[k] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[k], scale_log2, -shift));
    float part[2] = {0.f, 0.f};
    if constexpr (HALF) {
#pragma unroll
      for (int k = 0; k < N / 2; ++k) w[k] = half_pair(x[2 * k], x[2 * k + 1], part[k & 1]);
    } else {
#pragma unroll
      for (int k = 0; k < N; ++k) part[k & 1] += x[k];
    }
    sum = part[0] + part[1];
  };
  const bool none = __any(st.m == -INFINITY);
  if (none) move();
  form();
  if constexpr (HALF) {
    bool out = __any(sum < kSumLeast || sum > kSumMost<HALF>);
    if (__builtin_expect(none || out, 0)) {  // out of line: a prompt of 8,192 tokens with 64 dims 197 | 189 us
      float top = 0.f;
#pragma unroll
      for (int k = 0; k < N; ++k) top = fmaxf(top, x[k]);
      out = __any((sum < kSumLeast && top > 0.f) || sum > kSumMost<HALF>);  // not for lanes whose keys are all out of sight
      if (out) {
        move();
        form();
      }
      if (none || out) sum = small_page(x, w, sum, rescale, products);
    }
  } else if (__any(sum > kSumMost<HALF>)) {
    move();
    form();
  }
  st.l += sum;
}

// From probabilities in fp16 to those in bf16, whose reference is a page's largest.
template <typename Rescale>
__device__ __forceinline__ void leave_half(Softmax& st, Rescale rescale) {
  st.m += kLift;
  st.l *= 0x1p-7f;
  rescale(0x1p-7f);
}

// The two values of byte `i` of a word of codes, packed as the type's operand.
template <bool HALF>
__device__ __forceinline__ uint32_t value_pair(uint32_t w, float s, int i) {
  if constexpr (HALF) {
    return __builtin_bit_cast(uint32_t, i == 0   ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, 0)
                                        : i == 1 ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, 1)
                                        : i == 2 ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, 2)
                                                 : __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, 3));
  } else {
    return i == 0 ? code_pair<0>(w, s) : i == 1 ? code_pair<1>(w, s) : i == 2 ? code_pair<2>(w, s) : code_pair<3>(w, s);
  }
}

// O^T += V^T P^T over tokens 32h .. 32h + 31 of the page: accumulator i's rows are dimensions hd/16 c + i.  The lane's
// probabilities are x + 8 h, or as fp16 w + 4 h (HALF: V and P in fp16; else V in bf16 and P as NP pieces of it).
template <int HD, bool HALF, int NP>
__device__ __forceinline__ void half_values(const PageV<HD>& pg, int h, const float (&x)[16], const uint32_t (&w16)[8], f32x4_t (&o)[HD / 16]) {
  bf16x8_t pf[NP];
  f16x8 ph;
  if constexpr (HALF) {
    ph = __builtin_bit_cast(f16x8, u32x4{w16[4 * h], w16[4 * h + 1], w16[4 * h + 2], w16[4 * h + 3]});
  } else {
    float y[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) y[k] = x[8 * h + k];
    split8<NP>(y, pf);
  }
#pragma unroll
  for (int j = 0; j < HD / 32; ++j) {  // a pair of dimensions
    uint32_t v[8];                     // of eight tokens
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const uint32_t w = HD == 128 ? pg.v[2 * h + (k >> 2)][k & 3] : pg.v[h][k >> 1];
      v[k] = value_pair<HALF>(w, scale_of(pg.s[2 * h + (k >> 2)], k & 3), HD == 128 ? j : 2 * (k & 1) + j);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {  // its two dimensions: the low or high halves of neighbouring tokens' pairs
      u32x4 w;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = __builtin_amdgcn_perm(v[2 * e + 1], v[2 * e], i ? 0x07060302u : 0x05040100u);
      if constexpr (HALF) {
        o[2 * j + i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, w), ph, o[2 * j + i], 0, 0, 0);
      } else {
#pragma unroll
        for (int n = 0; n < NP; ++n) o[2 * j + i] = mfma16x16x32(__builtin_bit_cast(bf16x8_t, w), pf[n], o[2 * j + i]);
      }
    }
  }
}

// Whether fp16 holds every value of these blocks exactly: scale bytes 104 .. 135 (2^-23 .. 2^8).  A byte that carries into
// the next is out of range itself.
__device__ __forceinline__ bool fits_half(const u32x4& s) {
  uint32_t t = 0;
#pragma unroll
  for (int u = 0; u < 4; ++u) t |= (s[u] + 0x18181818u) ^ 0x80808080u;
  return !(t & 0xe0e0e0e0u);
}

// Scale bytes of tokens t .. t + 3, those from `end` on as 1: what lies behind the last key may be anything.
__device__ __forceinline__ uint32_t scales_below(uint32_t s, int t, int end) {
  const uint32_t keep = static_cast<uint32_t>((1ull << (8 * min(max(end - t, 0), 4))) - 1);
  return (s & keep) | (0x7f7f7f7fu & ~keep);
}

// A page with NaN blocks: their scales become 2^-127, which the zero probability of a key out of sight clears (as NaN it
// would not), and the lane's outputs turn NaN if its column sees the token.  A lane's outputs all lie in one block of 32
// dimensions.
template <int HD, int NO = HD / 16>
__device__ __forceinline__ void nan_values(PageV<HD>& pg, const char* block, int tok0, int lim, f32x4_t (&o)[NO]) {
  const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
  for (int u = 0; u < 4; ++u)
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (((pg.s[u] >> (8 * r)) & 255u) == 255u) pg.s[u] &= ~(255u << (8 * r));
  bool bad = false;
  for (int t = 0; t < kKvqPage; ++t)
    bad |= tok0 + t <= lim && static_cast<unsigned char>(block[kvq_v_scale(t, g * HD / 128, HD)]) == 255;
  if (bad) {
#pragma unroll
    for (int i = 0; i < NO; ++i) o[i] += __builtin_nanf("");
  }
}

}  // namespace

}  // namespace rollpack
