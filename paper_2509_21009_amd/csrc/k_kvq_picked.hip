// Causal attention over picked pages of the 4-bit KV cache (kvq_pages.hpp): each row and KV head has a list of pages.
#include <algorithm>
#include <type_traits>

#include "kernels.hpp"
#include "kvq_device.hpp"
#include "kvq_pages.hpp"

namespace rollpack {

namespace {

// Of a row: its sequence's row of the page table, its position, and whether its sequence is within the call's bounds.
struct PickedRow {
  const int32_t* table = nullptr;
  int pos = -1;
  bool ok = false, mine = false;  // mine: a row of the call
};

__device__ __forceinline__ PickedRow picked_row(const KvqBatch& bt, int row) {
  PickedRow p;
  const int b = wave_find_seq(bt, row);
  if (b < 0) return p;
  const KvqSeq s = kvq_seq(bt, b);
  const int i = row - s.r0;
  p.mine = i >= 0 && i < s.n;
  p.ok = s.ok;
  p.pos = s.ok ? s.ctx - s.n + i : -1;
  p.table = table_of(bt, b);
  return p;
}

// Which row, KV head and columns block `index` has.
struct PickedBlock {
  int row, kh, ct;
};
__device__ __forceinline__ PickedBlock picked_block(int index, int n_kv, int col_tiles) {
  PickedBlock p;
  const int unit = index / col_tiles;
  p.ct = index - unit * col_tiles;
  p.row = unit / n_kv;
  p.kh = unit - p.row * n_kv;
  return p;
}

// A page's parts from bases in scalar registers: as one base with offsets past an instruction's 4 KB each load would add in the
// vector ALU, 64 bits wide.
typedef const __attribute__((address_space(1))) char device_char;  // of device memory, which the compiler could not tell any more
__device__ __forceinline__ device_char* scalar_base(const char* p) {
  device_char* d = (device_char*)(p);
  asm("" : "+s"(d));
  return d;
}
__device__ __forceinline__ uint32_t this_lane() {  // anew in each place: offsets widened once for all would be added in the vector ALU
  uint32_t lane = threadIdx.x & 63;
  asm volatile("" : "+v"(lane));
  return lane;
}
template <bool NT, typename T>
__device__ __forceinline__ T load_at(device_char* base, uint32_t offset) {
  const auto p = (const __attribute__((address_space(1))) T*)(base + offset);
  if constexpr (NT) return __builtin_nontemporal_load(p);
  else return *p;
}
template <int HD, bool NT>
__device__ __forceinline__ void load_keys(PageK<HD>& pg, const char* block) {
  const uint32_t lane = this_lane();
  device_char *keys = scalar_base(block), *scales = scalar_base(block + 64 * HD);
#pragma unroll
  for (int i = 0; i < HD / 32; ++i) pg.k[i] = load_at<NT, u32x4>(keys + 1024 * i, lane * 16);
  pg.s = load_at<NT, uint32_t>(scales, ((lane >> 4) * HD / 128) * 64 + (lane & 15) * 4);
}
template <int HD, bool NT>
__device__ __forceinline__ void load_values(PageV<HD>& pg, const char* block) {
  const uint32_t lane = this_lane();
  device_char *values = scalar_base(block + 32 * HD), *scales = scalar_base(block + 66 * HD);
#pragma unroll
  for (int i = 0; i < HD / 32; ++i) pg.v[i] = load_at<NT, u32x4>(values + 1024 * i, lane * 16);
  pg.s = load_at<NT, u32x4>(scales, ((lane & 15) * HD / 512) * 64 + (lane >> 4) * 16);
}

// Up to eight query heads take half of a product's 16 columns, and the other half saves two kinds of work:
//   Columns c and c + 8 are the same head.  Of a page's probabilities lanes c form those of its tokens 0 .. 31, lanes c + 8
// those of 32 .. 63; each half gets the other's as packed words.
//   A byte of V holds two dimensions of a token, d and d + 1.  Converted, they are neighbours in an operand, not two operands'
// elements, and stay so: the 32 elements of a product are 16 tokens' pairs, the probability of a token stands in the
// place of d, beside zero, for column c and in that of d + 1 for column c + 8.  So column c gets dimension d and column c + 8
// dimension d + 1, as many products as with a dimension to each, without the 64 instructions that would part the pairs.
struct NarrowWords {
  uint32_t sel[2][2];  // [tokens 32 .. 63][odd]: where a token's probability is in {own word, other half's}, and where it goes
  __device__ __forceinline__ explicit NarrowWords(bool upper) {
    sel[0][0] = upper ? 0x01000c0cu : 0x0c0c0504u;  // byte 0x0c is zero, bytes 4 .. 7 are the own word's
    sel[0][1] = upper ? 0x03020c0cu : 0x0c0c0706u;
    sel[1][0] = upper ? 0x05040c0cu : 0x0c0c0100u;
    sel[1][1] = upper ? 0x07060c0cu : 0x0c0c0302u;
  }
};

// O^T += V^T P^T of a page: the lane's eight probabilities are x, or as fp16 w (HALF; else pieces of bf16), accumulator j's row
// c' is dimension hd/16 c' + 2 j (+ 1 in columns from 8 on).
template <int HD, bool HALF, int NP>
__device__ __forceinline__ void narrow_values(const PageV<HD>& pg, const float (&x)[8], const uint32_t (&w16)[4], const NarrowWords& nw, f32x4_t (&o)[HD / 32]) {
  u32x4 own[NP];
  if constexpr (HALF) {
    own[0] = u32x4{w16[0], w16[1], w16[2], w16[3]};
  } else {
    float y[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) y[k] = x[k];
    bf16x8_t p[NP];
    split8<NP>(y, p);
#pragma unroll
    for (int n = 0; n < NP; ++n) own[n] = __builtin_bit_cast(u32x4, p[n]);
  }
  u32x4 other[NP];
#pragma unroll
  for (int n = 0; n < NP; ++n)
#pragma unroll
    for (int k = 0; k < 4; ++k) other[n][k] = static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(own[n][k]), 0x128, 0xf, 0xf, true));  // lane c ^ 8
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    u32x4 b[NP];
#pragma unroll
    for (int n = 0; n < NP; ++n)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int k = 2 * (u & 1) + (r >> 1);
        b[n][r] = __builtin_amdgcn_perm(own[n][k], other[n][k], nw.sel[u >> 1][r & 1]);
      }
#pragma unroll
    for (int j = 0; j < HD / 32; ++j) {
      u32x4 v;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const uint32_t w = HD == 128 ? pg.v[u][r] : pg.v[u >> 1][2 * (u & 1) + (r >> 1)];
        v[r] = value_pair<HALF>(w, scale_of(pg.s[u], r), HD == 128 ? j : 2 * (r & 1) + j);
      }
      if constexpr (HALF) {
        o[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, v), __builtin_bit_cast(f16x8, b[0]), o[j], 0, 0, 0);
      } else {
#pragma unroll
        for (int n = 0; n < NP; ++n) o[j] = mfma16x16x32(__builtin_bit_cast(bf16x8_t, v), __builtin_bit_cast(bf16x8_t, b[n]), o[j]);
      }
    }
  }
}

// One block of NW waves takes an item: the up to 16 (NARROW: 8) query heads of a row and KV head over a share of the row's list,
// whose entries the waves take in turn, 64 looked up at a time (entry, then its page).  What a wave does with a page is
// k_kvq_attend's: S^T = K Q^T, an online softmax in base 2 and O^T += V^T P^T from registers, P in fp16 while V's scales
// allow it.  The next page's K is loaded when the scores are formed, its V when the outputs are (two pages in registers left
// room for fewer waves: 64 rows of 48 pages 45 | 43 us).
//   HBM bounds decoding: one token each of 64 sequences, 48 pages each (8 KV heads of 128, 214 MB) 39 us, 5.5 TB/s.  The vector ALU
// bounds many rows, whose pages come from the caches: 512 rows of 32 pages (4 KV heads) 53 us, 11 TB/s, 77% of the cycles
// vector instructions, 298 a page, nearly half of them conversions from 4 bits, and 30% products, of which 7 columns of 16 are heads.
// NARROW took this from 61 us.
template <int HD, bool F32, int NW, bool KEEP, bool NARROW>
__global__ __launch_bounds__(64 * NW, F32 ? 2 : NARROW ? 4 : 3) void k_kvq_attend_picked(KvqPickedArgs a, PickedPlan plan) {
  constexpr int NT = HD / 16, OLD = HD + 4, COLS = NARROW ? 8 : 16, NX = NARROW ? 8 : 16;  // NX: scores of a lane and page
  __shared__ __attribute__((aligned(16))) float so[NW][COLS * OLD];
  __shared__ float sm[NW][16], sl[NW][16];
  __shared__ int some[NW];
  const KvqBatch& bt = a.batch;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 4, c = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n_kv = a.cache.n_kv, G = a.n_q / n_kv;
  const int index = blockIdx.x, split = blockIdx.y;
  const PickedBlock pb = picked_block(index, n_kv, plan.col_tiles);
  const int per_item = (a.n + plan.items - 1) / plan.items, e0 = split * per_item;
  const int entries = max(0, min(per_item, a.n - e0));
  const int n_cols = min(16, G - 16 * pb.ct), head0 = pb.kh * G + 16 * pb.ct;
  const float scale_log2 = a.scale * kLog2e;
  const int32_t* list = a.picks + (static_cast<size_t>(pb.row) * n_kv + pb.kh) * a.n + e0;
  auto entry_of = [&](int i) { return i < entries ? list[i] : -1; };
  int entry = entry_of(wave + NW * lane);  // on its way while the row is looked up
  const PickedRow pr = picked_row(bt, pb.row);
  if (!pr.mine) return;

  constexpr int NO = NARROW ? NT / 2 : NT;
  f32x4_t o[NO];
#pragma unroll
  for (int i = 0; i < NO; ++i) o[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  Softmax st;
  const bool upper = NARROW && c >= 8;
  const NarrowWords narrow(upper);
  // The wave's entries: `todo` has a bit for each of the 64 looked up that names a page the row sees.
  uint64_t todo = 0;
  int looked = wave, id = 0;
  const size_t bytes = kvq_block_bytes(HD);
  const char* base = a.cache.blocks + pb.kh * bytes;
  struct Page {
    const char* at;
    int tok0;
    bool there, lost;  // lost: its id is outside the cache; page 0 stands in, and its scores are NaN
  };
  auto advance = [&]() {
    while (!todo && looked < entries) {
      if (looked != wave) entry = entry_of(looked + NW * lane);
      const bool seen = entry >= 0 && entry <= (pr.pos >> 6);  // the position -1 sees none
      id = seen ? pr.table[entry] : 0;
      todo = __ballot(seen);
      looked += NW * 64;
    }
    Page p{base, 0, todo != 0, false};
    if (p.there) {
      const int src = __ffsll(static_cast<unsigned long long>(todo)) - 1;
      todo &= todo - 1;
      const int page = __builtin_amdgcn_readlane(id, src);
      p.lost = !kvq_page_ok(a.cache, page);
      p.tok0 = __builtin_amdgcn_readlane(entry, src) * kKvqPage;
      p.at = base + static_cast<size_t>(p.lost ? 0 : page) * n_kv * bytes;
    }
    return p;
  };
  Page now = advance();
  const bool any = now.there;
  if (any) {
    Page next = advance();
    Query<HD, F32 ? 3 : 1> qf;
    qf.load(a.q, pb.row, head0 + min(c & (COLS - 1), n_cols - 1));
    auto rescale = [&](float alpha) {
#pragma unroll
      for (int t = 0; t < NO; ++t) o[t] *= alpha;
    };
    PageV<HD> pv;
    auto nan_outputs = [&](const Page& p) { nan_values<HD, NO>(pv, p.at, p.tok0, pr.pos, o); };
    // The wave's pages from `now` on.  HALF: V and P in fp16, up to the first page that does not fit; else in bf16.
    auto walk = [&](auto half_tag) {
      constexpr bool HALF = half_tag.value;
      PageK<HD> pk;
      load_keys<HD, !KEEP>(pk, now.at);
      load_values<HD, !KEEP>(pv, now.at);
      while (now.there) {
        f32x4_t s[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) s[u] = qf.scores(pk, u);
        load_keys<HD, !KEEP>(pk, next.at);
        const int held = now.lost ? now.tok0 : pr.pos + 1;  // what lies behind, or in a page that stands in, may be anything
        if (now.tok0 + kKvqPage > held) {
          asm volatile("");  // a branch: as selects it would cost every page
#pragma unroll
          for (int u = 0; u < 4; ++u) pv.s[u] = scales_below(pv.s[u], now.tok0 + 16 * u + 4 * g, held);
        }
        if (HALF && !__all(fits_half(pv.s))) return;
        float x[NX];
        uint32_t w[NX / 2];
#pragma unroll
        for (int k = 0; k < NX; ++k) x[k] = NARROW && upper ? s[2 + (k >> 2) % 2][k & 3] : s[k >> 2][k & 3];
        if (now.lost || now.tok0 + kKvqPage > pr.pos + 1) {
          asm volatile("");
          const int tok = now.tok0 + 4 * g + (upper ? 32 : 0);
#pragma unroll
          for (int k = 0; k < NX; ++k) {
            const float v = now.lost ? __builtin_nanf("") : x[k];
            x[k] = tok + 16 * (k >> 2) + (k & 3) > pr.pos ? -INFINITY : v;
          }
        }
        auto products = [&](const uint32_t (&p)[NX / 2]) {
          if constexpr (NARROW) {
            narrow_values<HD, HALF, HALF ? 1 : F32 ? 3 : 2>(pv, x, p, narrow, o);
          } else {
            half_values<HD, HALF, F32 ? 3 : 2>(pv, 0, x, p, o);
            half_values<HD, HALF, F32 ? 3 : 2>(pv, 1, x, p, o);
          }
        };
        auto small_products = [&](const uint32_t (&p)[NX / 2]) {
          if constexpr (HALF) products(p);
        };
        if constexpr (NARROW) softmax_page<HALF>(st, x, w, scale_log2, rescale, small_products, 8, 16, 32);
        else softmax_page<HALF>(st, x, w, scale_log2, rescale, small_products, 16, 32);
        if (!HALF && !__all(fits_half(pv.s))) nan_outputs(now);
        products(w);
        now = next;
        load_values<HD, !KEEP>(pv, now.at);
        if (now.there) next = advance();
      }
    };
    if constexpr (!F32) {
      walk(std::true_type{});
      if (now.there) leave_half(st, rescale);
    }
    if (F32 || now.there) walk(std::false_type{});
    if constexpr (NARROW) st.l += __shfl_xor(st.l, 8, 64);
    st.l += __shfl_xor(st.l, 16, 64);
    st.l += __shfl_xor(st.l, 32, 64);
  }

  // Combine the waves: one without a page has m = -inf, l = 0, o = 0.
  if (g == 0) {
    sm[wave][c] = st.m;
    sl[wave][c] = st.l;
  }
  if (lane == 0) some[wave] = any;
  __syncthreads();
  float mx = sm[0][c];
#pragma unroll
  for (int w = 1; w < NW; ++w) mx = fmaxf(mx, sm[w][c]);
  const float fac = st.m == -INFINITY ? (st.l == 0.f ? 0.f : 1.f) : __builtin_amdgcn_exp2f(st.m - mx);
  if ((c & (COLS - 1)) < n_cols) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float* to = &so[wave][(c & (COLS - 1)) * OLD + (4 * g + e) * NT];  // dimensions hd/16 (4g + e) ..
      if constexpr (NARROW) {
#pragma unroll
        for (int j = 0; j < NO; ++j) to[2 * j + upper] = o[j][e] * fac;
      } else {
#pragma unroll
        for (int i = 0; i < NT; i += 4) *reinterpret_cast<f32x4_t*>(to + i) = f32x4_t{o[i][e], o[i + 1][e], o[i + 2][e], o[i + 3][e]} * fac;
      }
    }
  }
  __syncthreads();
  int n_some = 0;
#pragma unroll
  for (int w = 0; w < NW; ++w) n_some |= some[w];
  const int64_t part = static_cast<int64_t>(index) * plan.items + split;
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
    if (plan.items == 1) {
      // a list without a page that the row sees: zeros; a sequence out of bounds: NaN
      const float inv = !pr.ok ? __builtin_nanf("") : !n_some ? 0.f : 1.f / den;
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] = y[k >> 2][k & 3] * inv;
      store8<!F32>(a.out, pb.row, head0 + col, d, x);
    } else {
      float* po = a.part_o + (part * plan.cols + col) * HD + d;
      *reinterpret_cast<f32x4_t*>(po) = y[0];
      *reinterpret_cast<f32x4_t*>(po + 4) = y[1];
      if (d == 0) {
        a.part_ml[part * 2 * plan.cols + col] = m4;
        a.part_ml[part * 2 * plan.cols + plan.cols + col] = den;
      }
    }
  }
}

// Joins the items of a block's list: one block per (block, column).  Four dimensions to a thread, the items dealt out to
// groups of threads whose loads are all in flight at once.
template <int HD, bool F32>
__global__ __launch_bounds__(256) void k_kvq_join_picked(KvqPickedArgs a, PickedPlan plan) {
  constexpr int LPC = HD / 4, NG = 256 / LPC, PER = kKvqTileItems / NG;
  __shared__ float sw[kKvqTileItems];
  __shared__ __attribute__((aligned(16))) f32x4_t sx[NG][LPC];
  const int n_kv = a.cache.n_kv, G = a.n_q / n_kv, col = blockIdx.y;
  const PickedBlock pb = picked_block(blockIdx.x, n_kv, plan.col_tiles);
  const PickedRow pr = picked_row(a.batch, pb.row);
  if (!pr.mine || col >= G - 16 * pb.ct) return;
  const int n = plan.items;
  const int64_t part = static_cast<int64_t>(blockIdx.x) * n;
  const int grp = threadIdx.x / LPC, d = threadIdx.x % LPC * 4;
  const float* po = a.part_o + (part * plan.cols + col) * HD + d;
  const int64_t step = static_cast<int64_t>(plan.cols) * HD;
  f32x4_t x[PER];
#pragma unroll
  for (int k = 0; k < PER; ++k) x[k] = *reinterpret_cast<const f32x4_t*>(po + min(grp + NG * k, n - 1) * step);
  bool some = false;
  const int32_t* list = a.picks + (static_cast<size_t>(pb.row) * n_kv + pb.kh) * a.n;
  for (int i = threadIdx.x; i < a.n; i += 256) some |= list[i] >= 0 && list[i] <= (pr.pos >> 6);
  float den = 0.f;
  if (threadIdx.x < 64) {
    const int lane = threadIdx.x;
    const float* ml = a.part_ml + (part + min(lane, n - 1)) * 2 * plan.cols + col;
    const float m = lane < n ? ml[0] : -INFINITY, l = lane < n ? ml[plan.cols] : 0.f;
    const float mx = wave_max(m);
    const float w = m == -INFINITY ? (l == 0.f ? 0.f : 1.f) : __builtin_amdgcn_exp2f(m - mx);
    sw[lane] = w;
    den = wave_sum(w * l);
  }
  some = __syncthreads_or(some);
  f32x4_t sum{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int k = 0; k < PER; ++k)
    if (grp + NG * k < n) sum += x[k] * sw[grp + NG * k];
  sx[grp][threadIdx.x % LPC] = sum;
  __syncthreads();
  if (threadIdx.x < HD / 8) {
    const float inv = !pr.ok ? __builtin_nanf("") : !some ? 0.f : 1.f / den;
    f32x4_t y[2]{};
#pragma unroll
    for (int k = 0; k < NG; ++k) {
      y[0] += sx[k][2 * threadIdx.x];
      y[1] += sx[k][2 * threadIdx.x + 1];
    }
    float out[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) out[k] = y[k >> 2][k & 3] * inv;
    store8<!F32>(a.out, pb.row, pb.kh * G + 16 * pb.ct + col, threadIdx.x * 8, out);
  }
}

template <int HD, bool F32>
hipError_t picked_launch(KvqPickedArgs a, float* ws, hipStream_t s) {
  const PickedPlan p = picked_plan(a.cache, a.batch, a.n, a.n_q);
  const size_t n = picked_part_floats(a.cache, a.batch, p);
  a.part_o = ws;
  a.part_ml = n ? ws + n : nullptr;
  const uint32_t blocks = static_cast<uint32_t>(picked_blocks(a.cache, a.batch, p));
  const dim3 grid(blocks, p.items);
#define RP_PICKED_AS(W, KEEP, NARROW) launch_kernel((k_kvq_attend_picked<HD, F32, W, KEEP, NARROW>), grid, dim3(64 * W), 0, s, a, p)
#define RP_PICKED(W)                                          \
  case W:                                                     \
    if (p.cols <= 8 && p.shared) RP_PICKED_AS(W, true, true); \
    else if (p.cols <= 8) RP_PICKED_AS(W, false, true);       \
    else if (p.shared) RP_PICKED_AS(W, true, false);          \
    else RP_PICKED_AS(W, false, false);                       \
    break;
  switch (p.waves) {
    RP_PICKED(4) RP_PICKED(8)
    case 2:  // of rows that share pages
      if (p.cols <= 8) RP_PICKED_AS(2, true, true);
      else RP_PICKED_AS(2, true, false);
      break;
    default: return hipErrorInvalidValue;
  }
#undef RP_PICKED
#undef RP_PICKED_AS
  if (n) launch_kernel((k_kvq_join_picked<HD, F32>), dim3(blocks, p.cols), dim3(256), 0, s, a, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_kvq_attend_picked(const KvqPickedArgs& a, void* ws, hipStream_t s) {
  float* w = static_cast<float*>(ws);
  if (a.q.bf16) return a.cache.hd == 128 ? picked_launch<128, false>(a, w, s) : picked_launch<64, false>(a, w, s);
  return a.cache.hd == 128 ? picked_launch<128, true>(a, w, s) : picked_launch<64, true>(a, w, s);
}

}  // namespace rollpack
