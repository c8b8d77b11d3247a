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

// One block of NW waves takes an item: the up to 16 query heads of a row and KV head over a share of the row's list, whose
// entries the waves take in turn, 64 looked up at a time (entry, then its page).  What a wave does with a page is
// k_kvq_attend's: S^T = K Q^T, an online softmax in base 2 and O^T += V^T P^T from registers, P in fp16 while V's scales
// allow it.
template <int HD, bool F32, int NW, bool KEEP>
__global__ __launch_bounds__(64 * NW, F32 ? 2 : 3) void k_kvq_attend_picked(KvqPickedArgs a, PickedPlan plan) {
  constexpr int NT = HD / 16, OLD = HD + 4;
  __shared__ __attribute__((aligned(16))) float so[NW][16 * OLD];
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

  f32x4_t o[NT];
#pragma unroll
  for (int i = 0; i < NT; ++i) o[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  Softmax st;
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
    qf.load(a.q, pb.row, head0 + min(c, n_cols - 1));
    auto rescale = [&](float alpha) {
#pragma unroll
      for (int t = 0; t < NT; ++t) o[t] *= alpha;
    };
    // The wave's pages from `now` on.  HALF: V and P in fp16, up to the first page that does not fit; else in bf16.
    auto walk = [&](auto half_tag) {
      constexpr bool HALF = half_tag.value;
      PageK<HD> pk;
      PageV<HD> pv;
      pk.template load<!KEEP>(now.at);
      pv.template load<!KEEP>(now.at);
      while (now.there) {
        f32x4_t s[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) s[u] = qf.scores(pk, u);
        pk.template load<!KEEP>(next.at);
        const int held = now.lost ? now.tok0 : pr.pos + 1;  // what lies behind, or in a page that stands in, may be anything
        if (now.tok0 + kKvqPage > held) {
#pragma unroll
          for (int u = 0; u < 4; ++u) pv.s[u] = scales_below(pv.s[u], now.tok0 + 16 * u + 4 * g, held);
        }
        if (HALF && !__all(fits_half(pv.s))) return;
        if (now.lost || now.tok0 + kKvqPage > pr.pos + 1) {
          asm volatile("");  // a branch: as selects it would cost every page
#pragma unroll
          for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float v = now.lost ? __builtin_nanf("") : s[u][e];
              s[u][e] = now.tok0 + 16 * u + 4 * g + e > pr.pos ? -INFINITY : v;
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
        if (!HALF && !__all(fits_half(pv.s))) nan_values<HD>(pv, now.at, now.tok0, pr.pos, o);
        half_values<HD, HALF, F32 ? 3 : 2>(pv, 0, x, w, o);
        half_values<HD, HALF, F32 ? 3 : 2>(pv, 1, x, w, o);
        now = next;
        pv.template load<!KEEP>(now.at);
        if (now.there) next = advance();
      }
    };
    if constexpr (!F32) {
      walk(std::true_type{});
      if (now.there) leave_half(st, rescale);
    }
    if (F32 || now.there) walk(std::false_type{});
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
  if (c < n_cols) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int i = 0; i < NT; i += 4)  // dimensions hd/16 (4g + e) + i ..
        *reinterpret_cast<f32x4_t*>(&so[wave][c * OLD + (4 * g + e) * NT + i]) =
            f32x4_t{o[i][e], o[i + 1][e], o[i + 2][e], o[i + 3][e]} * fac;
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
#define RP_PICKED(W)                                                                                              \
  case W:                                                                                                         \
    if (p.shared) launch_kernel((k_kvq_attend_picked<HD, F32, W, true>), grid, dim3(64 * W), 0, s, a, p);         \
    else launch_kernel((k_kvq_attend_picked<HD, F32, W, false>), grid, dim3(64 * W), 0, s, a, p);                 \
    break;
  switch (p.waves) {
    RP_PICKED(4) RP_PICKED(8)
    default: return hipErrorInvalidValue;
  }
#undef RP_PICKED
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
