// Pages of the 4-bit KV cache (kvq_pages.hpp): handing them out, the ranges of their keys, their scores for a query, and the
// pages that are picked by these.
#include <algorithm>
#include <type_traits>

#include "kernels.hpp"
#include "kvq_device.hpp"
#include "kvq_pages.hpp"

namespace rollpack {

namespace {

typedef short s16x2 __attribute__((ext_vector_type(2)));

// ---- pages handed out ------------------------------------------------------------------
//
// With have = ceil(context / 64) and want = ceil(length / 64) pages, a sequence gives back pages want .. have - 1 or needs pages
// have .. want - 1.  Counted over the sequences in order and each one's pages in order, of R given back the j-th becomes
// entry n_free + R - 1 - j of the list, and the k-th needed is entry n_free + R - 1 - k: a call and the one that takes it back are
// each other's inverse, and what is given back is handed out again first.
//   k_kvq_fit: checks, sums over the sequences, offsets, contexts, pages given back, and the rows: a row's page is new or in the
// table, and the first row of a new page enters it there.  Every block of a launch does the sums for itself, and has a part of the
// pages given back and of the rows.  What the blocks start from, contexts and the count of free pages, is written by the last one to
// have read it, whichever that is: nothing waits.  Nothing else that is read is written: pages are taken from below n_free and given
// back above it, a new page that was just given back is looked up where its last owner's table has it, and the table's new entries lie
// behind those of the sequence's old pages.
//   More sequences than a block has threads: one block, and the rows in a launch of their own, k_kvq_fit_rows.
//   Bound by reads that wait for each other (state, context and length; the pages given back; the rows' pages), and by what 16 waves
// issue for the sums.  A call and its taking back, us: 64 sequences 8.3; 512 of 162,000 tokens that turn into as many others, both
// ways, 15; 1,024 prompts of 590,000 tokens (4.7 MB written) 20.6.  With the rows in a second launch the last two took 24.
constexpr int kFitThreads = 1024;
// Rows of a block, up to 256 blocks; then these have more.  In blocks of 1,024 | one block, us, with a call without rows: 512 sequences
// of 4 tokens 10.8 | 9.9, of 8 10.6 | 12.1, of 64 10.4 | 32; 16 of 500 9.8 | 13.0.  Blocks of 1,024 | 256 blocks: 590,000 rows 27.6 | 20.6.
constexpr int kFitBlock = 1024;
constexpr int kFitUnroll = 4;

// The last of lo .. hi whose start is not past j, of starts that do not descend.
template <typename F>
__device__ __forceinline__ int last_from(int lo, int hi, int j, F start) {
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (start(mid) <= j) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// The same for a j of the wave's, in n <= 1024 starts in LDS, from 0: 16 to a lane, then these 16.
__device__ __forceinline__ int wave_last(const int* start, int n, int j) {
  const int lane = threadIdx.x & 63;
  const int at = 16 * (__builtin_popcountll(__ballot(16 * lane < n && start[min(16 * lane, n)] <= j)) - 1);
  return at + __builtin_popcountll(__ballot(lane < 16 && at + lane < n && start[min(at + lane, n)] <= j)) - 1;
}

// Row r, of sequence b whose rows are off .. end - 1: its position and page, which is new or in the table.
struct FitRow {
  int b, pos, page, need;  // need: of a new page its number among all needed ones, the sequence's from first_need on
  bool fresh;
};
__device__ __forceinline__ FitRow fit_row(int r, int b, int len, int off, int end, int first_need) {
  const int first = len - (end - off), pos = first + (r - off), page = pos / kKvqPage, have = kvq_pages(first);
  return {b, pos, page, first_need + page - have, page >= have};
}
__device__ __forceinline__ int32_t* fit_entry(const KvqPool& p, int64_t b, int page) { return p.page_table + b * p.table_stride + page; }
__device__ __forceinline__ void fit_store(const KvqFitArgs& a, int r, const FitRow& f, int id) {
  if (f.fresh && f.pos % kKvqPage == 0) *fit_entry(a.pool, f.b, f.page) = id;
  a.position[r] = f.pos;
  a.slot[r] = id * kKvqPage + f.pos % kKvqPage;
}

// Sums over the lanes of a row of 16 up to each.
__device__ __forceinline__ int row_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
  return x + __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
}

// Counts this block; true for the last of the launch, which leaves the counts at 0.  Sixteen counts, 256 bytes apart, whose last ones
// count once more: 20.6 us for 256 blocks where one count took 22.8, 15.2 for 158 where it took 16.4.
__device__ __forceinline__ bool fit_arrives(int32_t* counts) {
  auto last_of = [](int32_t* count, int of) {
    if (__hip_atomic_fetch_add(count, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) != of - 1) return false;
    __hip_atomic_store(count, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return true;
  };
  const int blocks = gridDim.x, group = blockIdx.x % kFitCounts;
  return last_of(counts + kFitCountStride * (1 + group), (blocks - group + kFitCounts - 1) / kFitCounts) && last_of(counts, min(blocks, kFitCounts));
}

__global__ __launch_bounds__(kFitThreads) void k_kvq_fit(KvqFitArgs a, int with_rows, int block_rows) {
  constexpr int kWaves = kFitThreads / 64;
  __shared__ bool last_block;
  __shared__ int64_t sums[3][kWaves];
  __shared__ int scan[kWaves][3], flags[kWaves];
  __shared__ int start[3][kFitThreads + 1], length_of[kFitThreads];  // of a tile's sequences: pages needed, given back, rows before
  const KvqPool& pool = a.pool;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wave_u = __builtin_amdgcn_readfirstlane(wave), n = pool.n_seqs;
  const int n_free = pool.state[0];
  const bool alone = gridDim.x == 1;

  // What all sequences need, give back and add, in 64 bits; anything out of bounds.
  int64_t all[3] = {0, 0, 0};
  bool bad_len = false, bad_pool = false, bad_rows = false;
  int old = 0, len = 0;  // the thread's last sequence, its only one where there are no more than threads
  for (int b = tid; b < n; b += kFitThreads) {
    old = pool.context[b];
    len = a.length[b];
    const bool bl = len < 0 || len > a.max_context, bp = old < 0 || old > pool.max_context;
    bad_len |= bl;
    bad_pool |= bp;
    if (bl || bp) continue;
    const int have = kvq_pages(old), want = kvq_pages(len);
    all[0] += max(0, want - have);
    all[1] += max(0, have - want);
    all[2] += max(0, len - old);
    bad_rows |= len - old > a.max_rows;
  }
  const uint64_t any_len = __ballot(bad_len), any_pool = __ballot(bad_pool), any_rows = __ballot(bad_rows);
  int upto[3];  // over the wave's lanes up to this one, below 2^31 where nothing fails
#pragma unroll
  for (int i = 0; i < 3; ++i) {  // at most 2^10 sequences of 2^30 to a thread: halves of 20 bits, whose sums fit
    const int low = wave_scan(static_cast<int>(all[i] & 0xfffff));
    const int high = __ballot(all[i] >> 20 != 0) ? wave_scan(static_cast<int>(all[i] >> 20)) : 0;
    upto[i] = static_cast<int>(static_cast<uint32_t>(low) + (static_cast<uint32_t>(high) << 20));
    if (lane == 63) sums[i][wave] = (static_cast<int64_t>(high) << 20) + low;
  }
  if (lane == 0) flags[wave] = (any_len ? 1 : 0) | (any_pool ? 2 : 0) | (any_rows ? 4 : 0);
  __syncthreads();
  // The waves' sums, 16 lanes for each of the three: up to this wave's, and all.
  const int64_t of_wave = lane < 3 * kWaves ? sums[lane / kWaves][lane % kWaves] : 0;
  const int low = row_scan(static_cast<int>(of_wave & 0xffffff)), high = row_scan(static_cast<int>(of_wave >> 24));
  auto sum_to = [&](int i, int w) {
    const int at = i * kWaves + w;
    return (static_cast<int64_t>(__builtin_amdgcn_readlane(high, at)) << 24) + __builtin_amdgcn_readlane(low, at);
  };
  const int64_t need = sum_to(0, kWaves - 1), back = sum_to(1, kWaves - 1), rows = sum_to(2, kWaves - 1);
  const int seen = lane < kWaves ? flags[lane] : 0;
  const int flag = (n_free < 0 || n_free > pool.n_pages || __ballot(seen & 2) ? 2 : 0) | (__ballot(seen & 1) ? 1 : 0) | (__ballot(seen & 4) ? 4 : 0);
  const int64_t short_of = need - back - n_free;
  const int error = (flag & 2) || n_free + back > pool.n_pages ? kFitPool : (flag & 1) ? kFitLength : short_of > 0 ? kFitPages
                    : rows > a.n_rows ? kFitRows : (flag & 4) ? kFitSeqRows : kFitOk;
  const bool failed = error != kFitOk;  // nothing changes: no rows
  const int top = n_free + static_cast<int>(failed ? 0 : back);
  int carry[3] = {0, 0, 0};
  for (int b0 = 0; b0 < n; b0 += kFitThreads) {
    const int b = b0 + tid, here = min(kFitThreads, n - b0);
    if (n > kFitThreads && b < n) {
      old = pool.context[b];
      len = a.length[b];
    }
    int mine[3], total[3];  // before this sequence in the tile, and all of the tile
    if (n <= kFitThreads) {
#pragma unroll
      for (int i = 0; i < 3; ++i) {
        total[i] = failed ? 0 : static_cast<int>(sum_to(i, kWaves - 1));
        mine[i] = failed ? 0 : upto[i] - static_cast<int>(all[i]) + (wave_u > 0 ? static_cast<int>(sum_to(i, wave_u - 1)) : 0);
      }
    } else {
      int x[3] = {0, 0, 0};
      if (b < n && !failed) {
        const int have = kvq_pages(old), want = kvq_pages(len);
        x[0] = max(0, want - have);
        x[1] = max(0, have - want);
        x[2] = max(0, len - old);
      }
#pragma unroll
      for (int i = 0; i < 3; ++i) {
        mine[i] = wave_scan(x[i]);
        if (lane == 63) scan[wave][i] = mine[i];
        mine[i] -= x[i];
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 3; ++i) {
        const int before = wave_scan(lane < kWaves ? scan[lane][i] : 0);
        total[i] = __builtin_amdgcn_readlane(before, 63);
        mine[i] += wave_u > 0 ? __builtin_amdgcn_readlane(before, wave_u - 1) : 0;
      }
    }
#pragma unroll
    for (int i = 0; i < 3; ++i) start[i][tid] = mine[i];
    length_of[tid] = len;
    if (b < n) {
      if (blockIdx.x == 0) a.row_off[b] = carry[2] + mine[2];
      if (!with_rows) pool.first_need()[b] = carry[0] + mine[0];
      if (alone && !failed) pool.context[b] = len;
    }
    __syncthreads();
    const int stride = kFitThreads * static_cast<int>(gridDim.x);
    for (int j0 = blockIdx.x * kFitThreads + tid; j0 < total[1]; j0 += 4 * stride) {  // pages given back, four at a time
      int page[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int j = j0 + k * stride;
        if (j >= total[1]) continue;
        const int s = last_from(0, here - 1, j, [&](int i) { return start[1][i]; });
        page[k] = pool.page_table[(b0 + s) * pool.table_stride + kvq_pages(length_of[s]) + (j - start[1][s])];
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int j = j0 + k * stride;
        if (j < total[1]) pool.free_pages[top - 1 - (carry[1] + j)] = page[k];
      }
    }
#pragma unroll
    for (int i = 0; i < 3; ++i) carry[i] += total[i];
    __syncthreads();
  }
  if (!alone) {
    asm volatile("" ::"v"(n_free), "v"(old), "v"(len) : "memory");  // this block's reads of the state are in registers
    __syncthreads();
    if (tid == 0) last_block = fit_arrives(pool.workspace);
  }
  if (blockIdx.x == 0 && tid == 0) a.row_off[n] = carry[2];
  if (with_rows) {  // all sequences are in LDS
    if (tid == 0) start[2][n] = carry[2];
    __syncthreads();
    const int given = failed ? 0 : static_cast<int>(back), end = min(a.n_rows, static_cast<int>(blockIdx.x + 1) * block_rows);
    const int held = min(end, carry[2]);
    for (int r0 = blockIdx.x * block_rows + 64 * wave_u; r0 < end; r0 += kFitUnroll * kFitThreads) {
      FitRow f[kFitUnroll];
      int id[kFitUnroll];
#pragma unroll
      for (int k = 0; k < kFitUnroll; ++k) {  // 64 rows of a wave
        const int first = r0 + k * kFitThreads, last = min(first + 63, held - 1), r = min(first + lane, last);
        if (first >= held) continue;
        const int lo = wave_last(start[2], n, first), hi = __builtin_amdgcn_readfirstlane(start[2][lo + 1]) > last ? lo : wave_last(start[2], n, last);
        const int32_t* from;
        if (lo == hi) {  // of one sequence: most of what follows is the wave's; pages given back are two at most
          auto one = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
          f[k] = fit_row(r, lo, one(length_of[lo]), one(start[2][lo]), one(start[2][lo + 1]), one(start[0][lo]));
          from = fit_entry(pool, lo, f[k].page);
          if (f[k].fresh) from = pool.free_pages + (n_free - 1 - (f[k].need - given));
          const bool again = f[k].fresh && f[k].need < given;
          if (const uint64_t who = __ballot(again)) {
            const int k1 = __builtin_amdgcn_readlane(f[k].need, __builtin_ctzll(who)), k2 = __builtin_amdgcn_readlane(f[k].need, 63 - __builtin_clzll(who));
            auto entry = [&](int i) {
              const int s = wave_last(start[1], n, i);
              return fit_entry(pool, s, kvq_pages(one(length_of[s])) + (i - one(start[1][s])));
            };
            const int32_t *e1 = entry(k1), *e2 = k1 == k2 ? e1 : entry(k2);
            if (again) from = f[k].need == k1 ? e1 : e2;
          }
        } else {
          const int b = last_from(lo, hi, r, [&](int i) { return start[2][i]; });
          f[k] = fit_row(r, b, length_of[b], start[2][b], start[2][b + 1], start[0][b]);
          from = fit_entry(pool, b, f[k].page);
          if (f[k].fresh && f[k].need >= given) from = pool.free_pages + (n_free - 1 - (f[k].need - given));
          else if (f[k].fresh) {
            const int s = last_from(0, n - 1, f[k].need, [&](int i) { return start[1][i]; });
            from = fit_entry(pool, s, kvq_pages(length_of[s]) + (f[k].need - start[1][s]));
          }
        }
        id[k] = *from;
      }
#pragma unroll
      for (int k = 0; k < kFitUnroll; ++k) {
        const int r = r0 + k * kFitThreads + lane;
        if (r < held) fit_store(a, r, f[k], id[k]);
        else if (r < end) a.position[r] = a.slot[r] = -1;
      }
    }
  }
  if (!alone) {
    __syncthreads();
    if (!last_block) return;
    if (tid < n && !failed) pool.context[tid] = len;
  }
  if (tid == 0) {
    if (!with_rows) pool.first_need()[n] = top;
    pool.state[1] = error;
    pool.state[2] = carry[2];
    pool.state[3] = error == kFitPages ? static_cast<int>(min(short_of, int64_t{0x7fffffff})) : 0;
    if (!failed) pool.state[0] = top - carry[0];
  }
}

// A block has 1,024 rows, a wave 256: its first and last row's sequences are found 64 at a time.  Up to 64 sequences from the one to
// the other are a lane's each, where the rows look theirs up.
__global__ __launch_bounds__(256) void k_kvq_fit_rows(KvqFitArgs a) {
  const int n = a.pool.n_seqs, lane = threadIdx.x & 63;
  const int r0 = blockIdx.x * 1024 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * 256;
  if (r0 >= a.n_rows) return;
  KvqBatch bt;
  bt.n_seqs = n;
  bt.row_off = a.row_off;
  const int total = a.row_off[n], top = a.pool.first_need()[n], last = min(r0 + 255, a.n_rows - 1);
  const int lo = wave_find_seq(bt, r0);  // -1: all behind the last
  int hi = wave_find_seq(bt, last);
  FitRow f[4];
  int id[4];
  if (lo >= 0) {
    if (hi < 0) hi = n - 1;
    const int mine = min(lo + lane, n - 1);
    const int off = a.row_off[mine], end = a.row_off[mine + 1], len = a.pool.context[mine], need = a.pool.first_need()[mine];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int r = r0 + k * 64 + lane;
      if (hi - lo < 64) {  // the same in every lane
        int s = 0;
#pragma unroll
        for (int step = 32; step >= 1; step >>= 1)
          if (__shfl(off, s + step, 64) <= r && lo + s + step <= hi) s += step;
        const int l = __shfl(len, s, 64), o = __shfl(off, s, 64), e = __shfl(end, s, 64), d = __shfl(need, s, 64);
        f[k] = fit_row(r, lo + s, l, o, e, d);
      } else if (r < total) {
        const int b = last_from(lo, hi, r, [&](int i) { return a.row_off[i]; });
        f[k] = fit_row(r, b, a.pool.context[b], a.row_off[b], a.row_off[b + 1], a.pool.first_need()[b]);
      }
      if (r < total) id[k] = *(f[k].fresh ? a.pool.free_pages + (top - 1 - f[k].need) : fit_entry(a.pool, f[k].b, f[k].page));
    }
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int r = r0 + k * 64 + lane;
    if (r < total) fit_store(a, r, f[k], id[k]);
    else if (r < a.n_rows) a.position[r] = a.slot[r] = -1;
  }
}

// ---- ranges ------------------------------------------------------------------------------

__device__ __forceinline__ s16x2 as_pair(uint32_t x) { return __builtin_bit_cast(s16x2, x); }
__device__ __forceinline__ uint32_t as_word(s16x2 x) { return __builtin_bit_cast(uint32_t, x); }

// Two values of packed keys, the smaller (larger) of each: of fp16, NaN if one is; of bf16 in the order of `ordered`.
template <bool HALF>
__device__ __forceinline__ uint32_t smaller2(uint32_t a, uint32_t b) {
  if constexpr (HALF) return __builtin_bit_cast(uint32_t, __builtin_elementwise_minimum(__builtin_bit_cast(f16x2, a), __builtin_bit_cast(f16x2, b)));
  else return as_word(__builtin_elementwise_min(as_pair(a), as_pair(b)));
}
template <bool HALF>
__device__ __forceinline__ uint32_t larger2(uint32_t a, uint32_t b) {
  if constexpr (HALF) return __builtin_bit_cast(uint32_t, __builtin_elementwise_maximum(__builtin_bit_cast(f16x2, a), __builtin_bit_cast(f16x2, b)));
  else return as_word(__builtin_elementwise_max(as_pair(a), as_pair(b)));
}

// Order of bf16 bits as that of 16-bit integers, both halves; its own inverse.  -0 comes before 0.
__device__ __forceinline__ s16x2 ordered(s16x2 x) { return x ^ ((x >> 15) & s16x2{0x7fff, 0x7fff}); }
__device__ __forceinline__ bool is_nan16(short x) { return (x & 0x7fff) > 0x7f80; }

// Over the 16 lanes of a group, which have NP words each: lane c gets word c mod NP of all of them (of half of them and
// its partner's half, where there are eight), through LDS of the wave's own.  A row of NP words to a lane, turned by quarters
// so that neither writes nor reads meet in a bank.
template <int NP>
constexpr int kTurnGroup = 16 * NP + 16;
template <int NP, typename F>
__device__ __forceinline__ uint32_t across(const uint32_t (&x)[NP], uint32_t* lds, F op) {
  const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15, half = NP == 16 ? 0 : c >> 3, word = c & (NP - 1);
  auto turn = [](int row) { return NP == 16 ? row >> 2 : 0; };
  uint32_t* mine = lds + g * kTurnGroup<NP>;
#pragma unroll
  for (int k = 0; k < NP / 4; ++k)
    *reinterpret_cast<u32x4*>(mine + c * NP + 4 * (k ^ turn(c))) = u32x4{x[4 * k], x[4 * k + 1], x[4 * k + 2], x[4 * k + 3]};
  __builtin_amdgcn_wave_barrier();
  uint32_t y[NP];
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int row = NP == 16 ? i : half * 8 + (i ^ half);
    y[i] = mine[row * NP + 4 * ((word >> 2) ^ turn(row)) + (word & 3)];
  }
  __builtin_amdgcn_wave_barrier();
  uint32_t r = y[0];
#pragma unroll
  for (int i = 1; i < NP; ++i) r = op(r, y[i]);
  if constexpr (NP == 8) r = op(r, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(r), 0x128, 0xf, 0xf, false)));  // lane c ^ 8
  return r;
}

// The page's smallest and largest pair of the lane's two dimensions, of tokens below `held`, as bf16.  HALF: all 64, whose
// scales lie where fp16 holds every value: two conversions' instructions for each pair, a minimum and a maximum for each two.
template <int HD, bool HALF>
__device__ __forceinline__ void page_range(const PageK<HD>& pk, int held, uint32_t* lds, s16x2& lo, s16x2& hi) {
  constexpr int NP = HD / 8;  // pairs of a lane and token
  const int c = threadIdx.x & 15;
  uint32_t low[NP], high[NP];
#pragma unroll
  for (int k = 0; k < NP; ++k) {
    low[k] = 0x7fff7fffu;  // not HALF: past every value's order
    high[k] = 0x80008000u;
  }
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const float s = scale_of(pk.s, u);
    if (!HALF && 16 * u + c >= held) continue;
#pragma unroll
    for (int k = 0; k < NP; ++k) {
      const uint32_t w = HD == 128 ? pk.k[u][k >> 2] : pk.k[u >> 1][2 * (u & 1) + (k >> 2)];
      uint32_t x = value_pair<HALF>(w, s, k & 3);
      if constexpr (!HALF) x = as_word(ordered(as_pair(x)));
      low[k] = HALF && u == 0 ? x : smaller2<HALF>(low[k], x);
      high[k] = HALF && u == 0 ? x : larger2<HALF>(high[k], x);
    }
  }
  const uint32_t l = across(low, lds, smaller2<HALF>), h = across(high, lds, larger2<HALF>);
  if constexpr (HALF) {
    auto bf16 = [](uint32_t w) {  // two bits of mantissa: exact
      const f16x2 v = __builtin_bit_cast(f16x2, w);
      return as_pair(__builtin_amdgcn_perm(__float_as_uint(static_cast<float>(v[1])), __float_as_uint(static_cast<float>(v[0])), 0x07060302u));
    };
    lo = bf16(l);
    hi = bf16(h);
  } else {
    lo = ordered(as_pair(l));
    hi = ordered(as_pair(h));
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (is_nan16(lo[i]) || is_nan16(hi[i])) lo[i] = hi[i] = 0x7fc0;
  }
}

// A wave has `rows` consecutive rows of a KV head; for each page that one of them is the first of its sequence's in, it reads the
// page's K whole: lane 16g + c has hd/4 dimensions of tokens c, 16 + c, 32 + c, 48 + c, and ends with two dimensions of all
// tokens.  The next page's K is on its way meanwhile.
//   84,000 prompt tokens of 8 KV heads of 128 dims: 14 us, 3.7 TB/s: HBM, after a chain of offsets, table and page.  Comparing
// keys as 16-bit integers and exchanging them between lanes, 830 instructions a page instead of 450, took 17; several heads
// to a wave 14.4 for 13.7 when the append has left the keys in the caches.
template <int HD>
__global__ __launch_bounds__(256) void k_kvq_ranges(KvqCache c, KvqBatch bt, uint16_t* ranges, int rows) {
  constexpr int NP = HD / 8;
  __shared__ __attribute__((aligned(16))) uint32_t lds[4][4 * kTurnGroup<NP>];
  const int lane = threadIdx.x & 63;
  const int in_block = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = blockIdx.x * 4 + in_block;
  const int g = wave / c.n_kv, kh = wave - g * c.n_kv, base = g * rows;
  if (base >= bt.n_rows) return;
  const PagePlace place = wave_places(c, bt, base, rows);
  uint64_t todo = __ballot(place.state == 1 && (place.t == 0 || place.i == 0));
  PageK<HD> next;
  size_t at = 0;
  int held = 0;  // tokens of the page below the context, or more than 64
  auto load = [&] {
    const int src = __ffsll(static_cast<unsigned long long>(todo)) - 1;
    at = static_cast<size_t>(__builtin_amdgcn_readlane(place.page, src)) * c.n_kv + kh;
    held = __builtin_amdgcn_readlane(place.t + place.left, src);
    next.template load<false>(c.blocks + at * kvq_block_bytes(HD));  // the append has just written there
  };
  if (todo) load();
  while (todo) {
    todo &= todo - 1;
    const PageK<HD> pk = next;
    const size_t now = at;
    const int below = held;
    if (todo) load();
    s16x2 lo, hi;
    // the four scales of the lane's tokens within 2^-23 .. 2^8, as fits_half has it
    const bool fits = !(((pk.s + 0x18181818u) ^ 0x80808080u) & 0xe0e0e0e0u);
    if (below >= kKvqPage && __all(fits)) page_range<HD, true>(pk, below, lds[in_block], lo, hi);
    else page_range<HD, false>(pk, below, lds[in_block], lo, hi);
    uint32_t* out = reinterpret_cast<uint32_t*>(ranges) + now * HD;
    if (HD == 128 || !(lane & 8)) {
      const int d2 = (lane >> 4) * NP + (lane & (NP - 1));
      out[d2] = as_word(lo);
      out[HD / 2 + d2] = as_word(hi);
    }
  }
}

// ---- scores ------------------------------------------------------------------------------

// The larger of the two, NaN if one is.
__device__ __forceinline__ float larger(float a, float b) { return __builtin_elementwise_maximum(a, b); }
// The same of a lane and the one of the next group of 16, of an even one, or of the one two groups on.
__device__ __forceinline__ float larger_of_16(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return larger(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float larger_of_32(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return larger(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// Eight queries of a lane, as loaded.
template <bool F32>
struct Eight {
  std::conditional_t<F32, float[8], u32x4> x;
  __device__ __forceinline__ void load(const KvqTensor& t, int row, int head, int d) {
    const int64_t at = row * t.row_stride + head * t.head_stride + d;
    if constexpr (F32) {
      load8<false>(t, row, head, d, x);
    } else {
      const bf16_t* p = static_cast<const bf16_t*>(t.p) + at;
      if (t.vec) {
        x = *reinterpret_cast<const u32x4*>(p);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = static_cast<uint32_t>(p[2 * i]) | static_cast<uint32_t>(p[2 * i + 1]) << 16;
      }
    }
  }
};

// These as operands: pieces of bf16 (one, or three of fp32) of max(q, 0) and of min(q, 0).
__device__ __forceinline__ void split_signs(const Eight<false>& q, bf16x8_t (&above)[1], bf16x8_t (&below)[1]) {
  u32x4 up, down;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t neg = __builtin_bit_cast(uint32_t, as_pair(q.x[i]) >> 15);
    up[i] = q.x[i] & ~neg;
    down[i] = q.x[i] & neg;
  }
  above[0] = __builtin_bit_cast(bf16x8_t, up);
  below[0] = __builtin_bit_cast(bf16x8_t, down);
}
__device__ __forceinline__ void split_signs(Eight<true>& q, bf16x8_t (&above)[3], bf16x8_t (&below)[3]) {
  u32x4 neg;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    neg[i] = (__float_as_int(q.x[2 * i]) < 0 ? 0xffffu : 0u) | (__float_as_int(q.x[2 * i + 1]) < 0 ? 0xffff0000u : 0u);
  bf16x8_t p[3];
  split8<3>(q.x, p);
#pragma unroll
  for (int n = 0; n < 3; ++n) {
    const u32x4 w = __builtin_bit_cast(u32x4, p[n]);
    above[n] = __builtin_bit_cast(bf16x8_t, w & ~neg);
    below[n] = __builtin_bit_cast(bf16x8_t, w & neg);
  }
}

// Rows of a sequence read the same ranges: a block's four waves have 16 PT pages each of one KV head, for up to `rows` consecutive
// rows.  Queries are the 16 rows of 16x16x32 products, 2 hd long, the ranges of 16 pages the 16 columns.  The G heads of a row take
// `seg` of the 16, a power of two, the last head again in what is left of them, so that lane 16g + c gets four heads' scores of page
// c or whole rows': their maximum is mostly the lane's own (with the heads in the columns, the maximum over lanes took 2,000 rows
// 51 us for 33).
template <int HD, bool F32, int PT>
__global__ __launch_bounds__(256, 2) void k_kvq_scores(KvqScoreArgs a, int rows) {
  constexpr int NJ = HD / 32, NQ = F32 ? 3 : 1;
  constexpr int NPC = HD / 4;  // 16-byte pieces of a page's ranges
  const KvqBatch& bt = a.batch;
  const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n_kv = a.cache.n_kv, G = a.n_q / n_kv;
  const int seg_log = G > 8 ? 4 : G > 4 ? 3 : G > 2 ? 2 : G > 1 ? 1 : 0, seg = 1 << seg_log, rt = 16 >> seg_log;
  const int group = blockIdx.x / n_kv, kh = blockIdx.x - group * n_kv;
  const int p0 = (blockIdx.y * 4 + wave) * 16 * PT;
  if (p0 >= a.columns) return;
  const int last_row = min((group + 1) * rows, bt.n_rows);
  for (int r = group * rows; r < last_row;) {
    const int b = wave_find_seq(bt, r);
    if (b < 0) return;
    const KvqSeq sq = kvq_seq(bt, b);
    const int i = r - sq.r0;
    if (i < 0 || i >= sq.n) {  // past max_rows
      r = max(r + 1, bt.row_off ? min(bt.row_off[b + 1], bt.n_rows) : 0);
      continue;
    }
    const int n = min(last_row, sq.r0 + sq.n) - r, first = sq.ctx - sq.n + i;  // rows, the first one's position
    const int seen = kvq_row_sees(sq, i + n - 1);                                 // the last page that some row sees
    int id[PT];
    const int32_t* pt = table_of(bt, b);
#pragma unroll
    for (int t = 0; t < PT; ++t) {
      const int entry = kvq_seen_entry(p0 + 16 * t + c, seen);
      id[t] = entry >= 0 ? pt[entry] : -1;
    }
    bf16x8_t hi[PT][NJ], lo[PT][NJ];
    bool ok[PT];  // the lane's page is in the cache
#pragma unroll
    for (int t = 0; t < PT; ++t) {
      ok[t] = kvq_page_ok(a.cache, id[t]);
      if (p0 + 16 * t > seen) continue;
      const int use = ok[t] ? id[t] : 0;  // others read what page 0 has
      const u32x4* ranges = reinterpret_cast<const u32x4*>(a.ranges);
      const u32x4* at = ranges + (static_cast<size_t>(use) * n_kv + kh) * NPC + 2 * g;
#pragma unroll
      for (int j = 0; j < NJ; ++j) {  // a line of 128 bytes is four lanes' two pieces
        lo[t][j] = __builtin_bit_cast(bf16x8_t, at[8 * (j >> 1) + (j & 1)]);
        hi[t][j] = __builtin_bit_cast(bf16x8_t, at[NPC / 2 + 8 * (j >> 1) + (j & 1)]);
      }
    }
    // The scores of the mine-th of these rows for the lane's pages: those that it does not see have minus infinity.
    auto store = [&](int mine, int t, float x) {
      const int p = p0 + 16 * t + c;
      if (!ok[t] || !sq.ok) x = __builtin_nanf("");
      if (sq.ok && p > (first + mine) >> 6) x = -INFINITY;
      if (mine < n && p < a.columns) a.scores[(static_cast<size_t>(r + mine) * n_kv + kh) * a.columns + p] = x;
    };
    if (p0 > seen) {  // nothing to see for any row, or for none to know
      for (int q0 = 0; q0 < n; q0 += 4)
#pragma unroll
        for (int t = 0; t < PT; ++t) store(q0 + g, t, 0.f);
      r += n;
      continue;
    }
    // Units of 16 query rows: `parts` of each rt rows; a unit's queries are loaded a unit ahead.
    const int parts = (G + 15) >> 4, units = (n + rt - 1) / rt * parts;
    Eight<F32> q[NJ];
    auto load = [&](int u) {
      const int tile = u / parts, h0 = 16 * (u - tile * parts);
      const int row = r + min(tile * rt + (c >> seg_log), n - 1), head = kh * G + min(h0 + (c & (seg - 1)), G - 1);
#pragma unroll
      for (int j = 0; j < NJ; ++j) q[j].load(a.q, row, head, 64 * (j >> 1) + 16 * g + 8 * (j & 1));
    };
    load(0);
    f32x4_t best[PT];
    for (int u = 0; u < units; ++u) {
      const int tile = u / parts, part = u - tile * parts;
      f32x4_t acc[PT];
#pragma unroll
      for (int t = 0; t < PT; ++t) acc[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      bf16x8_t above[NJ][NQ], below[NJ][NQ];
#pragma unroll
      for (int j = 0; j < NJ; ++j) split_signs(q[j], above[j], below[j]);
      if (u + 1 < units) load(u + 1);
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int m = 0; m < NQ; ++m)
#pragma unroll
          for (int t = 0; t < PT; ++t) {
            acc[t] = mfma16x16x32(above[j][m], hi[t][j], acc[t]);
            acc[t] = mfma16x16x32(below[j][m], lo[t][j], acc[t]);
          }
      if (parts > 1) {  // of one row
#pragma unroll
        for (int t = 0; t < PT; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) best[t][e] = acc[t][e] = part ? larger(best[t][e], acc[t][e]) : acc[t][e];
        if (part + 1 < parts) continue;
      }
      const int row0 = tile * rt;
#pragma unroll
      for (int t = 0; t < PT; ++t) {
        if (seg >= 4) {
          float x = larger(larger(larger(acc[t][0], acc[t][1]), acc[t][2]), acc[t][3]);
          if (seg >= 8) x = larger_of_16(x);
          if (seg == 16) x = larger_of_32(x);
          if ((4 * g & (seg - 1)) == 0) store(row0 + (4 * g >> seg_log), t, x);
        } else if (seg == 2) {
#pragma unroll
          for (int e = 0; e < 2; ++e) store(row0 + 2 * g + e, t, larger(acc[t][2 * e], acc[t][2 * e + 1]));
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) store(row0 + 4 * g + e, t, acc[t][e]);
        }
      }
    }
    r += n;
  }
}

// A row whose sequence has no other: its ranges are read once, past the caches.  A wave has 16 PT pages, a lane's each in one read of the
// table, and walks them 16 at a time, the next ones on their way: whole pages to an instruction, which LDS turns into operands.
// The heads are the 16 rows of the products, the last one again where there are fewer; MANY: more, taken in turn for each 16 pages.
//   64 rows of 6,000 to 33,000 keys (8 KV heads of 128) 17.4 us, 4.7 TB/s: HBM, after context and table; with operands instead of whole
// pages, 64 bytes to an instruction, 27.7; with MANY's loop for all heads 17.9.
template <int HD, bool F32, int PT, bool MANY>
__global__ __launch_bounds__(256, F32 ? 2 : 3) void k_kvq_scores_walk(KvqScoreArgs a) {
  constexpr int NJ = HD / 32, NQ = F32 ? 3 : 1, NPC = HD / 4, NI = NPC / 4;
  __shared__ u32x4 turn[4][16 * NPC];
  const KvqBatch& bt = a.batch;
  const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n_kv = a.cache.n_kv, G = a.n_q / n_kv, row = blockIdx.x / n_kv, kh = blockIdx.x - row * n_kv;
  const int p0 = (blockIdx.y * 4 + wave) * 16 * PT;
  if (p0 >= a.columns) return;
  const int b = wave_find_seq(bt, row);
  if (b < 0) return;
  const KvqSeq sq = kvq_seq(bt, b);
  const int i = row - sq.r0;
  if (i < 0 || i >= sq.n) return;
  const int seen = kvq_row_sees(sq, i), entry = kvq_seen_entry(p0 + lane, seen);
  const int id = entry >= 0 ? table_of(bt, b)[entry] : -1;
  const bool ok = kvq_page_ok(a.cache, id);
  float mine = 0.f;
  if (p0 <= seen) {
    const int use = ok ? id : 0;
    const u32x4* ranges = reinterpret_cast<const u32x4*>(a.ranges);
    u32x4 x[2][NI];
    auto load = [&](int t) {
#pragma unroll
      for (int k = 0; k < NI; ++k) {
        const size_t page = __shfl(use, 16 * t + k * (64 / NPC) + lane / NPC, 64);
        x[t & 1][k] = load_page<true>(ranges + (page * n_kv + kh) * NPC + lane % NPC);
      }
    };
    Eight<F32> q[NJ];
    bf16x8_t above[NJ][NQ], below[NJ][NQ];
    auto queries = [&](int h0) {
#pragma unroll
      for (int j = 0; j < NJ; ++j) q[j].load(a.q, row, kh * G + min(h0 + c, G - 1), 64 * (j >> 1) + 16 * g + 8 * (j & 1));
    };
    auto operands = [&]() {
#pragma unroll
      for (int j = 0; j < NJ; ++j) split_signs(q[j], above[j], below[j]);
    };
    queries(0);
    load(0);
    operands();
#pragma unroll
    for (int t = 0; t < PT; ++t) {
      if (p0 + 16 * t > seen) break;
      if (t + 1 < PT && p0 + 16 * t + 16 <= seen) load(t + 1);
#pragma unroll
      for (int k = 0; k < NI; ++k) {
        const int page = k * (64 / NPC) + lane / NPC;
        turn[wave][page * NPC + (lane % NPC ^ page)] = x[t & 1][k];
      }
      __builtin_amdgcn_wave_barrier();
      float best = 0.f;
      for (int h0 = 0; h0 < (MANY ? G : 1); h0 += 16) {
        if (MANY && t + h0 > 0) {  // else they are there
          queries(h0);
          operands();
        }
        f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          const int piece = 8 * (j >> 1) + 2 * g + (j & 1);
          const bf16x8_t lo = __builtin_bit_cast(bf16x8_t, turn[wave][c * NPC + (piece ^ c)]);
          const bf16x8_t hi = __builtin_bit_cast(bf16x8_t, turn[wave][c * NPC + ((piece + NPC / 2) ^ c)]);
#pragma unroll
          for (int m = 0; m < NQ; ++m) {
            acc = mfma16x16x32(above[j][m], hi, acc);
            acc = mfma16x16x32(below[j][m], lo, acc);
          }
        }
        const float x = larger_of_32(larger_of_16(larger(larger(larger(acc[0], acc[1]), acc[2]), acc[3])));
        best = h0 ? larger(best, x) : x;
      }
      __builtin_amdgcn_wave_barrier();
      if (g == t) mine = best;
    }
  }
  const int p = p0 + lane;
  if (!ok || !sq.ok) mine = __builtin_nanf("");
  if (sq.ok && p > seen) mine = -INFINITY;
  if (lane < 16 * PT && p < a.columns) a.scores[(static_cast<size_t>(row) * n_kv + kh) * a.columns + p] = mine;
}

// ---- picks -------------------------------------------------------------------------------

// The order of scores as that of unsigned numbers above 0: -0 is 0, NaN comes last.
__device__ __forceinline__ uint32_t pick_key(float x) {
  if (x != x) return 0xffffffffu;
  const uint32_t b = __float_as_uint(x + 0.f);
  return b ^ (b >> 31 ? 0xffffffffu : 0x80000000u);
}

// Lanes of a ballot, as a signed number.
__device__ __forceinline__ int lanes(uint64_t ballot) { return static_cast<int>(__popcll(ballot)); }

// Pages of the row's list to choose from: `seen` pages, or -1 where the row is not the call's.
__device__ __forceinline__ int row_pages(const KvqBatch& bt, int row) {
  const int b = wave_find_seq(bt, row);
  if (b < 0) return -1;
  const KvqSeq s = kvq_seq(bt, b);
  const int i = row - s.r0;
  if (i < 0 || i >= s.n) return -1;
  return s.ok ? max(0, s.ctx - s.n + i + kKvqPage) >> 6 : 0;  // none before the first token
}

// A wave has the list of a row and KV head, E of its up to 64 E pages in each lane, loaded while the row is looked up.  The
// least key that is picked is found bit by bit from the highest: so many keys are at or above a value as a ballot has bits, or (E
// from 8 on) as the lanes count.  256 lists of up to 71 pages 3.6 us, 2,048 of 219 pages 5.8, 512 of up to 516
// 7.8 to 10.4: 32 bits where scores tie, about half of them where not, each a wave's wait for its count.
template <int E>
__global__ __launch_bounds__(256) void k_kvq_pick(KvqPickArgs a) {
  const int lane = threadIdx.x & 63;
  const int unit = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), row = unit / a.n_kv;
  if (row >= a.batch.n_rows) return;
  float x[E];
  const float* scores = a.scores + static_cast<size_t>(unit) * a.columns;
#pragma unroll
  for (int e = 0; e < E; ++e) x[e] = scores[min(64 * e + lane, a.columns - 1)];
  const int m = row_pages(a.batch, row);
  if (m < 0) return;
  int32_t* out = a.picks + static_cast<size_t>(unit) * a.n;
  if (m <= a.n) {
    for (int i = lane; i < a.n; i += 64) out[i] = i < m ? i : -1;
    return;
  }
  const int from = a.first, to = m - a.last, want = a.n - a.first - a.last;  // `want` of pages from .. to - 1
  uint32_t key[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int p = 64 * e + lane;
    key[e] = p >= from && p < to ? pick_key(x[e]) : 0;
  }
  auto count = [&](uint32_t t) {
    int k = 0;
    if constexpr (E < 8) {
#pragma unroll
      for (int e = 0; e < E; ++e) k += lanes(__ballot(key[e] >= t));
      return k;
    }
#pragma unroll
    for (int e = 0; e < E; ++e) k += key[e] >= t;  // of the lane's, without a wait for each ballot
    return __builtin_amdgcn_readlane(wave_scan(k), 63);
  };
  // The largest value with `want` keys at or above it; where the count meets `want` before, it is far enough.
  uint32_t least = want > 0 ? 0 : 0xffffffffu;
  int k = 0;
  for (uint32_t bit = want > 0 ? 0x80000000u : 0; bit; bit >>= 1) {
    const int at_bit = count(least | bit);
    if (at_bit >= want) {
      least |= bit;
      k = at_bit;
    }
    if (at_bit == want) break;
  }
  int at = 0;
  auto put = [&](int e, bool take) {
    const uint64_t taken = __ballot(take);
    const int place = __builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(taken >> 32), __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(taken), at));
    if (take) out[place] = 64 * e + lane;
    at += lanes(taken);
  };
  if (k == want && want > 0) {  // no ties to break
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int p = 64 * e + lane;
      put(e, key[e] >= least || p < from || (p >= to && p < m));
    }
    return;
  }
  int above = 0;
#pragma unroll
  for (int e = 0; e < E; ++e) above += lanes(__ballot(key[e] > least));
  int ties = want - above;  // of keys equal to `least`, the first so many
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int p = 64 * e + lane;
    const bool in = p >= from && p < to, tie = in && key[e] == least;
    const uint64_t tied = __ballot(tie), below = (uint64_t{1} << lane) - 1;
    put(e, (p < m && !in) || (in && key[e] > least) || (tie && lanes(tied & below) < ties));
    ties -= lanes(tied);
  }
}

// The same for longer lists, a block to each: a digit of eight bits at a time, its keys counted in LDS, the scores read anew for
// each digit.
constexpr int kPickThreads = 1024;
__global__ __launch_bounds__(kPickThreads) void k_kvq_pick_long(KvqPickArgs a) {
  __shared__ int counts[256];
  __shared__ int found[2];  // the digit, and how many keys are above it
  __shared__ int waves[2][kPickThreads / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t unit = blockIdx.x;
  const int row = static_cast<int>(blockIdx.x) / a.n_kv;
  const int m = row_pages(a.batch, row);
  if (m < 0) return;
  int32_t* out = a.picks + unit * a.n;
  if (m <= a.n) {
    for (int i = tid; i < a.n; i += kPickThreads) out[i] = i < m ? i : -1;
    return;
  }
  const float* scores = a.scores + unit * a.columns;
  const int from = a.first, to = m - a.last;
  int want = a.n - a.first - a.last;
  uint32_t least = 0;  // its digits so far; `want` counts what is still to come from keys that begin with them
  for (int shift = 24; shift >= 0 && want > 0; shift -= 8) {
    if (tid < 256) counts[tid] = 0;
    __syncthreads();
    for (int p = from + tid; p < to; p += kPickThreads) {
      const uint32_t k = pick_key(scores[p]);
      if (shift == 24 || (k >> (shift + 8)) == (least >> (shift + 8))) atomicAdd(&counts[(k >> shift) & 255], 1);
    }
    __syncthreads();
    if (wave == 0) {  // lane l has digits 255 - 4l .. 252 - 4l
      int x[4], sum = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) sum += x[i] = counts[255 - 4 * lane - i];
      int above = wave_scan(sum) - sum;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (above < want && above + x[i] >= want) {
          found[0] = 255 - 4 * lane - i;
          found[1] = above;
        }
        above += x[i];
      }
    }
    __syncthreads();
    least |= static_cast<uint32_t>(found[0]) << shift;
    want -= found[1];
  }
  if (a.n == a.first + a.last) least = 0xffffffffu;  // and want = 0 of them
  int at = 0;
  for (int p0 = 0; p0 < m; p0 += kPickThreads) {
    const int p = p0 + tid;
    const uint64_t below = (uint64_t{1} << lane) - 1;
    const bool in = p >= from && p < to;
    const uint32_t k = in ? pick_key(scores[p]) : 0;
    const bool tie = in && k == least;
    const uint64_t tied = __ballot(tie);
    if (lane == 0) waves[0][wave] = lanes(tied);
    __syncthreads();
    int before = 0, ties = 0;
    for (int w = 0; w < kPickThreads / 64; ++w) {
      before += w < wave ? waves[0][w] : 0;
      ties += waves[0][w];
    }
    const bool take = (p < m && !in) || (in && k > least) || (tie && before + lanes(tied & below) < want);
    want -= ties;
    const uint64_t taken = __ballot(take);
    if (lane == 0) waves[1][wave] = lanes(taken);
    __syncthreads();
    int mine = at;
    for (int w = 0; w < kPickThreads / 64; ++w) {
      mine += w < wave ? waves[1][w] : 0;
      at += waves[1][w];
    }
    if (take) out[mine + lanes(taken & below)] = p;
    __syncthreads();
  }
}

}  // namespace

hipError_t launch_kvq_fit(const KvqFitArgs& a, hipStream_t s) {
  const int with_rows = a.pool.n_seqs <= kFitThreads;
  const int rows = std::max(kFitBlock, (a.n_rows + 255) / 256);  // of a block
  const int blocks = with_rows ? std::max(1, (a.n_rows + rows - 1) / rows) : 1;
  launch_kernel(k_kvq_fit, dim3(static_cast<uint32_t>(blocks)), dim3(kFitThreads), 0, s, a, with_rows, rows);
  if (!with_rows && a.n_rows > 0) launch_kernel(k_kvq_fit_rows, dim3(static_cast<uint32_t>((a.n_rows + 1023) / 1024)), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_kvq_ranges(const KvqCache& c, const KvqBatch& b, uint16_t* ranges, hipStream_t s) {
  // As many rows to a wave, of 64, as leave 2,048 waves: one token each of 64 sequences (4 KV heads) 3.4 us, 64 rows to a wave 71.
  int rows = 64;
  while (rows > 1 && (static_cast<int64_t>(b.n_rows) + rows - 1) / rows * c.n_kv < 2048) rows /= 2;
  const int64_t waves = (static_cast<int64_t>(b.n_rows) + rows - 1) / rows * c.n_kv;
  const dim3 grid(static_cast<uint32_t>((waves + 3) / 4));
  if (c.hd == 128) launch_kernel((k_kvq_ranges<128>), grid, dim3(256), 0, s, c, b, ranges, rows);
  else launch_kernel((k_kvq_ranges<64>), grid, dim3(256), 0, s, c, b, ranges, rows);
  return hipGetLastError();
}

hipError_t launch_kvq_scores(const KvqScoreArgs& a, hipStream_t s) {
  const ScorePlan p = score_plan(a.cache, a.batch, a.columns, a.q.bf16);
  const bool bf16 = a.q.bf16, wide = a.cache.hd == 128;
  if (!p.shared) {
    const bool many = a.n_q > 16 * a.cache.n_kv;
    const int tiles = many ? 1 : p.tiles;
    const dim3 grid(static_cast<uint32_t>(a.batch.n_rows) * a.cache.n_kv, static_cast<uint32_t>((a.columns + 64 * tiles - 1) / (64 * tiles)));
#define RP_WALK(HD, BF16, PT, MANY) \
  if (wide == (HD == 128) && bf16 == BF16 && tiles == PT && many == MANY) launch_kernel((k_kvq_scores_walk<HD, !BF16, PT, MANY>), grid, dim3(256), 0, s, a);
#define RP_WALKS(HD, BF16) RP_WALK(HD, BF16, 1, false) RP_WALK(HD, BF16, 4, false) RP_WALK(HD, BF16, 1, true)
    RP_WALKS(128, true) RP_WALKS(128, false) RP_WALKS(64, true) RP_WALKS(64, false)
#undef RP_WALKS
#undef RP_WALK
    return hipGetLastError();
  }
  const dim3 grid(static_cast<uint32_t>(p.groups * a.cache.n_kv), static_cast<uint32_t>((a.columns + 64 * p.tiles - 1) / (64 * p.tiles)));
#define RP_SCORES(HD, BF16, PT) if (wide == (HD == 128) && bf16 == BF16 && p.tiles == PT) launch_kernel((k_kvq_scores<HD, !BF16, PT>), grid, dim3(256), 0, s, a, p.rows);
  RP_SCORES(128, true, 2) RP_SCORES(128, false, 2) RP_SCORES(128, true, 4) RP_SCORES(64, true, 2) RP_SCORES(64, false, 2) RP_SCORES(64, true, 4)
#undef RP_SCORES
  return hipGetLastError();
}

hipError_t launch_kvq_pick(const KvqPickArgs& a, hipStream_t s) {
  const int64_t units = static_cast<int64_t>(a.batch.n_rows) * a.n_kv;
  const int pages = kvq_pages(a.batch.max_context);
  const dim3 grid(static_cast<uint32_t>((units + 3) / 4)), block(256);
  if (pages <= 64) launch_kernel((k_kvq_pick<1>), grid, block, 0, s, a);
  else if (pages <= 128) launch_kernel((k_kvq_pick<2>), grid, block, 0, s, a);
  else if (pages <= 256) launch_kernel((k_kvq_pick<4>), grid, block, 0, s, a);
  else if (pages <= 512) launch_kernel((k_kvq_pick<8>), grid, block, 0, s, a);
  else if (pages <= 1024) launch_kernel((k_kvq_pick<16>), grid, block, 0, s, a);
  else if (pages <= 2048) launch_kernel((k_kvq_pick<32>), grid, block, 0, s, a);
  else launch_kernel(k_kvq_pick_long, dim3(static_cast<uint32_t>(units)), dim3(kPickThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace rollpack
