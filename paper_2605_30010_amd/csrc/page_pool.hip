// Pages for sequences that grow, shrink and end: page tables, positions and places of new tokens, built on the device from lengths.
#include <algorithm>

#include "kv_cache.h"
#include "select_common.h"

namespace et {

// What a resize works on.  Sequence b goes from old(b) to fresh(b) tokens and from pages(old) to pages(fresh) entries of its table row.
struct PoolArgs {
  int32_t *ring;
  int32_t *table;
  const int32_t *len, *new_len;
  int n_pages, page_shift, table_stride, pages_per_seq, n_seqs;
  __device__ __forceinline__ int pages(int tokens) const {
    return (int)min(((uint32_t)tokens + (1u << page_shift) - 1) >> page_shift, (uint32_t)pages_per_seq);
  }
  __device__ __forceinline__ bool is_page(int p) const { return p >= 0 && p < n_pages; }
  // cell of the ring: i below n_pages
  __device__ __forceinline__ int cell(int head, int i) const {
    const uint32_t c = (uint32_t)head + (uint32_t)i;
    return (int)(c >= (uint32_t)n_pages ? c - (uint32_t)n_pages : c);
  }
};
// The ring's free pages: count of them from cell head on, whatever the state holds.
struct PoolState {
  int head, count;
  __device__ __forceinline__ PoolState(const int32_t *state, int n_pages) {
    const int2 s = *reinterpret_cast<const int2 *>(state);
    head = (int)((uint32_t)s.x % (uint32_t)n_pages);
    count = min(max(s.y, 0), n_pages);
  }
};

constexpr int kPoolThreads = 1024, kPoolWaves = kPoolThreads / 64;

// Sums over the workgroup's threads before mine of three numbers, and the totals.  The first may pass 32 bits: its halves are added apart.
struct Triple {
  int64_t rows;
  int grow, shrink;
};
__device__ __forceinline__ Triple scan_threads(Triple mine, Triple &total, Triple (&lds)[kPoolWaves]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int low = wave_inclusive_scan((int)(mine.rows & 0xFFFF)), high = wave_inclusive_scan((int)(mine.rows >> 16));
  const int64_t r = ((int64_t)high << 16) + low;
  const int g = wave_inclusive_scan(mine.grow), s = wave_inclusive_scan(mine.shrink);
  if (lane == 63) lds[wave] = {r, g, s};
  __syncthreads();
  Triple before{0, 0, 0};
  total = {0, 0, 0};
#pragma unroll
  for (int w = 0; w < kPoolWaves; ++w) {
    if (w == wave) before = total;
    total.rows += lds[w].rows, total.grow += lds[w].grow, total.shrink += lds[w].shrink;
  }
  return {before.rows + r - mine.rows, before.grow + g - mine.grow, before.shrink + s - mine.shrink};
}
__device__ __forceinline__ int clipped(int64_t rows) { return (int)min(rows, (int64_t)INT32_MAX); }

// The largest s in [lo, hi] with first[s] <= x (first ascends, first[lo] <= x).
__device__ __forceinline__ int find_seq(const int *first, int lo, int hi, int x) {
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (first[mid] <= x) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// The same for all lanes of a wavefront together, 64 probes at a time.
__device__ __forceinline__ int find_seq_all(const int *first, int from, int n_seqs, int x) {
  const int lane = threadIdx.x & 63;
  int len = n_seqs - from;                               // the answer is in [from, from + len)
  while (len > 1) {
    const int step = (len + 63) / 64, i = from + lane * step;
    const int hits = __popcll(__ballot(lane * step < len && first[min(i, n_seqs - 1)] <= x));
    from += (hits - 1) * step;
    len = min(step, n_seqs - from);
  }
  return from;
}
// Gives pages behind sequences' ends back, in turns: of all `total` entries the workgroup takes up to 4096 from `back` on, a wavefront up to 256
// neighbours (their sequences lie between the first one's and the last one's).  Those that are pages go behind the ring's `count` free ones and the
// `given` before them, in order.  A turn's entries are on their way while the turn before is put into the ring.
constexpr int kGiveTurn = 4 * kPoolThreads;
__device__ __forceinline__ int given_each(int64_t back, int total) {        // entries of a wavefront
  return 64 * (int)min((total - back + kPoolThreads - 1) / kPoolThreads, (int64_t)4);
}
template <typename NewLength>
__device__ __forceinline__ void find_given(const PoolArgs &a, const int *shrink_first, int64_t back, int total, NewLength new_of, int (&page)[4]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, each = given_each(back, total);
  const int64_t k0 = back + wave * each;
#pragma unroll
  for (int u = 0; u < 4; ++u) page[u] = -1;
  if (k0 < total) {
    const int lo = find_seq_all(shrink_first, 0, a.n_seqs, (int)k0), hi = find_seq_all(shrink_first, lo, a.n_seqs, (int)min(k0 + each - 1, total - 1ll));
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int64_t k = k0 + u * 64 + lane;
      if (k < min(k0 + each, (int64_t)total)) {
        const int b = find_seq(shrink_first, lo, hi, (int)k);
        page[u] = a.table[(int64_t)b * a.table_stride + a.pages(new_of(b)) + ((int)k - shrink_first[b])];
      }
    }
  }
}
__device__ __forceinline__ void put_given(const PoolArgs &a, PoolState st, const int (&page)[4], int &given, int (&lds)[kPoolWaves]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, room = a.n_pages - st.count;
  uint64_t votes[4];
  int mine = 0;
#pragma unroll
  for (int u = 0; u < 4; ++u) mine += __popcll(votes[u] = __ballot(a.is_page(page[u])));
  if (lane == 0) lds[wave] = mine;
  __syncthreads();
  int at = given;
#pragma unroll
  for (int w = 0; w < kPoolWaves; ++w) {
    const int n = lds[w];
    if (w < wave) at += n;
    given += n;
  }
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int to = at + __popcll(votes[u] & ((1ull << lane) - 1));
    if ((votes[u] >> lane & 1) && to < room) a.ring[a.cell(st.head, st.count + to)] = page[u];
    at += __popcll(votes[u]);
  }
  __syncthreads();
}
// Entry i of all that are wanted: the ring's i-th page, or none.
__device__ __forceinline__ int taken_page(const PoolArgs &a, PoolState st, int i) { return i < st.count ? a.ring[a.cell(st.head, i)] : -1; }

__device__ __forceinline__ void leave_state(const PoolArgs &a, PoolState st, int wanted, int given, int32_t *state_out) {
  const int used = min(wanted, st.count);
  *reinterpret_cast<int4 *>(state_out) = make_int4((int)(((uint32_t)st.head + (uint32_t)used) % (uint32_t)a.n_pages),
                                                   st.count - used + min(given, a.n_pages - st.count), wanted - used, 0);
}
// Place of token `pos` whose page is `page`.
__device__ __forceinline__ int64_t slot_of(const PoolArgs &a, int page, int pos) {
  return a.is_page(page) ? ((int64_t)page << a.page_shift) + (pos & ((1 << a.page_shift) - 1)) : -1;
}

// Up to 1024 PER sequences: every workgroup adds up all of them by itself, PER to a lane, and keeps the sums in LDS; then lanes take entries and
// rows and look their sequence up there.  kFill: tables, positions, places and row ranges (kRest: of all `rows`, also those behind the last sequence's);
// kGive: pages given back and the new state, by one workgroup.  The first workgroup gives and the others fill; where the new state takes the old
// one's place, which the others read, one workgroup does both, or a launch of its own gives.  The loads of a turn are issued together.
// A step of 256 sequences, some of which end, is two workgroups' chains, 5.9 to 6.4 us (in one 6.9): lengths, sums (two barriers), a search in LDS,
// table or ring, result.  A million
// rows are written in 11 us, 12 bytes each: four such turns of 255 workgroups, one a compute unit (127 / 383 / 511 / 1023 workgroups 14.9 / 13.3 / 12.9 /
// 17.2 us).  Two or four rows a lane and turn 12.2 / 14.2; 64 registers, so that a compute unit holds two workgroups, 13.0.
constexpr int kGive = 1, kFill = 2, kRest = 4;
template <int PER>
__global__ __launch_bounds__(kPoolThreads) void pool_resize_kernel(const int32_t *state, const int32_t *len, const int32_t *new_len, int rows,
                                                                  int what, PoolArgs a, int32_t *state_out, int32_t *cu, int32_t *positions,
                                                                  int64_t *slots) {
  constexpr int kSeqs = PER * kPoolThreads;
  __shared__ Triple lds_sum[kPoolWaves];
  __shared__ int row_first[kSeqs], grow_first[kSeqs], shrink_first[kSeqs], lds_given[kPoolWaves];
  __shared__ int2 lds_len[PER == 1 ? kSeqs : 1];          // old and new (of more sequences they are fetched again)
  const int t = threadIdx.x;
  const PoolState st(state, a.n_pages);
  Triple mine[PER], sum{0, 0, 0};
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int b = t * PER + i;
    int old = 0, fresh = 0;
    if (b < a.n_seqs) old = max(len[b], 0), fresh = max(new_len[b], 0);
    if constexpr (PER == 1) lds_len[b] = make_int2(old, fresh);
    const int p0 = a.pages(old), p1 = a.pages(fresh);
    mine[i] = {(int64_t)max(fresh - old, 0), max(p1 - p0, 0), max(p0 - p1, 0)};
    sum.rows += mine[i].rows, sum.grow += mine[i].grow, sum.shrink += mine[i].shrink;
  }
  Triple total;
  Triple before = scan_threads(sum, total, lds_sum);
  const bool several = gridDim.x > 1 && (what & kGive);   // the first workgroup gives, the others fill
  const bool gives = (what & kGive) && blockIdx.x == 0, fills = (what & kFill) && !(several && blockIdx.x == 0);
  const int place = several ? (int)blockIdx.x - 1 : (int)blockIdx.x, share = several ? (int)gridDim.x - 1 : (int)gridDim.x;
  const bool first_fill = fills && place == 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int b = t * PER + i;
    row_first[b] = clipped(before.rows), grow_first[b] = before.grow, shrink_first[b] = before.shrink;
    if (first_fill && b < a.n_seqs) cu[b] = clipped(before.rows);
    before.rows += mine[i].rows, before.grow += mine[i].grow, before.shrink += mine[i].shrink;
  }
  if (first_fill && t == 0) cu[a.n_seqs] = clipped(total.rows);
  __syncthreads();
  const auto old_of = [&](int b) { return PER == 1 ? lds_len[b].x : max(len[b], 0); };
  const auto new_of = [&](int b) { return PER == 1 ? lds_len[b].y : max(new_len[b], 0); };
  const int last = a.n_seqs - 1;
  const int n_rows = fills && (positions || slots) ? (int)min((int64_t)rows, total.rows) : 0, n_grow = fills ? total.grow : 0;
  const int n_all = fills && (positions || slots) && (what & kRest) ? rows : n_rows;
  const int n_shrink = gives ? total.shrink : 0;
  int given = 0;
  // turn by turn, an entry and a row, and entries that are given back
  const int64_t stride = (int64_t)share * kPoolThreads;
  int64_t base = fills ? (int64_t)place * kPoolThreads : 0;
  int back_page[4] = {-1, -1, -1, -1};
  if (n_shrink) find_given(a, shrink_first, 0, n_shrink, new_of, back_page);
  for (int64_t back = 0; base < max(n_all, n_grow) || back < n_shrink; base += stride, back += kGiveTurn) {
    const int64_t i = base + t;
    int fresh_page = -1, page = -1, pos = 0;
    int32_t *entry_at = nullptr;
    if (i < n_grow) {
      const int b = find_seq(grow_first, 0, last, (int)i);
      entry_at = a.table + (int64_t)b * a.table_stride + a.pages(old_of(b)) + ((int)i - grow_first[b]);
      fresh_page = taken_page(a, st, (int)i);
    }
    if (i < n_rows) {
      const int b = find_seq(row_first, 0, last, (int)i), old = old_of(b), had = a.pages(old);
      pos = old + ((int)i - row_first[b]);
      const int entry = pos >> a.page_shift;
      if (slots && entry < had) page = a.table[(int64_t)b * a.table_stride + entry];
      else if (slots && entry < a.pages_per_seq) page = taken_page(a, st, grow_first[b] + entry - had);
    }
    if (back < n_shrink) {
      int next_page[4] = {-1, -1, -1, -1};
      if (back + kGiveTurn < n_shrink) find_given(a, shrink_first, back + kGiveTurn, n_shrink, new_of, next_page);
      put_given(a, st, back_page, given, lds_given);
#pragma unroll
      for (int u = 0; u < 4; ++u) back_page[u] = next_page[u];
    }
    if (entry_at) *entry_at = fresh_page;
    if (i < n_all) {
      if (positions) positions[i] = pos;
      if (slots) slots[i] = slot_of(a, page, pos);
    }
  }
  if (gives && t == 0) leave_state(a, st, total.grow, given, state_out);
}

// More sequences, in two launches.  First one workgroup adds up all sequences, leaves the sums in `cu` and the workspace, gives pages back
// and writes the new state.
struct PoolPlan {
  int32_t state[4];                                      // as it was
  int32_t wanted, rows;                                  // pages and rows of all sequences
  int32_t unused[2];
  __host__ __device__ int32_t *grow_first() { return reinterpret_cast<int32_t *>(this + 1); }
};
__global__ __launch_bounds__(kPoolThreads) void pool_plan_kernel(const int32_t *state, PoolArgs a, int32_t *state_out, int32_t *cu, PoolPlan *plan) {
  __shared__ Triple lds_sum[kPoolWaves];
  __shared__ int lds_given[kPoolWaves];
  const int t = threadIdx.x;
  const PoolState st(state, a.n_pages);
  int32_t *grow_first = plan->grow_first(), *shrink_first = grow_first + a.n_seqs;
  Triple sum{0, 0, 0};
  for (int base = 0; base < a.n_seqs; base += kPoolThreads) {
    const int b = base + t;
    int old = 0, fresh = 0;
    if (b < a.n_seqs) old = max(a.len[b], 0), fresh = max(a.new_len[b], 0);
    const int p0 = a.pages(old), p1 = a.pages(fresh);
    Triple total;
    const Triple before = scan_threads({(int64_t)max(fresh - old, 0), max(p1 - p0, 0), max(p0 - p1, 0)}, total, lds_sum);
    if (b < a.n_seqs) {
      cu[b] = clipped(sum.rows + before.rows);
      grow_first[b] = sum.grow + before.grow;
      shrink_first[b] = sum.shrink + before.shrink;
    }
    sum.rows += total.rows, sum.grow += total.grow, sum.shrink += total.shrink;
    __syncthreads();                                     // (the sums' place is used again)
  }
  __threadfence_block();
  __syncthreads();
  int given = 0;
  const auto new_of = [&](int b) { return max(a.new_len[b], 0); };
  int page[4] = {-1, -1, -1, -1};
  if (sum.shrink) find_given(a, shrink_first, 0, sum.shrink, new_of, page);
  for (int64_t back = 0; back < sum.shrink; back += kGiveTurn) {
    int next[4] = {-1, -1, -1, -1};
    if (back + kGiveTurn < sum.shrink) find_given(a, shrink_first, back + kGiveTurn, sum.shrink, new_of, next);
    put_given(a, st, page, given, lds_given);
#pragma unroll
    for (int u = 0; u < 4; ++u) page[u] = next[u];
  }
  if (t == 0) {
    cu[a.n_seqs] = clipped(sum.rows);
    *reinterpret_cast<int4 *>(plan->state) = make_int4(st.head, st.count, 0, 0);
    plan->wanted = sum.grow;
    plan->rows = clipped(sum.rows);
    leave_state(a, st, sum.grow, given, state_out);
  }
}
// Then many fill tables, positions and places.  A wavefront takes 64 consecutive rows (or entries) at a time: their sequences lie between
// the first one's and the last one's, which all lanes look for together.
__device__ __forceinline__ int find_seq_wave(const int *first, int n_seqs, int x, int total) {
  const int x0 = __builtin_amdgcn_readfirstlane(x), x1 = total - x0 > 64 ? x0 + 63 : total - 1;
  const int lo = find_seq_all(first, 0, n_seqs, x0);
  return find_seq(first, lo, find_seq_all(first, lo, n_seqs, x1), min(x, x1));
}
__global__ __launch_bounds__(256) void pool_fill_kernel(PoolArgs a, const int32_t *cu, PoolPlan *plan, int rows, int rest, int row_blocks,
                                                        int32_t *positions, int64_t *slots) {
  const PoolState st(plan->state, a.n_pages);
  const int32_t *grow_first = plan->grow_first();
  if ((int)blockIdx.x >= row_blocks) {                   // entries
    const int total = plan->wanted, stride = ((int)gridDim.x - row_blocks) * 256;
    for (int64_t i0 = ((int64_t)blockIdx.x - row_blocks) * 256 + (threadIdx.x & ~63); i0 < total; i0 += stride) {
      const int i = (int)min(i0 + (threadIdx.x & 63), (int64_t)INT32_MAX), b = find_seq_wave(grow_first, a.n_seqs, i, total);
      if (i < total)
        a.table[(int64_t)b * a.table_stride + a.pages(max(a.len[b], 0)) + (i - grow_first[b])] = taken_page(a, st, i);
    }
    return;
  }
  const int n = min(rows, plan->rows), all = rest ? rows : n;
  for (int64_t i0 = (int64_t)blockIdx.x * 256 + (threadIdx.x & ~63); i0 < all; i0 += (int64_t)row_blocks * 256) {
    const int i = (int)min(i0 + (threadIdx.x & 63), (int64_t)INT32_MAX);
    int page = -1, pos = 0;
    if (i0 < n) {
      const int b = find_seq_wave(cu, a.n_seqs, i, n);
      if (i < n) {
        const int old = max(a.len[b], 0), had = a.pages(old);
        pos = old + (i - cu[b]);
        const int entry = pos >> a.page_shift;
        if (slots && entry < had) page = a.table[(int64_t)b * a.table_stride + entry];
        else if (slots && entry < a.pages_per_seq) page = taken_page(a, st, grow_first[b] + entry - had);
      }
    }
    if (i < all) {
      if (positions) positions[i] = pos;
      if (slots) slots[i] = slot_of(a, page, pos);
    }
  }
}

constexpr int kLdsSeqs = 4 * kPoolThreads;               // sequences whose sums a workgroup keeps

}  // namespace et

using namespace et;

extern "C" {

size_t et_kv_resize_workspace_bytes(int32_t n_seqs) {
  if (n_seqs <= kLdsSeqs) return 0;
  return sizeof(PoolPlan) + 2 * sizeof(int32_t) * (size_t)n_seqs;
}

int et_kv_resize(const et_kv_pool *pool, const int32_t *state_dev, int32_t *state_out_dev, int32_t *page_table_dev, int32_t table_stride,
                 int32_t pages_per_seq, const int32_t *kv_len_dev, const int32_t *new_len_dev, int32_t n_seqs, int32_t rows,
                 int32_t *cu_rows_dev, int32_t *positions_dev, int64_t *slots_dev, void *workspace_dev, size_t workspace_bytes,
                 void *hip_stream) {
  ET_REQUIRE(pool != nullptr, "pool is NULL");
  const int page = pool->page_size;
  ET_REQUIRE(page >= 16 && page <= 256 && (page & (page - 1)) == 0, "page_size = %d must be 16, 32, 64, 128 or 256", page);
  ET_REQUIRE(pool->n_pages >= 1 && pool->ring_dev != nullptr, "n_pages = %d must be at least 1, and ring_dev not NULL", pool->n_pages);
  ET_REQUIRE(pool->keep_rest == 0 || pool->keep_rest == 1, "keep_rest = %d must be 0 or 1", pool->keep_rest);
  ET_REQUIRE(state_dev && state_out_dev && (uintptr_t)state_dev % 16 == 0 && (uintptr_t)state_out_dev % 16 == 0,
             "state_dev or state_out_dev is NULL or not aligned to 16 bytes");
  ET_REQUIRE(n_seqs >= 0 && n_seqs <= 1 << 20, "n_seqs = %d must be in [0, 2^20]", n_seqs);
  ET_REQUIRE(pages_per_seq >= 1 && table_stride >= pages_per_seq && (int64_t)pages_per_seq * page <= 1 << 30,
             "pages_per_seq = %d must be at least 1, at most table_stride = %d, and at most 2^30 tokens", pages_per_seq, table_stride);
  ET_REQUIRE((int64_t)n_seqs * pages_per_seq < 1ll << 31, "n_seqs * pages_per_seq is above 2^31");
  ET_REQUIRE(rows >= 0, "rows = %d is negative", rows);
  ET_REQUIRE(cu_rows_dev != nullptr, "cu_rows_dev is NULL");
  ET_REQUIRE(n_seqs == 0 || (page_table_dev && kv_len_dev && new_len_dev), "page_table_dev, kv_len_dev or new_len_dev is NULL");
  ET_REQUIRE((uintptr_t)slots_dev % 8 == 0, "slots_dev is not aligned to 8 bytes");
  const size_t need = et_kv_resize_workspace_bytes(n_seqs);
  if (need) {
    ET_REQUIRE(workspace_dev != nullptr && (uintptr_t)workspace_dev % 16 == 0, "workspace_dev is NULL or not aligned to 16 bytes");
    if (workspace_bytes < need) {
      set_error("workspace of %zu bytes is smaller than the %zu needed", workspace_bytes, need);
      return ET_ERR_WORKSPACE;
    }
  }
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  const PoolArgs a{pool->ring_dev, page_table_dev, kv_len_dev, new_len_dev, pool->n_pages, __builtin_ctz(page), table_stride, pages_per_seq, n_seqs};
  if (!need) {
    // A turn of 1024 rows a workgroup, and one that gives; in place one workgroup for everything up to six turns, as the giving would be a launch of its own
    // (3 us).  us, one / several: 256 sequences, 253 rows 6.9 / 5.6; 4, 1544 4.9 / 4.6; 256, 2634 7.0 / 5.1, in place 7.0 / 8.2; in place 4, 5516 7.3 / 7.8;
    // 16, 8550 10.4 / 7.8; 4096, 4096 11.5 / 12.8.  With turns of 2048 rows 16 sequences, 62 605 rows 4.8 -> 5.7, 1000, 8000 5.7 -> 6.8.
    const int turns = std::max(1, (int)(((int64_t)std::max(rows, n_seqs) + kPoolThreads - 1) / kPoolThreads)), fillers = std::min(255, turns);
    const int fill = pool->keep_rest ? kFill : kFill | kRest;
    const bool in_place = state_out_dev == state_dev, one = in_place && turns <= 6, apart = in_place && !one;
    auto launch = [&](int blocks, int what) {
      (n_seqs <= kPoolThreads ? pool_resize_kernel<1> : pool_resize_kernel<4>)<<<blocks, kPoolThreads, 0, stream>>>(
          state_dev, kv_len_dev, new_len_dev, rows, what, a, state_out_dev, cu_rows_dev, positions_dev, slots_dev);
      ET_LAUNCH_CHECK();
      return ET_OK;
    };
    int rc;
    if ((rc = launch(one ? 1 : apart ? fillers : fillers + 1, apart ? fill : fill | kGive)) || !apart) return rc;
    return launch(1, kGive);
  }
  PoolPlan *plan = static_cast<PoolPlan *>(workspace_dev);
  pool_plan_kernel<<<1, kPoolThreads, 0, stream>>>(state_dev, a, state_out_dev, cu_rows_dev, plan);
  ET_LAUNCH_CHECK();
  const int row_blocks = positions_dev || slots_dev ? std::min(2048, (int)(((int64_t)rows + 255) / 256)) : 0;
  const int entry_blocks = (int)std::min<int64_t>(256, ((int64_t)n_seqs * pages_per_seq + 255) / 256);
  pool_fill_kernel<<<row_blocks + entry_blocks, 256, 0, stream>>>(a, cu_rows_dev, plan, rows, !pool->keep_rest, row_blocks, positions_dev,
                                                                   slots_dev);
  ET_LAUNCH_CHECK();
  return ET_OK;
}

}  // extern "C"
