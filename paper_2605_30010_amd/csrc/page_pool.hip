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
constexpr int kOneSeqs = 1024;                           // sequences and rows up to which one workgroup does everything
constexpr int kOneRows = 8192;

// Sums over the workgroup's threads before mine of three numbers, and the totals.  The first may pass 32 bits.
struct Triple {
  int64_t rows;
  int grow, shrink;
};
__device__ __forceinline__ Triple scan_threads(Triple mine, Triple &total, Triple (&lds)[kPoolWaves]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int64_t r = mine.rows;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int64_t up = __shfl_up(r, d, 64);
    if (lane >= d) r += up;
  }
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
  __syncthreads();                                       // (the sums may be written again)
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

// Gives the pages behind the sequences' ends back: entry i of all `total` goes, if it is a page, behind the ring's `count` free ones,
// in order.  By one workgroup; returns how many found room there.
__device__ __forceinline__ int give_back(const PoolArgs &a, PoolState st, const int *shrink_first, int total, int *lds) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, room = a.n_pages - st.count;
  int given = 0;
  for (int base = 0; base < total; base += kPoolThreads) {
    const int i = base + threadIdx.x;
    int page = -1;
    if (i < total) {
      const int b = find_seq(shrink_first, 0, a.n_seqs - 1, i);
      page = a.table[(int64_t)b * a.table_stride + a.pages(max(a.new_len[b], 0)) + (i - shrink_first[b])];
    }
    const bool good = a.is_page(page);
    const uint64_t votes = __ballot(good);
    if (lane == 0) lds[wave] = __popcll(votes);
    __syncthreads();
    int at = given + __popcll(votes & ((1ull << lane) - 1));
#pragma unroll
    for (int w = 0; w < kPoolWaves; ++w) {
      const int n = lds[w];
      if (w < wave) at += n;
      given += n;
    }
    if (good && at < room) a.ring[a.cell(st.head, st.count + at)] = page;
    __syncthreads();
  }
  return min(given, room);
}
// Entry i of all that are wanted: the ring's i-th page, or none.
__device__ __forceinline__ int taken_page(const PoolArgs &a, PoolState st, int i) { return i < st.count ? a.ring[a.cell(st.head, i)] : -1; }

__device__ __forceinline__ void leave_state(const PoolArgs &a, PoolState st, int wanted, int given, int32_t *state_out) {
  const int used = min(wanted, st.count);
  *reinterpret_cast<int4 *>(state_out) = make_int4((int)(((uint32_t)st.head + (uint32_t)used) % (uint32_t)a.n_pages), st.count - used + given,
                                                   wanted - used, 0);
}
// Place of token `pos` whose page is `page`.
__device__ __forceinline__ int64_t slot_of(const PoolArgs &a, int page, int pos) {
  return a.is_page(page) ? ((int64_t)page << a.page_shift) + (pos & ((1 << a.page_shift) - 1)) : -1;
}

// Everything by one workgroup: up to 1024 sequences (a lane each) and a decoding step's rows.
__global__ __launch_bounds__(kPoolThreads) void pool_step_kernel(const int32_t *state, const int32_t *len, const int32_t *new_len, int rows,
                                                                PoolArgs a, int32_t *state_out, int32_t *cu, int32_t *positions,
                                                                int64_t *slots) {
  __shared__ Triple lds_sum[kPoolWaves];
  __shared__ int row_first[kOneSeqs], grow_first[kOneSeqs], shrink_first[kOneSeqs], old_len[kOneSeqs], lds_votes[kPoolWaves];
  const int t = threadIdx.x;
  const PoolState st(state, a.n_pages);
  int old = 0, fresh = 0;
  if (t < a.n_seqs) old = max(len[t], 0), fresh = max(new_len[t], 0);
  const int p0 = a.pages(old), p1 = a.pages(fresh);
  Triple total;
  const Triple before = scan_threads({(int64_t)max(fresh - old, 0), max(p1 - p0, 0), max(p0 - p1, 0)}, total, lds_sum);
  row_first[t] = clipped(before.rows), grow_first[t] = before.grow, shrink_first[t] = before.shrink, old_len[t] = old;
  if (t < a.n_seqs) cu[t] = clipped(before.rows);
  if (t == 0) cu[a.n_seqs] = clipped(total.rows);
  __syncthreads();
  const int last = a.n_seqs - 1;
  for (int i = t; i < total.grow; i += kPoolThreads) {
    const int b = find_seq(grow_first, 0, last, i);
    a.table[(int64_t)b * a.table_stride + a.pages(old_len[b]) + (i - grow_first[b])] = taken_page(a, st, i);
  }
  if (positions || slots) {
    const int n = (int)min((int64_t)rows, total.rows);
    for (int i = t; i < n; i += kPoolThreads) {
      const int b = find_seq(row_first, 0, last, i), pos = old_len[b] + (i - row_first[b]);
      if (positions) positions[i] = pos;
      if (slots) {
        const int entry = pos >> a.page_shift, had = a.pages(old_len[b]);
        int page = -1;
        if (entry < had) page = a.table[(int64_t)b * a.table_stride + entry];
        else if (entry < a.pages_per_seq) page = taken_page(a, st, grow_first[b] + entry - had);
        slots[i] = slot_of(a, page, pos);
      }
    }
  }
  const int given = give_back(a, st, shrink_first, total.shrink, lds_votes);
  if (t == 0) leave_state(a, st, total.grow, given, state_out);
}

// The same in two launches.  First one workgroup adds up all sequences, leaves the sums in `cu` and the workspace, gives pages back
// and writes the new state.
struct PoolPlan {
  int32_t state[4];                                      // as it was
  int32_t wanted, rows;                                  // pages and rows of all sequences
  int32_t unused[2];
  __host__ __device__ int32_t *grow_first() { return reinterpret_cast<int32_t *>(this + 1); }
};
__global__ __launch_bounds__(kPoolThreads) void pool_plan_kernel(const int32_t *state, PoolArgs a, int32_t *state_out, int32_t *cu, PoolPlan *plan) {
  __shared__ Triple lds_sum[kPoolWaves];
  __shared__ int lds_votes[kPoolWaves];
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
  }
  __threadfence_block();
  __syncthreads();
  const int given = give_back(a, st, shrink_first, sum.shrink, lds_votes);
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
  const int lane = threadIdx.x & 63;
  const int x0 = __builtin_amdgcn_readfirstlane(x), x1 = min(x0 + 63, total - 1);
  int lo[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int want = k ? x1 : x0;
    int from = k ? lo[0] : 0, len = n_seqs - from;         // the answer is in [from, from + len)
    while (len > 1) {
      const int step = (len + 63) / 64, i = from + lane * step;
      const int hits = __popcll(__ballot(lane * step < len && first[min(i, n_seqs - 1)] <= want));
      from += (hits - 1) * step;
      len = min(step, n_seqs - from);
    }
    lo[k] = from;
  }
  return find_seq(first, lo[0], lo[1], min(x, x1));
}
__global__ __launch_bounds__(256) void pool_fill_kernel(PoolArgs a, const int32_t *cu, PoolPlan *plan, int rows, int row_blocks, int32_t *positions,
                                                        int64_t *slots) {
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
  const int n = min(rows, plan->rows);
  for (int64_t i0 = (int64_t)blockIdx.x * 256 + (threadIdx.x & ~63); i0 < n; i0 += (int64_t)row_blocks * 256) {
    const int i = (int)min(i0 + (threadIdx.x & 63), (int64_t)INT32_MAX), b = find_seq_wave(cu, a.n_seqs, i, n);
    if (i >= n) continue;
    const int old = max(a.len[b], 0), pos = old + (i - cu[b]);
    if (positions) positions[i] = pos;
    if (slots) {
      const int entry = pos >> a.page_shift, had = a.pages(old);
      int page = -1;
      if (entry < had) page = a.table[(int64_t)b * a.table_stride + entry];
      else if (entry < a.pages_per_seq) page = taken_page(a, st, grow_first[b] + entry - had);
      slots[i] = slot_of(a, page, pos);
    }
  }
}

static bool in_one(int n_seqs, int rows) { return n_seqs <= kOneSeqs && rows <= kOneRows; }

}  // namespace et

using namespace et;

extern "C" {

size_t et_kv_resize_workspace_bytes(int32_t n_seqs, int32_t rows) {
  if (n_seqs < 1 || rows < 0 || in_one(n_seqs, rows)) return 0;
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
  const size_t need = et_kv_resize_workspace_bytes(n_seqs, rows);
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
    pool_step_kernel<<<1, kPoolThreads, 0, stream>>>(state_dev, kv_len_dev, new_len_dev, rows, a, state_out_dev, cu_rows_dev, positions_dev, slots_dev);
    ET_LAUNCH_CHECK();
    return ET_OK;
  }
  PoolPlan *plan = static_cast<PoolPlan *>(workspace_dev);
  pool_plan_kernel<<<1, kPoolThreads, 0, stream>>>(state_dev, a, state_out_dev, cu_rows_dev, plan);
  ET_LAUNCH_CHECK();
  const int row_blocks = positions_dev || slots_dev ? std::min(2048, (int)(((int64_t)rows + 255) / 256)) : 0;
  const int entry_blocks = (int)std::min<int64_t>(256, ((int64_t)n_seqs * pages_per_seq + 255) / 256);
  pool_fill_kernel<<<row_blocks + entry_blocks, 256, 0, stream>>>(a, cu_rows_dev, plan, rows, row_blocks, positions_dev, slots_dev);
  ET_LAUNCH_CHECK();
  return ET_OK;
}

}  // extern "C"
