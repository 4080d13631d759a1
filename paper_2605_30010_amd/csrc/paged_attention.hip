// Attention of one new token per sequence over a paged key-value cache: joining the parts, and the entry points.
#include "paged_attention.h"

namespace et {

// Joins the parts of one query head, always in the same order: groups of lanes, four dimensions a lane, take every GROUPS-th part
// with a running maximum and sum, eight parts' loads in flight, and the groups' results are added up in the groups' order.
// A head whose sequence is one part has its result already.  THREADS: 64 where a sequence has few parts.  Bound by latency: 28 heads of
// 40 parts take 3.1 us, 32 of 64 5.0, 2048 of four 5.1.
template <int HD, int FMT, int THREADS, bool ONE>
__global__ __launch_bounds__(THREADS) void paged_join_kernel(const int32_t *len, const float *part_o, const float2 *part_ml, int n_seqs,
                                                             int share, int bound, int window, int n_heads, uint16_t *out) {
  constexpr int LANES = HD / 4, GROUPS = THREADS / LANES, BATCH = 8;
  __shared__ float lds_o[GROUPS][HD];
  __shared__ float2 lds_ml[GROUPS];
  const PagedArgs a{len, n_seqs, bound, window, share};
  const int b = blockIdx.x / n_heads, h = blockIdx.x % n_heads;
  const int tid = threadIdx.x, lane = tid % LANES, grp = tid / LANES;
  f32x4 v[BATCH];
  float2 s[BATCH];
  auto load = [&](int before, int first, int last) {
    const int64_t base = (int64_t)before * n_heads + h;
    const float2 *my_ml = part_ml + base;
    const float *my_o = part_o + base * HD;
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      const uint32_t at = (uint32_t)min(first + i * GROUPS, last) * n_heads;
      s[i] = my_ml[at];
      v[i] = *reinterpret_cast<const f32x4 *>(my_o + (at * HD + lane * 4));
    }
  };
  // a single sequence's parts come first, however many there are: their loads need not wait for its length
  if (ONE && grp < GROUPS) load(0, grp, share - 1);
  const Part p = find_part<ONE>(a, 0, b);
  if (p.count == 1) return;
  if (!ONE && grp < GROUPS && p.count) load(p.before, grp, p.count - 1);
  if (grp < GROUPS) {
    f32x4 x{0, 0, 0, 0};
    float top = -INFINITY, total = 0.f;
    for (int first = grp; first < p.count; first += BATCH * GROUPS) {
      if (first != grp) load(p.before, first, p.count - 1);
      float most = top;
#pragma unroll
      for (int i = 0; i < BATCH; ++i)
        if (first + i * GROUPS < p.count) most = fmaxf(most, s[i].x);
      const float old = part_factor(make_float2(top, total), most);
      total *= old;
      top = most;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] *= old;
#pragma unroll
      for (int i = 0; i < BATCH; ++i)
        if (first + i * GROUPS < p.count) {
          const float f = part_factor(s[i], top);
          total = fmaf(f, s[i].y, total);
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = fmaf(f, v[i][e], x[e]);
        }
    }
    *reinterpret_cast<f32x4 *>(&lds_o[grp][lane * 4]) = x;
    if (lane == 0) lds_ml[grp] = make_float2(top, total);
  }
  __syncthreads();
  float top = -INFINITY, total = 0.f, f[GROUPS];
#pragma unroll
  for (int i = 0; i < GROUPS; ++i) top = fmaxf(top, lds_ml[i].x);
#pragma unroll
  for (int i = 0; i < GROUPS; ++i) {
    f[i] = part_factor(lds_ml[i], top);
    total = fmaf(f[i], lds_ml[i].y, total);
  }
  for (int d = tid; d < HD; d += THREADS) {
    float x = 0.f;
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) x = fmaf(f[i], lds_o[i][d], x);
    out[(int64_t)blockIdx.x * HD + d] = f32_to_bf16_bits(total == 0.f ? 0.f : x * (value_factor<FMT>() / total));
  }
}

struct PagedPlan {
  int group, row_tiles, units, bound, share;
  int64_t items;                                         // workgroups per unit
  size_t slots, bytes;                                   // of the workspace
};
static PagedPlan paged_plan(const et_kv_cache &c, const et_kv_seqs &s, int n_heads, int max_len, int window) {
  PagedPlan p;
  p.group = n_heads / c.n_kv_heads;
  p.row_tiles = (p.group + 15) / 16;
  p.units = p.row_tiles * c.n_kv_heads;
  p.bound = std::min(max_len, s.pages_per_seq * c.page_size);
  const int span = window > 0 ? (int)std::min<int64_t>(p.bound, (int64_t)window + 15) : p.bound;
  const int64_t blocks = (int64_t)s.n_seqs * ((span + kBlock - 1) / kBlock);
  // One part each where that is as fast: short sequences, and longer ones that fill the chip by themselves.  us as one part / shared out:
  // 1 x 197 tokens 4.8 / 7.7, 256 x 500 of 4 key-value heads 50 / 58, 4 x 1000 of 32 13.7 / 16.7, 1024 x 100 to 2048 of 4 223 / 261;
  // but 1 x 700 of 8 10.0 / 7.8, 4 x 1500 of 4 16.8 / 8.6, 64 x 1000 to 16384 of 8 255 / 215.  The host knows the bound only, so a
  // generous one takes the second figure; and the rule counts tokens, not their bytes (64 x 1024 of one bfloat16 head of 256, one part
  // each: 24.0 / 20.3).
  // Beyond 4096 sequences too: every workgroup of a call that is shared out looks at all lengths, which would come to a minute for
  // a million sequences.  Bound 131072: 4097 x 60 tokens of 8 195 / 1200, 0 to 8000 8768 / 9167, 60 with one of 131072 among them
  // 1419 / 1261 (of one key-value head 1113 / 277).
  const int64_t all = (int64_t)s.n_seqs * p.units;
  // In 4 bits a part's tokens are a quarter of the bytes, and the same rule holds up to 2048 tokens (and a window's 15 more) from 192 on: one part
  // each / shared out, heads of 128, 9 x 2048 of 24 13.9 / 18.1, 64 x 1500 of 8 19.2 / 25.3, 64 x 2048 24.0 / 28.3, 64 x 64 to 2048 21.1 / 20.6;
  // but 32 x 2048 of 4 12.7 / 12.3, 64 x 64 to 4096 of 8 36.1 / 32.9.
  const bool full = c.format == ET_KV_MXFP4 ? span <= 2063 && all >= 192 : span <= 2048 && all >= 1024;
  const bool whole = span <= 512 || (span <= 1024 && all >= 64) || full || s.n_seqs > 4096;
  p.share = whole ? 0 : (int)std::min<int64_t>(blocks, (kShare + p.units - 1) / p.units);
  p.items = p.share * (s.n_seqs > 1 ? kFiner : 1) + (int64_t)s.n_seqs;
  p.slots = p.share ? (size_t)p.items * n_heads : 0;
  p.bytes = p.slots * (c.head_dim * sizeof(float) + sizeof(float2));
  return p;
}

static int check_paged(const et_kv_cache *cache, const et_kv_seqs *seqs, int n_heads, int max_len, int window) {
  int rc;
  if ((rc = check_kv(cache, seqs))) return rc;
  ET_REQUIRE(n_heads >= 1 && n_heads % cache->n_kv_heads == 0 && n_heads <= 65536,
             "n_heads = %d must be a multiple of n_kv_heads = %d, at most 65536", n_heads, cache->n_kv_heads);
  ET_REQUIRE(max_len >= 1, "max_len = %d must be at least 1", max_len);
  ET_REQUIRE(window >= 0, "window = %d is negative", window);
  ET_REQUIRE((int64_t)seqs->n_seqs * n_heads <= 1 << 24, "n_seqs * n_heads = %lld is above 2^24", (long long)seqs->n_seqs * n_heads);
  ET_REQUIRE((int64_t)seqs->n_seqs * std::min(max_len, seqs->pages_per_seq * cache->page_size) <= 1ll << 36,
             "n_seqs * max_len is above 2^36");
  // (a launch takes fewer than 2^32 lanes)
  const PagedPlan p = paged_plan(*cache, *seqs, n_heads, max_len, window);
  ET_REQUIRE(p.items * p.units < (1ll << 32) / (64 * kWaves), "n_seqs * n_kv_heads = %lld is too much for one launch",
             (long long)seqs->n_seqs * cache->n_kv_heads);
  return ET_OK;
}

}  // namespace et

using namespace et;

extern "C" {

size_t et_attention_paged_workspace_bytes(const et_kv_cache *cache, const et_kv_seqs *seqs, int32_t n_heads, int32_t max_len,
                                          int32_t window) {
  if (check_paged(cache, seqs, n_heads, max_len, window) || seqs->n_seqs == 0) return 0;
  return paged_plan(*cache, *seqs, n_heads, max_len, window).bytes;
}

int et_attention_paged(const et_kv_cache *cache, const et_kv_seqs *seqs, const uint16_t *q_dev, int64_t q_stride, int32_t n_heads,
                       int32_t max_len, int32_t window, float scale, void *workspace_dev, size_t workspace_bytes, uint16_t *out_dev,
                       void *hip_stream) {
  int rc;
  if ((rc = check_paged(cache, seqs, n_heads, max_len, window))) return rc;
  ET_REQUIRE(scale - scale == 0.f, "scale must be finite");
  if (seqs->n_seqs == 0) return ET_OK;
  ET_REQUIRE(q_dev && out_dev && (uintptr_t)q_dev % 16 == 0 && (uintptr_t)out_dev % 16 == 0,
             "q_dev or out_dev is NULL or not aligned to 16 bytes");
  ET_REQUIRE(q_stride % 8 == 0 && q_stride >= (int64_t)n_heads * cache->head_dim, "q_stride = %lld must be a multiple of 8 and at least %lld",
             (long long)q_stride, (long long)n_heads * cache->head_dim);
  const PagedPlan p = paged_plan(*cache, *seqs, n_heads, max_len, window);
  if (p.bytes) {
    ET_REQUIRE(workspace_dev != nullptr && (uintptr_t)workspace_dev % 16 == 0, "workspace_dev is NULL or not aligned to 16 bytes");
    if (workspace_bytes < p.bytes) {
      set_error("workspace of %zu bytes is smaller than the %zu needed", workspace_bytes, p.bytes);
      return ET_ERR_WORKSPACE;
    }
  }
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  float *part_o = static_cast<float *>(workspace_dev);
  float2 *part_ml = reinterpret_cast<float2 *>(part_o + p.slots * cache->head_dim);
  const int f = cache->format;
  const float scale_log2 = scale * 1.4426950408889634f * (f == ET_KV_INT8 ? 1.f / 127.f : f == ET_KV_E4M3 ? 1.f / 448.f : 1.f);
  const KvPages c = kv_pages(*cache);
  const PagedLaunch launch{seqs->kv_len_dev, seqs->page_table_dev, seqs->n_seqs, p.share, p.bound, window, p.units, p.row_tiles, c.page_shift,
                           seqs->table_stride, p.group,
                           PagedMore{q_dev, q_stride, c.data, c.page_bytes, part_o, part_ml, out_dev, c.n_pages, scale_log2},
                           (unsigned)(p.items * p.units), stream};
  auto join = [&](auto hd, auto fmt) {
    // (64 / 256 lanes a head, us: 64 x 100 to 2048 tokens, 32 heads 61.6 / 64.9; 2 x 60000, 16 heads, 196 parts each 30.1 / 20.2)
    const bool one = seqs->n_seqs == 1, few = !one && p.share <= 16 * (int64_t)seqs->n_seqs;
    const unsigned heads = (unsigned)(seqs->n_seqs * n_heads);
    (one ? paged_join_kernel<hd.value, fmt.value, 256, true> : few ? paged_join_kernel<hd.value, fmt.value, 64, false>
                                                                   : paged_join_kernel<hd.value, fmt.value, 256, false>)<<<
        heads, few ? 64 : 256, 0, stream>>>(seqs->kv_len_dev, part_o, part_ml, seqs->n_seqs, p.share, p.bound, window, n_heads, out_dev);
    ET_LAUNCH_CHECK();
    return ET_OK;
  };
  // (the parts of 4-bit tokens are results already, as those of bfloat16 ones)
  if (f == ET_KV_MXFP4) {
    if ((rc = launch_paged_mxfp4(cache->head_dim, launch)) || !p.share) return rc;
    return kv_dispatch(cache->head_dim, ET_KV_BF16, join);
  }
  return kv_dispatch(cache->head_dim, f, [&](auto hd, auto fmt) {
    const int launched = launch_paged<hd.value, fmt.value>(launch);
    return launched || !p.share ? launched : join(hd, fmt);
  });
}

}  // extern "C"
