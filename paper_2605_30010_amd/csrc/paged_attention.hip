// Attention of one new token per sequence over a paged key-value cache.
#include <type_traits>

#include "kv_cache.h"
#include "mfma_common.h"

namespace et {

// Value `d` of a row as the cache holds it, without the factor m / Q of the 8-bit formats.
template <int FMT>
__device__ __forceinline__ float kv_code(const char *row, int d) {
  if constexpr (FMT == ET_KV_BF16) return bf16_to_f32(reinterpret_cast<const uint16_t *>(row)[d]);
  else if constexpr (FMT == ET_KV_INT8) return (float)reinterpret_cast<const int8_t *>(row)[d];
  else return __builtin_amdgcn_cvt_f32_fp8((uint32_t)reinterpret_cast<const uint8_t *>(row)[d], 0);
}

// a * b rounded, never part of a fused multiply-add: a logit less the maximum has to be 0 for the maximum itself, however large.
__device__ __forceinline__ float whole_product(float a, float b) {
#pragma clang fp contract(off)
  return a * b;
}

// A wavefront per sequence and query head walks over the tokens, one at a time, with the running maximum and sum of the softmax.
template <int HD, int FMT>
__global__ __launch_bounds__(64) void paged_attention_kernel(KvPages c, KvSeqs s, const uint16_t *q, int64_t q_stride, int n_heads,
                                                             int max_len, int window, float scale, uint16_t *out) {
  using Lay = KvLayout<HD, FMT>;
  constexpr int N = (HD + 63) / 64;
  const int lane = threadIdx.x, b = blockIdx.x / n_heads, h = blockIdx.x % n_heads, kv = h / (n_heads / c.kv_heads);
  const int ps = 1 << c.page_shift, len = min(min(s.len[b], max_len), s.pages_per_seq << c.page_shift);
  const int first = window > 0 ? max(0, (int)min((int64_t)s.len[b], (int64_t)INT32_MAX) - window) : 0;
  float x[N], acc[N], m = -INFINITY, sum = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int d = i * 64 + lane;
    x[i] = d < HD ? bf16_to_f32(q[b * q_stride + h * HD + d]) * scale : 0.f;
    acc[i] = 0.f;
  }
  for (int t = first; t < len; ++t) {
    const int page = s.table[(int64_t)b * s.table_stride + (t >> c.page_shift)], at = t & (ps - 1);
    if (page < 0 || page >= c.n_pages) continue;
    const char *head = c.data + page * c.page_bytes + (int64_t)kv * Lay::head_bytes(ps);
    float km = 1.f, vm = 1.f, dot = 0.f;
    if constexpr (FMT != ET_KV_BF16) {
      km = bf16_to_f32(reinterpret_cast<const uint16_t *>(head + Lay::key_max(ps))[at]) * (1.f / kv_qmax<FMT>());
      vm = bf16_to_f32(reinterpret_cast<const uint16_t *>(head + Lay::value_max(ps))[at]) * (1.f / kv_qmax<FMT>());
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i * 64 + lane < HD) dot = fmaf(x[i], kv_code<FMT>(head + at * Lay::kRow, i * 64 + lane), dot);
    dot = whole_product(wave_sum(dot), km);
    const float m2 = dot > m ? dot : m, ref = m2 == -INFINITY ? 0.f : m2, old = __expf(m - ref), p = __expf(dot - ref);
    sum = sum * old + p;
    m = m2;
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i * 64 + lane < HD)
        acc[i] = acc[i] * old + p * (kv_code<FMT>(head + Lay::values(ps) + at * Lay::kRow, i * 64 + lane) * vm);
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int d = i * 64 + lane;
    if (d < HD) out[((int64_t)b * n_heads + h) * HD + d] = f32_to_bf16_bits(sum == 0.f ? 0.f : acc[i] / sum);
  }
}

}  // namespace et

using namespace et;

extern "C" {

size_t et_attention_paged_workspace_bytes(const et_kv_cache *cache, const et_kv_seqs *seqs, int32_t n_heads, int32_t max_len,
                                          int32_t window) {
  return 0;
}

int et_attention_paged(const et_kv_cache *cache, const et_kv_seqs *seqs, const uint16_t *q_dev, int64_t q_stride, int32_t n_heads,
                       int32_t max_len, int32_t window, float scale, void *workspace_dev, size_t workspace_bytes, uint16_t *out_dev,
                       void *hip_stream) {
  int rc;
  if ((rc = check_kv(cache, seqs))) return rc;
  ET_REQUIRE(n_heads >= 1 && n_heads % cache->n_kv_heads == 0 && n_heads <= 65536,
             "n_heads = %d must be a multiple of n_kv_heads = %d, at most 65536", n_heads, cache->n_kv_heads);
  ET_REQUIRE(max_len >= 1, "max_len = %d must be at least 1", max_len);
  ET_REQUIRE(window >= 0, "window = %d is negative", window);
  ET_REQUIRE(scale - scale == 0.f, "scale must be finite");
  if (seqs->n_seqs == 0) return ET_OK;
  ET_REQUIRE(q_dev && out_dev && (uintptr_t)q_dev % 16 == 0 && (uintptr_t)out_dev % 16 == 0,
             "q_dev or out_dev is NULL or not aligned to 16 bytes");
  ET_REQUIRE(q_stride % 8 == 0 && q_stride >= (int64_t)n_heads * cache->head_dim, "q_stride = %lld must be a multiple of 8 and at least %lld",
             (long long)q_stride, (long long)n_heads * cache->head_dim);
  ET_REQUIRE((int64_t)seqs->n_seqs * n_heads <= INT32_MAX, "n_seqs * n_heads is above 2^31 - 1");
  return kv_dispatch(cache->head_dim, cache->format, [&](auto hd, auto fmt) {
    paged_attention_kernel<hd.value, fmt.value><<<seqs->n_seqs * n_heads, 64, 0, static_cast<hipStream_t>(hip_stream)>>>(
        kv_pages(*cache), kv_seqs(*seqs), q_dev, q_stride, n_heads, max_len, window, scale, out_dev);
    ET_LAUNCH_CHECK();
    return ET_OK;
  });
}

}  // extern "C"
