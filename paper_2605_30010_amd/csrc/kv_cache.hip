// Storing keys and values in a paged cache, in bfloat16 or 8 bits, and reading them back.
#include <type_traits>

#include "kv_cache.h"
#include "mfma_common.h"

namespace et {

// Where a row of new (or wanted) tokens lies.  cu ascends; whatever it holds, the answer is inside the cache or "none".
struct KvPlace {
  int owned;                 // the row belongs to a sequence
  int64_t page;              // < 0: no place in the cache
  int at;                    // token of the page
};

// The same for all lanes of a wavefront (r is).  The sequence is found by up to 64 probes at a time: a batch of 64
// sequences takes one load, 4096 two.
__device__ __forceinline__ KvPlace kv_place(const int32_t *cu, int r, const KvSeqs &s, const KvPages &c) {
  KvPlace out{0, -1, 0};
  int seq = r, back = 1;                                  // back: the row's distance from the sequence's end
  if (cu) {
    const int lane = threadIdx.x & 63;
    int lo = 0, len = s.n_seqs;                           // cu[i] <= r holds for at least lo and at most lo + len of i = 1..n_seqs
    while (len > 64) {
      const int step = (len + 63) / 64, i = lo + (lane + 1) * step;
      const int hits = __popcll(__ballot(i <= lo + len && cu[min(i, lo + len)] <= r));
      const int last = lo + len;
      lo += hits * step;
      len = min(step - 1, last - lo);
    }
    const int i = lo + 1 + lane;
    lo += __popcll(__ballot(lane < len && cu[min(i, s.n_seqs)] <= r));
    seq = __builtin_amdgcn_readfirstlane(lo);
    if (seq >= s.n_seqs || cu[seq] > r) return out;
    back = cu[seq + 1] - r;
    if (back <= 0) return out;
  }
  out.owned = 1;
  const int64_t pos = (int64_t)s.len[seq] - back;
  if (pos < 0 || (pos >> c.page_shift) >= s.pages_per_seq) return out;
  const int page = s.table[(int64_t)seq * s.table_stride + (pos >> c.page_shift)];
  if (page < 0 || page >= c.n_pages) return out;
  out.page = page;
  out.at = (int)pos & ((1 << c.page_shift) - 1);
  return out;
}

// Lanes that share a head's row, eight values each; those past the row's end idle.
template <int HD>
constexpr int kv_lanes() { return HD <= 64 ? 8 : HD <= 128 ? 16 : 32; }

// Largest of the group's values, in every lane of it.
template <int LANES>
__device__ __forceinline__ uint32_t group_max(uint32_t v) {
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o, 64));
  return v;
}

// The codes of eight values (bf16 pairs) of a row whose largest magnitude has the bits `top`.  code = round(x Q / m): both
// are taken times a power of two that brings m into [1/2, 1), so nothing overflows; x Q is exact (8 + 7 bits), and the
// corrected product is the correctly rounded quotient: one of two 8-bit numbers and Q lies on a tie or at least 2^-9 of a
// step from it, so every code is the one of exact arithmetic.
template <int FMT>
__device__ __forceinline__ uint2 quantise8(u32x4 x, uint32_t top) {
  const float m = __uint_as_float(top << 16);
  const int e = __builtin_amdgcn_frexp_expf(m);
  const float a = ldexpf(m, -e), inv = __builtin_amdgcn_rcpf(a), q = kv_qmax<FMT>();
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float n = ldexpf(i & 1 ? bf16hi_to_f32(x[i / 2]) : bf16lo_to_f32(x[i / 2]), -e) * q;
    const float t = n * inv;
    y[i] = fmaf(fmaf(-t, a, n), inv, t);
  }
  uint32_t w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if constexpr (FMT == ET_KV_E4M3) {
      uint32_t v = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i], y[4 * i + 1], 0, false);
      w[i] = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i + 2], y[4 * i + 3], v, true);
    } else {
      w[i] = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) w[i] |= ((uint32_t)(int)rintf(y[4 * i + k]) & 0xFFu) << (8 * k);
    }
  }
  return make_uint2(w[0], w[1]);
}

// The values (bf16 pairs) of eight codes.  code * m is exact in float32 (8 + 8 bits; m is taken times 2^-9, so it does not
// overflow), the division is the only rounding before the one to bf16.
template <int FMT>
__device__ __forceinline__ u32x4 dequantise8(uint2 codes, uint16_t top) {
  const float m = __uint_as_float((uint32_t)top << 16) * 0x1p-9f, q = kv_qmax<FMT>() * 0x1p-9f;
  u32x4 out;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t w = i < 2 ? codes.x : codes.y;
    float a, b;
    if constexpr (FMT == ET_KV_E4M3) {
      const auto v = i & 1 ? __builtin_amdgcn_cvt_pk_f32_fp8(w, true) : __builtin_amdgcn_cvt_pk_f32_fp8(w, false);
      a = v[0];
      b = v[1];
    } else {
      a = (float)(int8_t)(w >> (16 * (i & 1)));
      b = (float)(int8_t)(w >> (16 * (i & 1) + 8));
    }
    out[i] = cvt_pk_bf16(a * m / q, b * m / q);
  }
  return out;
}

// One workgroup per row of tokens; its wavefronts share the row's 2 kv_heads head rows (keys first).
template <int HD, int FMT, bool STORE>
__global__ __launch_bounds__(256) void kv_rows_kernel(const int32_t *cu, KvSeqs s, KvPages c, uint16_t *k, int64_t k_stride,
                                                      uint16_t *v, int64_t v_stride) {
  using Lay = KvLayout<HD, FMT>;
  constexpr int LANES = kv_lanes<HD>(), PER = 64 / LANES;
  const int r = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const KvPlace place = kv_place(cu, r, s, c);
  if (!place.owned || (STORE && place.page < 0)) return;
  const int n = 1 << c.page_shift, sub = lane % LANES;
  const bool have = place.page >= 0, in_row = sub * 8 < HD;
  for (int j = wave * PER + lane / LANES; j < 2 * c.kv_heads; j += 4 * PER) {
    const bool value = j >= c.kv_heads;
    const int h = value ? j - c.kv_heads : j;
    uint16_t *row = (value ? v + r * v_stride : k + r * k_stride) + h * HD + sub * 8;
    char *head = c.data + (have ? place.page : 0) * c.page_bytes + (int64_t)h * Lay::head_bytes(n);
    char *cell = head + (value ? Lay::values(n) : 0) + place.at * Lay::kRow + sub * 8 * Lay::kBytes;
    uint16_t *top_at = reinterpret_cast<uint16_t *>(head + (value ? Lay::value_max(n) : Lay::key_max(n))) + place.at;
    if constexpr (STORE) {
      u32x4 x{0, 0, 0, 0};
      if (in_row) x = *reinterpret_cast<const u32x4 *>(row);
      if constexpr (FMT == ET_KV_BF16) {
        if (in_row) *reinterpret_cast<u32x4 *>(cell) = x;
      } else {
        uint32_t top = 0;                                  // of the magnitudes' bits: an infinity or a NaN is above all numbers
#pragma unroll
        for (int i = 0; i < 4; ++i) top = max(top, max(x[i] & 0x7FFFu, x[i] >> 16 & 0x7FFFu));
        top = group_max<LANES>(top);
        uint2 codes = make_uint2(0, 0);
        if (top >= 0x7F80u) top = 0x7FC0u;
        else if (top) codes = quantise8<FMT>(x, top);
        if (in_row) *reinterpret_cast<uint2 *>(cell) = codes;
        if (sub == 0) *top_at = (uint16_t)top;
      }
    } else if (in_row) {
      u32x4 x{0, 0, 0, 0};
      if (have) {
        if constexpr (FMT == ET_KV_BF16) x = *reinterpret_cast<const u32x4 *>(cell);
        else x = dequantise8<FMT>(*reinterpret_cast<const uint2 *>(cell), *top_at);
      }
      *reinterpret_cast<u32x4 *>(row) = x;
    }
  }
}

int check_kv(const et_kv_cache *c, const et_kv_seqs *s) {
  ET_REQUIRE(c != nullptr, "cache is NULL");
  ET_REQUIRE(s != nullptr, "seqs is NULL");
  ET_REQUIRE(c->format >= ET_KV_BF16 && c->format <= ET_KV_INT8, "unknown cache format %d", c->format);
  ET_REQUIRE(c->n_kv_heads >= 1 && c->n_kv_heads <= 1024, "n_kv_heads = %d must be in [1, 1024]", c->n_kv_heads);
  ET_REQUIRE(c->n_pages >= 1, "n_pages = %d must be at least 1", c->n_pages);
  if (et_kv_page_bytes(c->page_size, c->n_kv_heads, c->head_dim, c->format) == 0) {
    set_error("page_size %d (16, 32, 64, 128, 256) or head_dim %d (64, 80, 96, 128, 256) of the cache is not supported", c->page_size,
              c->head_dim);
    return ET_ERR_UNSUPPORTED;
  }
  ET_REQUIRE(c->data_dev != nullptr && (uintptr_t)c->data_dev % 16 == 0, "data_dev of the cache is NULL or not aligned to 16 bytes");
  ET_REQUIRE(s->n_seqs >= 0, "n_seqs = %d is negative", s->n_seqs);
  ET_REQUIRE(s->pages_per_seq >= 1 && s->table_stride >= s->pages_per_seq && (int64_t)s->pages_per_seq * c->page_size <= 1 << 30,
             "pages_per_seq = %d must be at least 1, at most table_stride = %d, and at most 2^30 tokens", s->pages_per_seq, s->table_stride);
  ET_REQUIRE(s->n_seqs == 0 || (s->page_table_dev && s->kv_len_dev), "page_table_dev or kv_len_dev is NULL");
  return ET_OK;
}

KvPages kv_pages(const et_kv_cache &c) {
  return {static_cast<char *>(c.data_dev), (int64_t)et_kv_page_bytes(c.page_size, c.n_kv_heads, c.head_dim, c.format), c.n_pages,
          __builtin_ctz(c.page_size), c.n_kv_heads};
}
KvSeqs kv_seqs(const et_kv_seqs &s) { return {s.page_table_dev, s.kv_len_dev, s.table_stride, s.pages_per_seq, s.n_seqs}; }

static int check_rows(const et_kv_cache *cache, const et_kv_seqs *seqs, const int32_t *cu, int rows, const void *k, int64_t k_stride,
                      const void *v, int64_t v_stride) {
  int rc;
  if ((rc = check_kv(cache, seqs))) return rc;
  ET_REQUIRE(rows >= 0, "rows = %d is negative", rows);
  ET_REQUIRE(cu || rows == seqs->n_seqs, "rows = %d without cu_rows_dev must be n_seqs = %d", rows, seqs->n_seqs);
  if (rows == 0) return ET_OK;
  const int64_t width = (int64_t)cache->n_kv_heads * cache->head_dim;
  ET_REQUIRE(k && v && (uintptr_t)k % 16 == 0 && (uintptr_t)v % 16 == 0, "a key or value pointer is NULL or not aligned to 16 bytes");
  ET_REQUIRE(k_stride >= width && v_stride >= width && k_stride % 8 == 0 && v_stride % 8 == 0,
             "row strides %lld and %lld must be multiples of 8 and at least %lld", (long long)k_stride, (long long)v_stride, (long long)width);
  return ET_OK;
}

template <bool STORE>
static int launch_rows(const et_kv_cache &cache, const et_kv_seqs &seqs, const int32_t *cu, int rows, uint16_t *k, int64_t k_stride,
                       uint16_t *v, int64_t v_stride, hipStream_t stream) {
  if (rows == 0 || seqs.n_seqs == 0) return ET_OK;
  return kv_dispatch(cache.head_dim, cache.format, [&](auto hd, auto fmt) {
    kv_rows_kernel<hd.value, fmt.value, STORE><<<rows, 256, 0, stream>>>(cu, kv_seqs(seqs), kv_pages(cache), k, k_stride, v, v_stride);
    ET_LAUNCH_CHECK();
    return ET_OK;
  });
}

}  // namespace et

using namespace et;

extern "C" {

size_t et_kv_page_bytes(int32_t page_size, int32_t n_kv_heads, int32_t head_dim, int32_t format) {
  const bool page_ok = page_size >= 16 && page_size <= 256 && (page_size & (page_size - 1)) == 0;
  const bool head_ok = head_dim == 64 || head_dim == 80 || head_dim == 96 || head_dim == 128 || head_dim == 256;
  if (!page_ok || !head_ok || n_kv_heads < 1 || n_kv_heads > 1024 || format < ET_KV_BF16 || format > ET_KV_INT8) return 0;
  const size_t row = format == ET_KV_BF16 ? 2 * (size_t)head_dim : (size_t)head_dim + 2;
  return 2 * row * (size_t)page_size * (size_t)n_kv_heads;
}

int et_kv_append(const et_kv_cache *cache, const et_kv_seqs *seqs, const int32_t *cu_rows_dev, int32_t rows, const uint16_t *k_dev,
                 int64_t k_stride, const uint16_t *v_dev, int64_t v_stride, void *hip_stream) {
  int rc;
  if ((rc = check_rows(cache, seqs, cu_rows_dev, rows, k_dev, k_stride, v_dev, v_stride))) return rc;
  return launch_rows<true>(*cache, *seqs, cu_rows_dev, rows, const_cast<uint16_t *>(k_dev), k_stride, const_cast<uint16_t *>(v_dev),
                           v_stride, static_cast<hipStream_t>(hip_stream));
}

int et_kv_read(const et_kv_cache *cache, const et_kv_seqs *seqs, const int32_t *cu_rows_dev, int32_t rows, uint16_t *k_out_dev,
               int64_t k_stride, uint16_t *v_out_dev, int64_t v_stride, void *hip_stream) {
  int rc;
  if ((rc = check_rows(cache, seqs, cu_rows_dev, rows, k_out_dev, k_stride, v_out_dev, v_stride))) return rc;
  return launch_rows<false>(*cache, *seqs, cu_rows_dev, rows, k_out_dev, k_stride, v_out_dev, v_stride,
                            static_cast<hipStream_t>(hip_stream));
}

}  // extern "C"
