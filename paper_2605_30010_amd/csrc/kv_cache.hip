// Storing keys and values in a paged cache, in bfloat16 or 8 bits, and reading them back.
#include <algorithm>
#include <type_traits>

#include "kv_cache.h"
#include "mfma_common.h"

namespace et {

// Where up to 64 consecutive rows of new (or wanted) tokens lie: lane i's row is first + i.  cu ascends; whatever it holds, the
// answer is inside the cache or "none".
struct KvPlace {
  int owned;                 // the row belongs to a sequence
  int page, at;              // page < 0: no place in the cache; at: token of the page
};
struct KvSeqs {
  const int32_t *table, *len;
  int table_stride, pages_per_seq, n_seqs;
};

// The first row's sequence is found by up to 64 probes at a time (a batch of 64 sequences takes one load, 4096 two), those
// of the other rows by counting the range ends behind it.
__device__ __forceinline__ KvPlace kv_place(const int32_t *cu, int first, int count, const KvSeqs &s, int n_pages, int page_shift) {
  KvPlace out{0, -1, 0};
  const int lane = threadIdx.x & 63, r = first + lane;
  int seq = r, back = 1;                                  // back: the row's distance from the sequence's end
  bool mine = lane < count && r < s.n_seqs;
  if (cu) {
    int lo = 0, len = s.n_seqs;                           // cu[i] <= first holds for at least lo and at most lo + len of i = 1..n_seqs
    while (len > 64) {
      const int step = (len + 63) / 64, i = lo + (lane + 1) * step, last = lo + len;
      const int hits = __popcll(__ballot(i <= last && cu[min(i, last)] <= first));
      lo += hits * step;
      len = min(step - 1, last - lo);
    }
    seq = lo;
    for (int base = lo; base < s.n_seqs; base += 64) {
      const int i = base + 1 + lane;
      const bool inside = i <= s.n_seqs;
      const int end = cu[min(i, s.n_seqs)];
      for (int j = 0; j < count; ++j) {
        const int passed = __popcll(__ballot(inside && end <= first + j));
        seq += lane == j ? passed : 0;
      }
      if (!__builtin_amdgcn_readlane(inside && end <= first + count - 1, 63)) break;
    }
    mine = lane < count && seq < s.n_seqs && seq >= 0;
    if (mine) {
      mine = cu[seq] <= r && r < cu[seq + 1];
      back = cu[seq + 1] - r;
    }
  }
  if (mine) {
    out.owned = 1;
    const int64_t pos = (int64_t)s.len[seq] - back;
    if (pos >= 0 && (pos >> page_shift) < s.pages_per_seq) {
      const int page = s.table[(int64_t)seq * s.table_stride + (pos >> page_shift)];
      if (page >= 0 && page < n_pages) {
        out.page = page;
        out.at = (int)pos & ((1 << page_shift) - 1);
      }
    }
  }
  return out;
}

// Lanes that share a head's row, eight values each; those past the row's end idle.
template <int HD>
constexpr int kv_lanes() { return HD <= 64 ? 8 : HD <= 128 ? 16 : 32; }

// Largest of the group's values, in every lane of it: neighbours, pairs, mirrored halves of 8 and of 16 lanes.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp_max(uint32_t v) {
  return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, false));
}
template <int LANES>
__device__ __forceinline__ uint32_t group_max(uint32_t v) {
  v = dpp_max<0x141>(dpp_max<0x4E>(dpp_max<0xB1>(v)));
  if constexpr (LANES >= 16) v = dpp_max<0x140>(v);
  if constexpr (LANES >= 32) v = max(v, (uint32_t)__shfl_xor((int)v, 16, 64));
  return v;
}

// The codes of eight values (bf16 pairs) of a row whose largest magnitude has the bits `top`.  code = round(x Q / m): both
// are taken times a power of two that brings m into [1/2, 1), so nothing overflows; x Q is exact (8 + 9 bits), and the
// corrected product is the correctly rounded quotient.  A quotient of two 8-bit numbers times Q lies on a tie of the codes or at least 2^-13 of
// a step from it (the smallest e4m3 steps; 2^-9 elsewhere), so every code is the one of exact arithmetic.
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

// The values (bf16 pairs) of eight codes, code * m / Q rounded once.  The factor m / Q is taken as the sum of two float32
// numbers, hi the nearest: what is rounded to bfloat16 is then the quotient rounded to float32, and neither rounding can go astray, since a
// quotient of code m (16 bits at most) by Q lies on a tie of bfloat16 or at least 2^-17 from it, relatively.  For int8 codes
// hi alone does: 127 is prime, so no quotient is on a tie.
struct KvFactor {
  float hi, lo;
};
template <int FMT>
__device__ __forceinline__ KvFactor kv_factor(uint16_t top) {
  const float m = bf16_to_f32(top), q = kv_qmax<FMT>(), hi = m / q;
  return {hi, fmaf(-hi, q, m) * (1.f / q)};
}
template <int FMT>
__device__ __forceinline__ u32x4 dequantise8(uint2 codes, KvFactor f) {
  u32x4 out;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t w = i < 2 ? codes.x : codes.y;
    float a, b;
    if constexpr (FMT == ET_KV_E4M3) {
      const auto v = i & 1 ? __builtin_amdgcn_cvt_pk_f32_fp8(w, true) : __builtin_amdgcn_cvt_pk_f32_fp8(w, false);
      a = fmaf(v[0], f.hi, v[0] * f.lo);
      b = fmaf(v[1], f.hi, v[1] * f.lo);
    } else {
      a = (float)(int8_t)(w >> (16 * (i & 1))) * f.hi;
      b = (float)(int8_t)(w >> (16 * (i & 1) + 8)) * f.hi;
    }
    out[i] = cvt_pk_bf16(a, b);
  }
  return out;
}

// A workgroup takes up to 64 consecutive rows of tokens.  One wavefront finds their places; then groups of LANES lanes take the rows'
// heads in turn (a token's key heads, its value heads, the next token), kBatch of them with their loads in flight.  Bound by memory:
// the way to a place is a chain of four loads, so rows share it when there are many.  What is read or written once in long
// streams (new rows, unquantised cells, rows read back) goes past the caches: 391 MB of e4m3 codes read back 265 -> 254 us, 130 000
// rows of 4 heads of 80 73 -> 65, 134 MB of bfloat16 rows stored 110 -> 101; codes and the cells of a read do not gain by it.
constexpr int kBatch = 4;
template <int HD, int FMT, bool STORE>
__global__ __launch_bounds__(256) void kv_rows_kernel(const int32_t *cu, const int32_t *len, const int32_t *table, int n_seqs, int rows,
                                                      int per_block, int table_stride, int pages_per_seq, int page_shift, KvPages c,
                                                      uint16_t *k, int64_t k_stride, uint16_t *v, int64_t v_stride) {
  using Lay = KvLayout<HD, FMT>;
  constexpr int LANES = kv_lanes<HD>(), GROUPS = 256 / LANES;
  __shared__ int4 lds_place[64];                         // byte offset of the page (two words), token of the page, 0 / 1 / 2
  const int first = blockIdx.x * per_block, count = min(per_block, rows - first);
  if (threadIdx.x < 64) {
    const KvPlace p = kv_place(cu, first, count, KvSeqs{table, len, table_stride, pages_per_seq, n_seqs}, c.n_pages, page_shift);
    const int64_t page = max(p.page, 0) * c.page_bytes;
    lds_place[threadIdx.x] = make_int4((int)page, (int)(page >> 32), p.at, p.owned ? (p.page >= 0 ? 2 : 1) : 0);
  }
  const int n = 1 << page_shift, sub = threadIdx.x % LANES, heads2 = 2 * c.kv_heads, head_bytes = Lay::head_bytes(n);
  const int skip = GROUPS / heads2, over = GROUPS % heads2;           // tokens and heads from one turn of a group to its next
  int token = threadIdx.x / LANES / heads2, j = threadIdx.x / LANES % heads2;
  const bool in_row = sub * 8 < HD;
  __syncthreads();
  auto turns = [&](auto batch) {
    constexpr int N = decltype(batch)::value;
    u32x4 x[N];
    uint2 codes[N];
    uint16_t top[N];
    uint16_t *row[N];
    char *cell[N], *top_at[N];
    int go[N];                                           // 0: nothing to do, 1: no place in the cache, 2: a place
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int4 place = lds_place[min(token, 63)];
      go[i] = token < count ? place.w : 0;
      const bool value = j >= c.kv_heads;
      const int h = value ? j - c.kv_heads : j;
      row[i] = (value ? v + (first + (int64_t)token) * v_stride : k + (first + (int64_t)token) * k_stride) + h * HD + sub * 8;
      char *page = c.data + (int64_t)((uint64_t)(uint32_t)place.y << 32 | (uint32_t)place.x);
      const uint32_t head = (uint32_t)h * head_bytes;
      cell[i] = page + (head + (value ? Lay::values(n) : 0) + place.z * Lay::kRow + sub * 8 * Lay::kBytes);
      top_at[i] = page + (head + (value ? Lay::value_max(n) : Lay::key_max(n)) + place.z * 2);
      x[i] = u32x4{0, 0, 0, 0};
      codes[i] = make_uint2(0, 0);
      top[i] = 0;
      if (go[i] == 2 && in_row) {
        if constexpr (STORE) x[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(row[i]));
        else if constexpr (FMT == ET_KV_BF16) x[i] = *reinterpret_cast<const u32x4 *>(cell[i]);
        else {
          codes[i] = *reinterpret_cast<const uint2 *>(cell[i]);
          top[i] = *reinterpret_cast<const uint16_t *>(top_at[i]);
        }
      }
      token += skip;
      j += over;
      if (j >= heads2) j -= heads2, ++token;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if constexpr (STORE && FMT != ET_KV_BF16) {
        uint32_t most = 0;                                // of the magnitudes' bits: an infinity or a NaN is above all numbers
#pragma unroll
        for (int e = 0; e < 4; ++e) most = max(most, max(x[i][e] & 0x7FFFu, x[i][e] >> 16 & 0x7FFFu));
        most = group_max<LANES>(most);
        const bool number = most - 1u < 0x7F7Fu;          // neither 0 nor without end
        codes[i] = quantise8<FMT>(x[i], number ? most : 0x3F80u);
        if (most >= 0x7F80u) most = 0x7FC0u, codes[i] = make_uint2(0, 0);
        if (go[i] == 2 && in_row) *reinterpret_cast<uint2 *>(cell[i]) = codes[i];
        if (go[i] == 2 && sub == 0) *reinterpret_cast<uint16_t *>(top_at[i]) = (uint16_t)most;
      } else if constexpr (STORE) {
        if (go[i] == 2 && in_row) __builtin_nontemporal_store(x[i], reinterpret_cast<u32x4 *>(cell[i]));
      } else {
        if constexpr (FMT != ET_KV_BF16) x[i] = dequantise8<FMT>(codes[i], kv_factor<FMT>(top[i]));
        if (go[i] && in_row) __builtin_nontemporal_store(x[i], reinterpret_cast<u32x4 *>(row[i]));
      }
    }
  };
  int left = (count * heads2 + GROUPS - 1) / GROUPS;
  for (; left >= kBatch; left -= kBatch) turns(std::integral_constant<int, kBatch>());
  for (; left > 0; --left) turns(std::integral_constant<int, 1>());
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
// A launch takes fewer than 2^32 lanes, 256 a workgroup, and a workgroup at most 64 rows.
constexpr int kMaxBlocks = (1 << 24) - 1, kMaxRows = 64 * kMaxBlocks;
static int check_rows(const et_kv_cache *cache, const et_kv_seqs *seqs, const int32_t *cu, int rows, const void *k, int64_t k_stride,
                      const void *v, int64_t v_stride) {
  int rc;
  if ((rc = check_kv(cache, seqs))) return rc;
  ET_REQUIRE(rows >= 0 && rows <= kMaxRows, "rows = %d must be in [0, 2^30 - 64]", rows);
  ET_REQUIRE(cu || rows == seqs->n_seqs, "rows = %d without cu_rows_dev must be n_seqs = %d", rows, seqs->n_seqs);
  if (rows == 0) return ET_OK;
  const int64_t width = (int64_t)cache->n_kv_heads * cache->head_dim;
  ET_REQUIRE(k && v && (uintptr_t)k % 16 == 0 && (uintptr_t)v % 16 == 0, "a key or value pointer is NULL or not aligned to 16 bytes");
  ET_REQUIRE(k_stride >= width && v_stride >= width && k_stride % 8 == 0 && v_stride % 8 == 0,
             "row strides %lld and %lld must be multiples of 8 and at least %lld", (long long)k_stride, (long long)v_stride, (long long)width);
  return ET_OK;
}

// Rows of a workgroup: enough for a group of lanes to have four turns of copying or sixteen of quantising (at most the 64 that a
// wavefront locates), as long as a thousand workgroups remain.  Measured, us at 1 / 4 / 8 / 16 / 32 rows: 65 600 bfloat16 rows of 8 heads of
// 128 stored 116 / 110 / 112 / 118 / 118, e4m3 stored and read back 251 / 190 / 177 / 175 / 178; 130 000 bfloat16 rows of 4 heads of 80
// read 179 / 93 / 73 / 72 / 77; 5000 int8 rows of 4 heads of 128 stored and read back 17.7 / 12.9 / 15.1 / 19.0 / 26.7; at 16 / 32 / 64
// rows: 928 000 int8 rows of 3 heads of 64 read 293 / 261 / 251, 630 000 of one head of 128 stored and read back 259 / 222 / 220.
static int rows_per_block(int rows, const et_kv_cache &c) {
  const int lanes = c.head_dim <= 64 ? 8 : c.head_dim <= 128 ? 16 : 32, turns = c.format == ET_KV_BF16 ? 4 : 16;
  const int least = (int)(((int64_t)rows + kMaxBlocks - 1) / kMaxBlocks);
  return std::max(least, std::min({64, rows / 1024, turns * (256 / lanes) / (2 * c.n_kv_heads)}));
}

template <bool STORE>
static int launch_rows(const et_kv_cache &cache, const et_kv_seqs &seqs, const int32_t *cu, int rows, uint16_t *k, int64_t k_stride,
                       uint16_t *v, int64_t v_stride, hipStream_t stream) {
  if (rows == 0 || seqs.n_seqs == 0) return ET_OK;
  const KvPages c = kv_pages(cache);
  const int per_block = rows_per_block(rows, cache);
  return kv_dispatch(cache.head_dim, cache.format, [&](auto hd, auto fmt) {
    kv_rows_kernel<hd.value, fmt.value, STORE><<<(rows + per_block - 1) / per_block, 256, 0, stream>>>(
        cu, seqs.kv_len_dev, seqs.page_table_dev, seqs.n_seqs, rows, per_block, seqs.table_stride, seqs.pages_per_seq, c.page_shift, c,
        k, k_stride, v, v_stride);
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
