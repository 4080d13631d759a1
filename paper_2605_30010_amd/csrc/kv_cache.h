// The paged key-value cache: where a token's keys and values lie, and what a byte of them stands for.
#pragma once
#include <type_traits>

#include "mfma_common.h"

namespace et {

// Q of the 8-bit formats (the code of a row's largest magnitude).
template <int FMT>
constexpr float kv_qmax() { return FMT == ET_KV_INT8 ? 127.f : 448.f; }

// The cache as kernels take it.
struct KvPages {
  char *data;
  int64_t page_bytes;
  int32_t n_pages, page_shift;             // tokens per page = 1 << page_shift
  int32_t kv_heads;
};
// Dimensions that share an exponent in 4 bits (the last block of a row may be shorter).
constexpr int kMxBlock = 32;
constexpr int kv_mx_blocks(int head_dim) { return (head_dim + kMxBlock - 1) / kMxBlock; }
// Byte offsets within a head's part of a page.  What scales a row's codes stands behind both: a maximum of two bytes a row, or in 4 bits
// one byte a block, the keys' by token (a lane of the attention takes a token's keys), the values' by block (it takes several tokens'
// values of the same dimensions).
template <int HD, int FMT>
struct KvLayout {
  static constexpr int kBlocks = FMT == ET_KV_MXFP4 ? kv_mx_blocks(HD) : 0;
  static constexpr int kRow = FMT == ET_KV_BF16 ? 2 * HD : FMT == ET_KV_MXFP4 ? HD / 2 : HD;   // bytes of one row
  static constexpr int kEight = kRow * 8 / HD;                     // and of eight of its values
  static constexpr int kScale = FMT == ET_KV_BF16 ? 0 : FMT == ET_KV_MXFP4 ? kBlocks : 2;     // bytes that scale a row
  static __host__ __device__ constexpr int values(int page_size) { return page_size * kRow; }
  static __host__ __device__ constexpr int key_scale(int page_size) { return 2 * page_size * kRow; }
  static __host__ __device__ constexpr int value_scale(int page_size) { return key_scale(page_size) + kScale * page_size; }
  static __host__ __device__ constexpr int head_bytes(int page_size) { return 2 * page_size * (kRow + kScale); }
};

// bf16 pair of two 4-bit codes, byte SEL of w, times the power of two whose exponent field `unit` has (its other bits do not count: the
// conversion takes the exponent alone).  Exact, and NaN where the field is 255.
template <int SEL>
__device__ __forceinline__ uint32_t mx_pair(uint32_t w, uint32_t unit) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, __uint_as_float(unit), SEL));
}
__device__ __forceinline__ u32x4 mx_decode8(uint32_t w, uint32_t exponent) {
  const uint32_t unit = exponent << 23;
  return u32x4{mx_pair<0>(w, unit), mx_pair<1>(w, unit), mx_pair<2>(w, unit), mx_pair<3>(w, unit)};
}

int check_kv(const et_kv_cache *cache, const et_kv_seqs *seqs);   // ET_OK or an error with its message
KvPages kv_pages(const et_kv_cache &c);

// Calls f with the head width and the format as constants (not for 4 bits).
template <typename F>
int kv_dispatch(int head_dim, int format, F &&f) {
#define ET_KV_HD(hd)                                                                                      \
  case hd:                                                                                                \
    return format == ET_KV_BF16 ? f(std::integral_constant<int, hd>(), std::integral_constant<int, ET_KV_BF16>()) \
         : format == ET_KV_E4M3 ? f(std::integral_constant<int, hd>(), std::integral_constant<int, ET_KV_E4M3>()) \
                                : f(std::integral_constant<int, hd>(), std::integral_constant<int, ET_KV_INT8>());
  switch (head_dim) {
    ET_KV_HD(64)
    ET_KV_HD(80)
    ET_KV_HD(96)
    ET_KV_HD(128)
    ET_KV_HD(256)
  }
#undef ET_KV_HD
  set_error("head_dim %d of a key-value cache is not among 64, 80, 96, 128, 256", head_dim);
  return ET_ERR_UNSUPPORTED;
}
// The same for 4 bits, with the head width alone.
template <typename F>
int kv_dispatch_mxfp4(int head_dim, F &&f) {
  switch (head_dim) {
    case 64: return f(std::integral_constant<int, 64>());
    case 80: return f(std::integral_constant<int, 80>());
    case 96: return f(std::integral_constant<int, 96>());
    case 128: return f(std::integral_constant<int, 128>());
    case 256: return f(std::integral_constant<int, 256>());
  }
  set_error("head_dim %d of a key-value cache is not among 64, 80, 96, 128, 256", head_dim);
  return ET_ERR_UNSUPPORTED;
}

}  // namespace et
