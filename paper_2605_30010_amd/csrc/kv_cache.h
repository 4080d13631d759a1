// The paged key-value cache: where a token's keys and values lie, and what a byte of them stands for.
#pragma once
#include "et_common.h"

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
// Byte offsets within a head's part of a page.
template <int HD, int FMT>
struct KvLayout {
  static constexpr int kBytes = FMT == ET_KV_BF16 ? 2 : 1;
  static constexpr int kRow = HD * kBytes;                         // bytes of one row
  static __host__ __device__ constexpr int values(int page_size) { return page_size * kRow; }
  static __host__ __device__ constexpr int key_max(int page_size) { return 2 * page_size * kRow; }
  static __host__ __device__ constexpr int value_max(int page_size) { return key_max(page_size) + 2 * page_size; }
  static __host__ __device__ constexpr int head_bytes(int page_size) { return key_max(page_size) + (FMT == ET_KV_BF16 ? 0 : 4 * page_size); }
};

int check_kv(const et_kv_cache *cache, const et_kv_seqs *seqs);   // ET_OK or an error with its message
KvPages kv_pages(const et_kv_cache &c);

// Calls f with the head width and the format as constants.
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

}  // namespace et
