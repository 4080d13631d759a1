// Attention of one new token per sequence over a paged key-value cache in 4 bits.
#include "paged_attention.h"

namespace et {

int launch_paged_mxfp4(int head_dim, const PagedLaunch &l) {
  return kv_dispatch_mxfp4(head_dim, [&](auto hd) { return launch_paged<hd.value, ET_KV_MXFP4>(l); });
}

}  // namespace et
