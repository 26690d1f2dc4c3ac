// The tensor-core attention kernels over a microscaled cache of 4-bit elements (attn_mx_loader.cuh).
#include "attn_tc.cuh"
#include "attn_tc_pair.cuh"

namespace quoka {

AttnKernel pick_attn_mx4(bool pair, int d, bool sparse, bool parts, bool in_cluster) {
  if (pair) return pick_attn_tc_pair<QUOKA_KV_MXFP4>(sparse, parts, in_cluster);
  return d == 128 ? pick_attn_tc<128, QUOKA_KV_MXFP4>(sparse, parts, in_cluster) : pick_attn_tc<64, QUOKA_KV_MXFP4>(sparse, parts, in_cluster);
}

}  // namespace quoka
