// Launches of the tensor-core attention over a microscaled cache: the plan of the bf16 kernels, whose tiles, products and softmax
// these share (attn_tc.cuh, attn_tc_pair.cuh), with the loaders of attn_mx_loader.cuh.
#include "attn_tc.cuh"
#include "attn_tc_pair.cuh"

namespace quoka {

AttnKernel pick_attn_mx8(bool pair, int d, bool sparse, bool parts, bool in_cluster);
AttnKernel pick_attn_mx4(bool pair, int d, bool sparse, bool parts, bool in_cluster);

bool attn_mx_tc_supported(const quoka_params* p) {
  if (p->dtype != QUOKA_BF16) return false;
  // the loaders count cache rows, and units of 16 elements, in 32 bits
  const int64_t rows = (p->page_size ? p->kv_rows * kPage : (int64_t)p->batch * p->kv_rows) * p->n_kv_heads;
  return kv_places_fit(p, 16) && rows < (int64_t)0xFFFFFFFFll;
}

template <bool PAIR, bool WIDE, bool FP8>
static AttnKernel pick(bool sparse, bool parts, bool in_cluster) {
  return (FP8 ? pick_attn_mx8 : pick_attn_mx4)(PAIR, WIDE ? 128 : 64, sparse, parts, in_cluster);
}

quoka_status launch_attn_mx_tc(const quoka_params* p, const DevParams& P0, int fmt, const void* q, const void* k, const void* v,
                               const int32_t* k_idx, const int32_t* k_cnt, void* out, float* lse, cudaStream_t st, bool after_selection,
                               const AttnPlan& plan) {
  DevParams P = attn_of_plan(P0, plan);
  P.list_of_selection = after_selection ? 1 : 0;
  CUtensorMap tm_q, tm_k, tm_v;
  if (!encode_q_tensor_map(&tm_q, P, q)) return QUOKA_ERR_CUDA;
  // (a pair's CTA takes half of V's columns)
  if (!encode_mx_tensor_map(&tm_k, p, fmt, k, P.d) || !encode_mx_tensor_map(&tm_v, p, fmt, v, plan.ctas == 2 ? 64 : P.d)) return QUOKA_ERR_CUDA;
  const bool pair = plan.ctas == 2, wide = P.d == 128, fp8 = fmt == QUOKA_KV_MXFP8;
  AttnKernel (*const kernel)(bool, bool, bool) = pair ? (fp8 ? pick<true, true, true> : pick<true, true, false>)
                                                 : wide ? (fp8 ? pick<false, true, true> : pick<false, true, false>)
                                                        : (fp8 ? pick<false, false, true> : pick<false, false, false>);
  const size_t smem = pair ? (fp8 ? attn_tc_pair_smem<QUOKA_KV_MXFP8>(plan) : attn_tc_pair_smem<QUOKA_KV_MXFP4>(plan))
                      : wide ? (fp8 ? attn_tc_smem<128, QUOKA_KV_MXFP8>() : attn_tc_smem<128, QUOKA_KV_MXFP4>())
                             : (fp8 ? attn_tc_smem<64, QUOKA_KV_MXFP8>() : attn_tc_smem<64, QUOKA_KV_MXFP4>());
  return launch_attn_plan(p, P, plan, kernel, pair ? "attn_tc_pair_mx" : "attn_tc_mx", pair ? 2 : 1, kMxAttnThreads,
                          smem, tm_q, tm_k, tm_v, k, v, k_idx, k_cnt, out, lse, st,
                          after_selection);
}

}  // namespace quoka
