// Launches of the paired-CTA attention kernels over a bf16 cache (attn_tc_pair.cuh).
#include "attn_tc_pair.cuh"

namespace quoka {

quoka_status launch_attn_tc_pair(const quoka_params* p, const DevParams& P, const void* q, const void* k, const void* v,
                                 const int32_t* k_idx, const int32_t* k_cnt, void* out, float* lse, cudaStream_t st,
                                 bool after_selection, const AttnPlan& plan) {
  CUtensorMap tm_q;
  if (!encode_q_tensor_map(&tm_q, P, q)) return QUOKA_ERR_CUDA;
  CUtensorMap tm_k, tm_v;
  if (!encode_kv_tensor_map(&tm_k, p, k, 64) || !encode_kv_tensor_map(&tm_v, p, v, 64)) return QUOKA_ERR_CUDA;
  return launch_attn_plan(p, P, plan, pick_attn_tc_pair<0>, "attn_tc_pair", /*cluster=*/2, kAttnThreads, attn_tc_pair_smem<0>(plan), tm_q, tm_k, tm_v, k, v, k_idx, k_cnt, out, lse,
                          st, after_selection);
}

}  // namespace quoka
