// What the files with the C entry points share: validation, workspace carving, the device copy of the parameters.
#pragma once

#include "common.cuh"
#include "tensor_kernels.cuh"

namespace quoka {

struct Workspace {
  int32_t* status;
  int32_t* q_idx;
  void* qbar;
  float* scores;
  int32_t* k_idx;
  int32_t* k_cnt;
  float* attn_partials;      // split attention of small grids: partial results and arrival counters, or null
  int32_t* attn_counters;
  int n_attn_counters;
  size_t total;
};

int budget_cap_of(const quoka_params* p);
Workspace carve(const quoka_params* p, void* ws, size_t ws_bytes = 0, const AttnPlan* plan = nullptr);
size_t attn_room(const quoka_params* p, size_t ws_bytes);
quoka_status validate(const quoka_params* p);
bool aligned16(const void* ptr);
quoka_status check_ws(const quoka_params* p, void* ws, size_t ws_bytes);
DevParams make_dev(const quoka_params* p, void* ws, const Workspace& w);
DevParams make_dev(const quoka_params* p, void* ws);
quoka_status run_select_queries(const quoka_params* p, const DevParams& P, const void* q, int32_t* q_idx, void* qbar, cudaStream_t st,
                                bool early = false);

#define QUOKA_TRY_CUDA(expr)                          \
  do {                                                \
    cudaError_t e_ = (expr);                          \
    if (e_ != cudaSuccess) return QUOKA_ERR_CUDA;     \
  } while (0)

}  // namespace quoka
