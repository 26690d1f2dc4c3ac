// Launch functions of the microscaled cache's kernels (host side).  The scale arrays come in DevParams.
#pragma once

#include <type_traits>

#include "common.cuh"

namespace quoka {

// fn(element of the type, integral constant of the format, of head_dim) for the call's data type, format and head_dim.
template <typename F>
inline cudaError_t mx_dispatch(int dtype, int fmt, int d, F&& fn) {
  const auto with = [&](auto elem) {
    const auto of_format = [&](auto f) {
      return d == 128 ? fn(elem, f, std::integral_constant<int, 128>{}) : fn(elem, f, std::integral_constant<int, 64>{});
    };
    return fmt == QUOKA_KV_MXFP8 ? of_format(std::integral_constant<int, QUOKA_KV_MXFP8>{})
                                 : of_format(std::integral_constant<int, QUOKA_KV_MXFP4>{});
  };
  return dtype == QUOKA_BF16 ? with(__nv_bfloat16{}) : with(0.f);
}

cudaError_t launch_append_kv_mx(const DevParams& P, int dtype, int fmt, const void* k_new, const void* v_new, void* k_cache, void* v_cache,
                                uint8_t* k_scale, uint8_t* v_scale, float* k_inv_norm, cudaStream_t st);
// first < 0: rows T_s ..; v_cache == nullptr: keys only
cudaError_t launch_read_kv_mx(const DevParams& P, int dtype, int fmt, const void* k_cache, const void* v_cache, int first, int n_rows,
                              void* k_out, void* v_out, cudaStream_t st);
cudaError_t launch_score_keys_mx_simt(const DevParams& P, int dtype, int fmt, const void* qbar, const void* k, float* scores, cudaStream_t st);
cudaError_t launch_attn_mx_simt(const DevParams& P, int dtype, int fmt, const void* q, const void* k, const void* v, const int32_t* k_idx,
                                const int32_t* k_cnt, void* out, float* lse, cudaStream_t st);

// Eight retained queries or fewer (score_few_mx.cu)
bool score_few_mx_applies(const quoka_params* p);
cudaError_t launch_score_few_mx(const DevParams& P, int fmt, const void* qbar, const void* k, float* scores, cudaStream_t st, bool chained);
// A few query rows per KV head (decode_mx.cu); parts: scratch of decode_mx_scratch_bytes
bool decode_mx_applies(const quoka_params* p);
size_t decode_mx_scratch_bytes(const quoka_params* p);
cudaError_t launch_decode_mx(const DevParams& P, int fmt, const void* q, const void* k, const void* v, const int32_t* k_idx, const int32_t* k_cnt, void* out,
                             float* lse, float* parts, cudaStream_t st, bool chained);

}  // namespace quoka
