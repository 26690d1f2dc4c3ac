// C entry points of the microscaled cache: validation, workspace, launch sequencing.
#include <algorithm>

#include "api_host.cuh"
#include "mx.cuh"
#include "mx_host.cuh"

namespace quoka {

// What every call checks of its parameters and of the cache's description.
static quoka_status validate_mx(const quoka_params* p, const quoka_mx_cache* mx) {
  const quoka_status st = validate(p);
  if (st != QUOKA_OK) return st;
  if (!mx) return QUOKA_ERR_INVALID_ARG;
  if (mx->format != QUOKA_KV_MXFP8 && mx->format != QUOKA_KV_MXFP4) return QUOKA_ERR_INVALID_ARG;
  if (!mx->k_scale || !mx->v_scale || !aligned16(mx->k_scale) || !aligned16(mx->v_scale)) return QUOKA_ERR_INVALID_ARG;
  for (int64_t s : {p->kv_stride_b, p->kv_stride_h, p->kv_stride_t})       // whole blocks, and 16 bytes of either format
    if (s % kMxBlock != 0) return QUOKA_ERR_INVALID_ARG;
  return QUOKA_OK;
}

static DevParams make_dev_mx(const quoka_params* p, const quoka_mx_cache* mx, void* ws, const Workspace& w) {
  DevParams P = make_dev(p, ws, w);
  P.k_scale = mx->k_scale;
  P.v_scale = mx->v_scale;
  return P;
}

static quoka_status run_score_keys_mx(const quoka_params* p, const quoka_mx_cache* mx, const DevParams& P, const void* qbar, const void* k,
                                      float* scores, cudaStream_t st, bool chained = false) {
  if (p->max_ctx_len == 0) return QUOKA_OK;
  if (p->impl == QUOKA_IMPL_AUTO && score_keys_mx_tc_supported(p) && score_few_mx_applies(p)) {
    QUOKA_TRY_CUDA(launch_score_few_mx(P, mx->format, qbar, k, scores, st, chained));
    return QUOKA_OK;
  }
  if (p->impl != QUOKA_IMPL_SIMT && score_keys_mx_tc_supported(p)) return launch_score_keys_mx_tc(p, P, mx->format, qbar, k, scores, st, chained);
  if (p->impl == QUOKA_IMPL_TENSOR) return QUOKA_ERR_UNSUPPORTED;
  QUOKA_TRY_CUDA(launch_score_keys_mx_simt(P, p->dtype, mx->format, qbar, k, scores, st));
  return QUOKA_OK;
}

// The scratch of a few query rows' attention comes last and has to be there; that of unpacked rows comes last too and may be missing.
static size_t scratch_mx(const quoka_params* p) {
  return p->impl == QUOKA_IMPL_AUTO && p->dtype == QUOKA_BF16 && decode_mx_applies(p) ? decode_mx_scratch_bytes(p) : 0;
}
static quoka_status check_ws_mx(const quoka_params* p, void* ws, size_t ws_bytes) {
  const quoka_status st = check_ws(p, ws, ws_bytes);
  if (st != QUOKA_OK) return st;
  return ws_bytes < workspace_bytes_unsplit(p) + scratch_mx(p) ? QUOKA_ERR_WORKSPACE : QUOKA_OK;
}

// How an attention call is done: its plan, buffers, and scratch of unpacked rows.
struct MxAttn {
  AttnPlan plan;
  Workspace w;
  void* unpacked = nullptr;
};
static MxAttn plan_attn_mx(const quoka_params* p, void* ws, size_t ws_bytes, bool listed) {
  MxAttn a;
  const auto plan = [&](size_t room) { return listed ? attn_plan_sparse(p, budget_cap_of(p), room) : attn_plan_dense(p, room); };
  if (scratch_mx(p) > 0) {
    a.plan = plan(0);
    a.w = carve(p, ws);
    a.w.attn_partials = reinterpret_cast<float*>(static_cast<unsigned char*>(ws) + a.w.total);
    return a;
  }
  const size_t room = attn_room(p, ws_bytes), unpack = attn_mx_tc_supported(p) ? attn_unpack_bytes(p, listed) : 0;
  const bool unpacks = unpack > 0 && unpack <= room;
  a.plan = plan(unpacks ? room - unpack : room);
  a.w = carve(p, ws, unpacks ? ws_bytes - unpack : ws_bytes, &a.plan);
  if (unpacks) a.unpacked = static_cast<unsigned char*>(ws) + a.w.total;
  return a;
}

static quoka_status run_attn_mx(const quoka_params* p, const quoka_mx_cache* mx, const DevParams& P, const MxAttn& a, const void* q, const void* k,
                                const void* v, const int32_t* k_idx, const int32_t* k_cnt, void* out, float* lse, cudaStream_t st,
                                bool after_selection = false) {
  if (p->impl == QUOKA_IMPL_AUTO && attn_mx_tc_supported(p) && decode_mx_applies(p)) {
    QUOKA_TRY_CUDA(launch_decode_mx(P, mx->format, q, k, v, k_idx, k_cnt, out, lse, P.attn_partials, st, after_selection));
    return QUOKA_OK;
  }
  if (a.unpacked) return launch_attn_mx_unpacked(p, P, mx->format, q, k, v, k_idx, k_cnt, out, lse, a.unpacked, st, after_selection, a.plan);
  if (p->impl != QUOKA_IMPL_SIMT && attn_mx_tc_supported(p))
    return launch_attn_mx_tc(p, P, mx->format, q, k, v, k_idx, k_cnt, out, lse, st, after_selection, a.plan);
  if (p->impl == QUOKA_IMPL_TENSOR) return QUOKA_ERR_UNSUPPORTED;
  QUOKA_TRY_CUDA(launch_attn_mx_simt(P, p->dtype, mx->format, q, k, v, k_idx, k_cnt, out, lse, st));
  return QUOKA_OK;
}

}  // namespace quoka

using namespace quoka;

extern "C" {

quoka_status quoka_workspace_size_mx(const quoka_params* p, const quoka_mx_cache* mx, size_t* bytes) {
  if (!bytes) return QUOKA_ERR_INVALID_ARG;
  const quoka_status st = validate_mx(p, mx);
  if (st != QUOKA_OK) return st;
  size_t attn = 0;
  if (quoka_workspace_size(p, &attn) != QUOKA_OK) return QUOKA_ERR_INVALID_ARG;
  // (with the scratch of the shortest chunks, whatever this one's length: the last chunk of a prompt comes with the workspace of its longest)
  *bytes = std::max(attn + std::max(attn_unpack_bytes(p, true), attn_unpack_bytes(p, false)),
                    workspace_bytes_unsplit(p) + (p->dtype == QUOKA_BF16 ? decode_mx_scratch_bytes(p) : 0));
  return QUOKA_OK;
}

quoka_status quoka_append_kv_mx(const quoka_params* p, const quoka_mx_cache* mx, const void* k_new, const void* v_new, void* k_cache,
                                void* v_cache, float* k_inv_norm, void* ws, size_t ws_bytes, void* stream) {
  quoka_status st = validate_mx(p, mx);
  if (st != QUOKA_OK) return st;
  if (!k_new || !v_new || !k_cache || !v_cache) return QUOKA_ERR_INVALID_ARG;
  if (!aligned16(k_new) || !aligned16(v_new) || !aligned16(k_cache) || !aligned16(v_cache)) return QUOKA_ERR_INVALID_ARG;
  if ((st = check_ws_mx(p, ws, ws_bytes)) != QUOKA_OK) return st;
  const DevParams P = make_dev_mx(p, mx, ws, carve(p, ws));
  QUOKA_TRY_CUDA(launch_append_kv_mx(P, p->dtype, mx->format, k_new, v_new, k_cache, v_cache, mx->k_scale, mx->v_scale, k_inv_norm,
                                     static_cast<cudaStream_t>(stream)));
  return QUOKA_OK;
}

quoka_status quoka_read_kv_mx(const quoka_params* p, const quoka_mx_cache* mx, const void* k_cache, const void* v_cache, int32_t first_row,
                              int32_t n_rows, void* k_out, void* v_out, void* ws, size_t ws_bytes, void* stream) {
  quoka_status st = validate_mx(p, mx);
  if (st != QUOKA_OK) return st;
  if (!k_cache || !k_out || (v_cache == nullptr) != (v_out == nullptr)) return QUOKA_ERR_INVALID_ARG;
  if (!aligned16(k_cache) || !aligned16(v_cache) || !aligned16(k_out) || !aligned16(v_out)) return QUOKA_ERR_INVALID_ARG;
  if (first_row < QUOKA_FROM_CTX_LEN || n_rows < 0) return QUOKA_ERR_INVALID_ARG;
  if ((st = check_ws_mx(p, ws, ws_bytes)) != QUOKA_OK) return st;
  if (n_rows == 0) return QUOKA_OK;
  const DevParams P = make_dev_mx(p, mx, ws, carve(p, ws));
  QUOKA_TRY_CUDA(launch_read_kv_mx(P, p->dtype, mx->format, k_cache, v_cache, first_row, n_rows, k_out, v_out, static_cast<cudaStream_t>(stream)));
  return QUOKA_OK;
}

quoka_status quoka_score_keys_mx(const quoka_params* p, const quoka_mx_cache* mx, const void* qbar, const void* k_cache, float* scores, void* ws,
                                 size_t ws_bytes, void* stream) {
  quoka_status st = validate_mx(p, mx);
  if (st != QUOKA_OK) return st;
  if (!qbar || !k_cache || !scores || !aligned16(qbar) || !aligned16(k_cache)) return QUOKA_ERR_INVALID_ARG;
  if ((st = check_ws_mx(p, ws, ws_bytes)) != QUOKA_OK) return st;
  return run_score_keys_mx(p, mx, make_dev_mx(p, mx, ws, carve(p, ws)), qbar, k_cache, scores, static_cast<cudaStream_t>(stream));
}

quoka_status quoka_sparse_attn_mx(const quoka_params* p, const quoka_mx_cache* mx, const void* q, const void* k_cache, const void* v_cache,
                                  const int32_t* k_idx, const int32_t* k_cnt, void* out, float* lse, void* ws, size_t ws_bytes, void* stream) {
  quoka_status st = validate_mx(p, mx);
  if (st != QUOKA_OK) return st;
  if (!q || !k_cache || !v_cache || !k_idx || !k_cnt || !out) return QUOKA_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(out)) return QUOKA_ERR_INVALID_ARG;
  if ((st = check_ws_mx(p, ws, ws_bytes)) != QUOKA_OK) return st;
  const MxAttn a = plan_attn_mx(p, ws, ws_bytes, /*listed=*/true);
  return run_attn_mx(p, mx, make_dev_mx(p, mx, ws, a.w), a, q, k_cache, v_cache, k_idx, k_cnt, out, lse, static_cast<cudaStream_t>(stream));
}

quoka_status quoka_dense_chunk_attn_mx(const quoka_params* p, const quoka_mx_cache* mx, const void* q, const void* k_cache, const void* v_cache,
                                       void* out, float* lse, void* ws, size_t ws_bytes, void* stream) {
  quoka_status st = validate_mx(p, mx);
  if (st != QUOKA_OK) return st;
  if (!q || !k_cache || !v_cache || !out) return QUOKA_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(out)) return QUOKA_ERR_INVALID_ARG;
  if ((st = check_ws_mx(p, ws, ws_bytes)) != QUOKA_OK) return st;
  const MxAttn a = plan_attn_mx(p, ws, ws_bytes, /*listed=*/false);
  return run_attn_mx(p, mx, make_dev_mx(p, mx, ws, a.w), a, q, k_cache, v_cache, nullptr, nullptr, out, lse, static_cast<cudaStream_t>(stream));
}

quoka_status quoka_prefill_chunk_mx(const quoka_params* p, const quoka_mx_cache* mx, const void* q, const void* k_cache, const void* v_cache,
                                    void* out, int32_t* k_idx_out, int32_t* k_cnt_out, void* ws, size_t ws_bytes, void* stream) {
  quoka_status st = validate_mx(p, mx);
  if (st != QUOKA_OK) return st;
  if (!q || !k_cache || !v_cache || !out) return QUOKA_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(out)) return QUOKA_ERR_INVALID_ARG;
  if (p->impl == QUOKA_IMPL_TENSOR && ((p->max_ctx_len > 0 && !score_keys_mx_tc_supported(p)) || !attn_mx_tc_supported(p))) return QUOKA_ERR_UNSUPPORTED;
  if ((st = check_ws_mx(p, ws, ws_bytes)) != QUOKA_OK) return st;
  cudaStream_t cs = static_cast<cudaStream_t>(stream);
  const MxAttn a = plan_attn_mx(p, ws, ws_bytes, /*listed=*/true);
  const Workspace& w = a.w;
  const DevParams P = make_dev_mx(p, mx, ws, w);
  int32_t* k_idx = k_idx_out ? k_idx_out : w.k_idx;
  int32_t* k_cnt = k_cnt_out ? k_cnt_out : w.k_cnt;
  // The chain of launches of the bf16 call.
  if (p->max_ctx_len > 0) {
    if ((st = run_select_queries(p, P, q, w.q_idx, w.qbar, cs, attn_below_a_wave(p))) != QUOKA_OK) return st;
    if ((st = run_score_keys_mx(p, mx, P, w.qbar, k_cache, w.scores, cs, /*chained=*/true)) != QUOKA_OK) return st;
  } else if (P.attn_counters) {
    QUOKA_TRY_CUDA(cudaMemsetAsync(P.attn_counters, 0, P.n_attn_counters * sizeof(int32_t), cs));
  }
  QUOKA_TRY_CUDA(launch_select_keys(P, w.scores, k_idx, k_cnt, cs, /*chained=*/p->max_ctx_len > 0));
  return run_attn_mx(p, mx, P, a, q, k_cache, v_cache, k_idx, k_cnt, out, nullptr, cs, /*after_selection=*/true);
}

}  // extern "C"
