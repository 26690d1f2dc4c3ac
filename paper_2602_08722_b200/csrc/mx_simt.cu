// Scalar fp32 scoring and attention over the microscaled cache: what serves f32 queries, and the on-device cross-check of the
// other kernels (QUOKA_IMPL_SIMT, both data types).  A warp per key, or per query row; the lanes split head_dim.
// Sums as in attn_simt_kernel (compensated, online softmax).
// Nothing is shared between the rows of a chunk, so f32 calls are far slower than over an f32 cache, which has tiled kernels.  us, MXFP8 / f32 cache,
// 32 heads of 8, d 128, 256 queries, 1024 of 8192 rows: scoring 64 queries 321 / 40, attention 3660 / 204; one query, 512 of 8192: 24 / 10, 451 / 12.
#include <algorithm>

#include "mx.cuh"
#include "mx_host.cuh"

namespace quoka {

// This lane's D / 32 elements of a cache row.
template <int FMT, int D>
__device__ __forceinline__ void load_lane(const DevParams& P, const uint8_t* cache, const uint8_t* scale, int s, int h, int t, int lane,
                                          float (&x)[D / 32]) {
  constexpr int NE = D / 32;
  const uint8_t* row = cache + kv_row_offset(P, s, h, t) * kMxBits<FMT> / 8;
  const float sc = mx_scale(__ldg(scale + mx_scale_index<D>(P, s, h, t) + lane * NE / kMxBlock));
#pragma unroll
  for (int i = 0; i < NE; ++i) {
    const int e = lane * NE + i;
    const uint32_t code = FMT == QUOKA_KV_MXFP8 ? __ldg(row + e) : __ldg(row + e / 2) >> (4 * (e % 2)) & 0xFu;
    x[i] = mx_element<FMT>(code) * sc;
  }
}

template <typename E, int FMT, int D>
__global__ void __launch_bounds__(256) score_keys_mx_simt_kernel(DevParams P, const E* __restrict__ qbar, const uint8_t* __restrict__ k,
                                                                 float* __restrict__ scores) {
  constexpr int NE = D / 32;
  const int lane = threadIdx.x & 31, s = blockIdx.z, kv = blockIdx.y, T = __ldg(P.ctx_len + s);
  for (int t = (blockIdx.x * blockDim.x + threadIdx.x) >> 5; t < T; t += (gridDim.x * blockDim.x) >> 5) {
    float kx[NE];
    load_lane<FMT, D>(P, k, P.k_scale, s, kv, t, lane, kx);
    float nn = 0.f, best = -INFINITY, total = 0.f;
#pragma unroll
    for (int i = 0; i < NE; ++i) nn = fmaf(kx[i], kx[i], nn);
    nn = warp_sum(nn);
    const E* qb = qbar + ((int64_t)s * P.n_kv + kv) * P.n_sel * D + lane * NE;
    for (int j = 0; j < P.n_sel; ++j) {
      float dot = 0.f;
#pragma unroll
      for (int i = 0; i < NE; ++i) dot = fmaf(kx[i], to_f32(qb[(int64_t)j * D + i]), dot);
      dot = warp_sum(dot);
      best = fmaxf(best, dot);
      total += dot;
    }
    const float agg = P.agg_mean ? total / (float)P.n_sel : best;
    const float inv = P.score_dot ? 1.f : P.k_inv_norm ? __ldg(P.k_inv_norm + kv_norm_index(P, s, kv, t)) : 1.f / fmaxf(sqrtf(nn), kNormEps);
    if (lane == 0) scores[((int64_t)s * P.n_kv + kv) * P.max_ctx + t] = agg * inv;
  }
}

template <typename E, int FMT, int D>
__global__ void __launch_bounds__(256) attn_mx_simt_kernel(DevParams P, const E* __restrict__ q, const uint8_t* __restrict__ k,
                                                           const uint8_t* __restrict__ v, const int32_t* __restrict__ k_idx,
                                                           const int32_t* __restrict__ k_cnt, E* __restrict__ out, float* __restrict__ lse) {
  constexpr int NE = D / 32;
  const int64_t warp = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) >> 5;
  const int lane = threadIdx.x & 31;
  if (warp >= (int64_t)P.batch * P.n_q * P.chunk) return;
  const int r = (int)(warp % P.chunk), h = (int)(warp / P.chunk % P.n_q), s = (int)(warp / ((int64_t)P.chunk * P.n_q));
  const int kv = h / P.group, T = __ldg(P.ctx_len + s), n_cached = k_idx ? __ldg(k_cnt + s) : T;
  const int32_t* idx = k_idx ? k_idx + ((int64_t)s * P.n_kv + kv) * P.budget_cap : nullptr;
  float qv[NE];
  load_vec<E, NE>(q + (int64_t)s * P.q_sb + (int64_t)h * P.q_sh + (int64_t)r * P.q_st + lane * NE, qv);
#pragma unroll
  for (int i = 0; i < NE; ++i) qv[i] *= P.scale;
  float m = -INFINITY, l = 0.f, cl = 0.f, o[NE], co[NE];
#pragma unroll
  for (int i = 0; i < NE; ++i) { o[i] = 0.f; co[i] = 0.f; }
  for (int u = 0; u < n_cached + r + 1; ++u) {
    const int t = u < n_cached ? (idx ? __ldg(idx + u) : u) : T + (u - n_cached);
    float kx[NE], vx[NE];
    load_lane<FMT, D>(P, k, P.k_scale, s, kv, t, lane, kx);
    load_lane<FMT, D>(P, v, P.v_scale, s, kv, t, lane, vx);
    float dot = 0.f;
#pragma unroll
    for (int i = 0; i < NE; ++i) dot = fmaf(qv[i], kx[i], dot);
    dot = warp_sum(dot);
    const float m_new = fmaxf(m, dot), alpha = m == m_new ? 1.f : expf(m - m_new), p = expf(dot - m_new);
    l *= alpha; cl *= alpha;
    const float y = p - cl, z = l + y;
    cl = (z - l) - y;
    l = z;
#pragma unroll
    for (int i = 0; i < NE; ++i) {
      o[i] *= alpha; co[i] *= alpha;
      const float yi = p * vx[i] - co[i], zi = o[i] + yi;
      co[i] = (zi - o[i]) - yi;
      o[i] = zi;
    }
    m = m_new;
  }
  const float inv = 1.f / l;
#pragma unroll
  for (int i = 0; i < NE; ++i) o[i] *= inv;
  store_vec<E, NE>(out + (int64_t)s * P.o_sb + (int64_t)h * P.o_sh + (int64_t)r * P.o_st + lane * NE, o);
  if (lse && lane == 0) lse[((int64_t)s * P.n_q + h) * P.chunk + r] = m + logf(l);
}

cudaError_t launch_score_keys_mx_simt(const DevParams& P, int dtype, int fmt, const void* qbar, const void* k, float* scores, cudaStream_t st) {
  const unsigned per_head = (unsigned)std::min<int64_t>(((int64_t)P.max_ctx + 7) / 8, 4096);
  const cudaError_t e = mx_dispatch(dtype, fmt, P.d, [&](auto elem, auto f, auto d) {
    using E = decltype(elem);
    return launch_kernel("score_keys_mx_simt", score_keys_mx_simt_kernel<E, f.value, d.value>, dim3(per_head, P.n_kv, P.batch), dim3(256), 0, st, 1,
                         false, P, (const E*)qbar, (const uint8_t*)k, scores);
  });
  if (e != cudaSuccess) return e;
  count_launch();
  return cudaGetLastError();
}

cudaError_t launch_attn_mx_simt(const DevParams& P, int dtype, int fmt, const void* q, const void* k, const void* v, const int32_t* k_idx,
                                const int32_t* k_cnt, void* out, float* lse, cudaStream_t st) {
  const int64_t warps = (int64_t)P.batch * P.n_q * P.chunk;
  const cudaError_t e = mx_dispatch(dtype, fmt, P.d, [&](auto elem, auto f, auto d) {
    using E = decltype(elem);
    return launch_kernel("attn_mx_simt", attn_mx_simt_kernel<E, f.value, d.value>, dim3((unsigned)((warps + 7) / 8)), dim3(256), 0, st, 1, false, P,
                         (const E*)q, (const uint8_t*)k, (const uint8_t*)v, k_idx, k_cnt, (E*)out, lse);
  });
  if (e != cudaSuccess) return e;
  count_launch();
  return cudaGetLastError();
}

}  // namespace quoka
