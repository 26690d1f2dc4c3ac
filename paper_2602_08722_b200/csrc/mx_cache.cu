// Writing the microscaled cache and reading it back.
//
// append: the chunk's K and V, dense [b][n_KV][C][D], go to cache rows T_s + r as blocks of 32 elements and a scale byte each.
//   A lane holds 8 elements of K and the same 8 of V, four lanes a block: its largest magnitude in two shuffles, the elements by
//   the conversion instruction.  The inverse norm of a key row is that of the values the cache then holds.
// read: cache rows first .. first + n - 1 to dense [b][n_KV][n][D] tensors; rows at and beyond T_s + C are left as they were.
//   A lane turns 8 elements of K and of V into 16 (bf16) or 32 bytes (f32).
// Both are bound by HBM; a generation step's rows by the launch.
#include "mx.cuh"
#include "mx_host.cuh"

namespace quoka {

constexpr int kMxThreads = 256;

// 8 new elements as floats.
template <typename E>
__device__ __forceinline__ void load8(const E* p, float (&x)[8]) { load_vec<E, 8, true>(p, x); }

// This lane's 8 elements to codes in w (MXFP8: two words, MXFP4: one) with their block's scale byte; x becomes the values the cache holds.
template <int FMT>
__device__ __forceinline__ uint32_t mx_quantise8(float (&x)[8], uint32_t (&w)[2]) {
  uint32_t amax = 0;                                 // (bits of magnitudes order like the magnitudes, NaN above infinity)
#pragma unroll
  for (int i = 0; i < 8; ++i) amax = max(amax, __float_as_uint(x[i]) & 0x7FFFFFFFu);
  amax = max(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, 1));
  amax = max(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, 2));
  const bool finite = amax < 0x7F800000u;
  const int e = mx_scale_exponent<FMT>(amax);
  const float down = __uint_as_float((uint32_t)(127 - e) << 23), up = __uint_as_float((uint32_t)(127 + e) << 23);
  uint32_t c[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)                        // (the product is exact: a value times a power of two)
    c[i] = finite ? mx_encode2<FMT>(x[2 * i] * down, x[2 * i + 1] * down) : 0u;
  if constexpr (FMT == QUOKA_KV_MXFP8) {
    w[0] = c[0] | c[1] << 16;
    w[1] = c[2] | c[3] << 16;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = mx_element<FMT>(w[i / 4] >> (8 * (i % 4)) & 0xFFu) * up;
  } else {
    w[0] = c[0] | c[1] << 8 | c[2] << 16 | c[3] << 24;
    w[1] = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = mx_element<FMT>(w[0] >> (4 * i) & 0xFu) * up;
  }
  if (!finite) x[0] = __uint_as_float(0x7FC00000u);
  return finite ? (uint32_t)(e + 127) : kMxNanScale;
}

template <int FMT>
__device__ __forceinline__ void store_codes(uint8_t* row, int piece, const uint32_t (&w)[2]) {
  if constexpr (FMT == QUOKA_KV_MXFP8) reinterpret_cast<uint2*>(row)[piece] = make_uint2(w[0], w[1]);
  else reinterpret_cast<uint32_t*>(row)[piece] = w[0];
}

template <typename E, int FMT, int D>
__global__ void __launch_bounds__(kMxThreads) append_kv_mx_kernel(DevParams P, const E* __restrict__ k_new, const E* __restrict__ v_new,
                                                                  uint8_t* __restrict__ k_cache, uint8_t* __restrict__ v_cache,
                                                                  uint8_t* __restrict__ k_scale, uint8_t* __restrict__ v_scale,
                                                                  float* __restrict__ k_inv_norm) {
  grid_dependency_wait();
  grid_launch_dependents();
  constexpr int LPR = D / 8;                         // lanes per row: 8 or 16
  const int64_t total = (int64_t)P.batch * P.n_kv * P.chunk * LPR;
  const int lane = threadIdx.x & 31, c = lane % LPR;
  for (int64_t e0 = (int64_t)blockIdx.x * kMxThreads + threadIdx.x - lane; e0 < total; e0 += (int64_t)gridDim.x * kMxThreads) {
    const bool live = e0 + lane < total;             // (whole rows: LPR divides a warp)
    const int64_t row = live ? (e0 + lane) / LPR : 0;
    const int r = (int)(row % P.chunk), h = (int)(row / P.chunk % P.n_kv), s = (int)(row / ((int64_t)P.chunk * P.n_kv));
    float kx[8], vx[8];
    load8(k_new + row * D + c * 8, kx);
    load8(v_new + row * D + c * 8, vx);
    const int t = load_input<true>(P.ctx_len + s) + r;
    uint32_t kw[2], vw[2];
    const uint32_t kb = mx_quantise8<FMT>(kx, kw), vb = mx_quantise8<FMT>(vx, vw);
    float nn = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) nn = fmaf(kx[i], kx[i], nn);
#pragma unroll
    for (int o = LPR / 2; o > 0; o >>= 1) nn += __shfl_xor_sync(0xFFFFFFFFu, nn, o);
    if (!live) continue;
    const int64_t off = kv_row_offset<true>(P, s, h, t) * kMxBits<FMT> / 8;
    store_codes<FMT>(k_cache + off, c, kw);
    store_codes<FMT>(v_cache + off, c, vw);
    const int64_t at = kv_norm_index<true>(P, s, h, t);
    if (c % 4 == 0) {
      k_scale[at * (D / kMxBlock) + c / 4] = (uint8_t)kb;
      v_scale[at * (D / kMxBlock) + c / 4] = (uint8_t)vb;
    }
    if (k_inv_norm != nullptr && c == 0) k_inv_norm[at] = 1.f / fmaxf(sqrtf(nn), kNormEps);
  }
}

// 8 elements of a row (a piece) as the values they stand for.
template <int FMT>
__device__ __forceinline__ void load_values8(const uint8_t* row, int piece, float scale, float (&x)[8]) {
  if constexpr (FMT == QUOKA_KV_MXFP8) {
    const uint2 w = load_input<true>(reinterpret_cast<const uint2*>(row) + piece);
    const uint32_t v[2] = {w.x, w.y};
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = mx_element<FMT>(v[i / 4] >> (8 * (i % 4)) & 0xFFu) * scale;
  } else {
    const uint32_t v = load_input<true>(reinterpret_cast<const uint32_t*>(row) + piece);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = mx_element<FMT>(v >> (4 * i) & 0xFu) * scale;
  }
}
template <typename E>
__device__ __forceinline__ void store8(E* p, const float (&x)[8]) {
  if constexpr (sizeof(E) == 4) {
    reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
  } else {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&b);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

template <typename E, int FMT, int D>
__global__ void __launch_bounds__(kMxThreads) read_kv_mx_kernel(DevParams P, const uint8_t* __restrict__ k_cache,
                                                                const uint8_t* __restrict__ v_cache, int first, int n_rows,
                                                                E* __restrict__ k_out, E* __restrict__ v_out) {
  grid_dependency_wait();
  grid_launch_dependents();
  constexpr int LPR = D / 8;
  const int64_t total = (int64_t)P.batch * P.n_kv * n_rows * LPR;
  for (int64_t e = (int64_t)blockIdx.x * kMxThreads + threadIdx.x; e < total; e += (int64_t)gridDim.x * kMxThreads) {
    const int64_t row = e / LPR;
    const int c = (int)(e % LPR);
    const int r = (int)(row % n_rows), h = (int)(row / n_rows % P.n_kv), s = (int)(row / ((int64_t)n_rows * P.n_kv));
    const int T = load_input<true>(P.ctx_len + s);
    const int64_t t = (int64_t)(first < 0 ? T : first) + r;
    if (t >= (int64_t)T + P.chunk) continue;
    const int64_t off = kv_row_offset<true>(P, s, h, (int)t) * kMxBits<FMT> / 8;
    const int64_t at = mx_scale_index<D, true>(P, s, h, (int)t) + c / 4;
    float x[8], y[8];
    load_values8<FMT>(k_cache + off, c, mx_scale(load_input<true>(P.k_scale + at)), x);
    if (v_cache) load_values8<FMT>(v_cache + off, c, mx_scale(load_input<true>(P.v_scale + at)), y);
    store8(k_out + row * D + c * 8, x);
    if (v_cache) store8(v_out + row * D + c * 8, y);
  }
}

// ---------------------------------------------------------------------------------------------- host
static unsigned mx_blocks(int64_t threads) {
  int64_t blocks = (threads + kMxThreads - 1) / kMxThreads;
  const int64_t most = 16ll * device_sm_count();                     // two waves of eight CTAs per SM; longer ones loop
  if (blocks > most && most > 0) blocks = most;
  return (unsigned)blocks;
}

cudaError_t launch_append_kv_mx(const DevParams& P, int dtype, int fmt, const void* k_new, const void* v_new, void* k_cache, void* v_cache,
                                uint8_t* k_scale, uint8_t* v_scale, float* k_inv_norm, cudaStream_t st) {
  const dim3 grid(mx_blocks((int64_t)P.batch * P.n_kv * P.chunk * (P.d / 8)));
  const cudaError_t e = mx_dispatch(dtype, fmt, P.d, [&](auto elem, auto f, auto d) {
    using E = decltype(elem);
    return launch_kernel("append_kv_mx", append_kv_mx_kernel<E, f.value, d.value>, grid, dim3(kMxThreads), 0, st, 1, true, P, (const E*)k_new,
                         (const E*)v_new, (uint8_t*)k_cache, (uint8_t*)v_cache, k_scale, v_scale, k_inv_norm);
  });
  if (e != cudaSuccess) return e;
  count_launch();
  return cudaGetLastError();
}

cudaError_t launch_read_kv_mx(const DevParams& P, int dtype, int fmt, const void* k_cache, const void* v_cache, int first, int n_rows,
                              void* k_out, void* v_out, cudaStream_t st) {
  const dim3 grid(mx_blocks((int64_t)P.batch * P.n_kv * n_rows * (P.d / 8)));
  const cudaError_t e = mx_dispatch(dtype, fmt, P.d, [&](auto elem, auto f, auto d) {
    using E = decltype(elem);
    return launch_kernel("read_kv_mx", read_kv_mx_kernel<E, f.value, d.value>, grid, dim3(kMxThreads), 0, st, 1, true, P, (const uint8_t*)k_cache,
                         (const uint8_t*)v_cache, first, n_rows, (E*)k_out, (E*)v_out);
  });
  if (e != cudaSuccess) return e;
  count_launch();
  return cudaGetLastError();
}

}  // namespace quoka
