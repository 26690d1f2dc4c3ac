// Writing the microscaled cache and reading it back.
//
// append: the chunk's K and V, dense [b][n_KV][C][D], go to cache rows T_s + r as blocks of 32 elements and a scale byte each.
//   A lane holds 8 elements of K and the same 8 of V, four lanes a block: its largest magnitude in two shuffles, the elements by
//   the conversion instruction.  The inverse norm of a key row is that of the values the cache then holds.
// read: cache rows first .. first + n - 1 to dense [b][n_KV][n][D] tensors; rows at and beyond T_s + C are left as they were.
//   A lane turns 8 elements of K and of V into 16 (bf16) or 32 bytes (f32).
// Both are bound by HBM (4 sequences of 20011 to 32768 rows, MXFP4 to bf16: 95 us among other work, 5.9 TB/s of 0.57 GB; one call after the other 90); a
// generation step's rows by the launch.
#include <cuda_fp16.h>

#include "mx.cuh"
#include "mx_host.cuh"

namespace quoka {

constexpr int kMxThreads = 256;

// 8 new elements: floats, or bf16 pairs, which stay pairs as long as they can (append of 8 times 4096 rows, 8 heads, d 128: 34.7 us, as floats
// 36.5, MXFP4 36.7 / 39.8).
template <typename E> struct MxNew;
template <> struct MxNew<float> {
  float x[8];
  __device__ __forceinline__ void load(const float* p) { load_vec<float, 8, true>(p, x); }
  // bits of the largest magnitude (they order like the magnitudes, NaN above infinity)
  __device__ __forceinline__ uint32_t largest() const {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(x[i]) & 0x7FFFFFFFu);
    return m;
  }
  // a pair times 2^-e: exact
  __device__ __forceinline__ float2 pair(int i, int e) const {
    const float down = __uint_as_float((uint32_t)(127 - e) << 23);
    return make_float2(x[2 * i] * down, x[2 * i + 1] * down);
  }
};
template <> struct MxNew<__nv_bfloat16> {
  uint4 w;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { w = load_input<true>(reinterpret_cast<const uint4*>(p)); }
  __device__ __forceinline__ uint32_t word(int i) const { return i == 0 ? w.x : i == 1 ? w.y : i == 2 ? w.z : w.w; }
  __device__ __forceinline__ uint32_t largest() const {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) m = __vmaxu2(m, word(i) & 0x7FFF7FFFu);
    return max(m & 0xFFFF0000u, m << 16);
  }
  // exact but for what becomes zero whatever is left of it
  __device__ __forceinline__ float2 pair(int i, int e) const {
    const uint32_t y = mul_bf16x2(word(i), ((uint32_t)(127 - e) << 7) * 0x10001u);
    return make_float2(__uint_as_float(y << 16), __uint_as_float(y & 0xFFFF0000u));
  }
};

// A pair of elements as numbers.
template <int FMT>
__device__ __forceinline__ float2 mx_decode2(uint32_t c) {
  uint32_t h;
  if constexpr (FMT == QUOKA_KV_MXFP8) asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)c));
  else asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, a;\n\t}" : "=r"(h) : "r"(c));
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}

// This lane's 8 elements to codes in w (MXFP8: two words, MXFP4: one) with their block's scale byte; `square`: the sum of the squares of the values
// the cache then holds (NaN where it holds NaN), where it is asked for.
template <int FMT, typename E>
__device__ __forceinline__ uint32_t mx_quantise8(const MxNew<E>& x, uint32_t (&w)[2], bool want_square, float& square) {
  uint32_t amax = x.largest();
  amax = max(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, 1));
  amax = max(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, 2));
  const bool finite = amax < 0x7F800000u;
  const int e = mx_scale_exponent<FMT>(amax);
  uint32_t c[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 y = x.pair(i, e);
    c[i] = finite ? mx_encode2<FMT>(y.x, y.y) : 0u;
  }
  if constexpr (FMT == QUOKA_KV_MXFP8) {
    w[0] = c[0] | c[1] << 16;
    w[1] = c[2] | c[3] << 16;
  } else {
    w[0] = c[0] | c[1] << 8 | c[2] << 16 | c[3] << 24;
    w[1] = 0;
  }
  if (want_square) {                                 // (squares of elements are exact in fp32, and so is their product with 2^(2 e) above 2^-126)
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 v = mx_decode2<FMT>(c[i]);
      sum = fmaf(v.x, v.x, sum);
      sum = fmaf(v.y, v.y, sum);
    }
    const float up = __uint_as_float((uint32_t)(127 + e) << 23);
    square = finite ? sum * up * up : __uint_as_float(0x7FC00000u);
  }
  return finite ? (uint32_t)(e + 127) : kMxNanScale;
}

template <int FMT>
__device__ __forceinline__ void store_codes(uint8_t* row, int piece, const uint32_t (&w)[2]) {
  if constexpr (FMT == QUOKA_KV_MXFP8) reinterpret_cast<uint2*>(row)[piece] = make_uint2(w[0], w[1]);
  else reinterpret_cast<uint32_t*>(row)[piece] = w[0];
}

// A CTA takes UNR * 256 / LPR rows of a (sequence, KV head), a thread the same piece of UNR of them, all loads before their first use.
template <typename E, int FMT, int D, int UNR>
__global__ void __launch_bounds__(kMxThreads) append_kv_mx_kernel(DevParams P, const E* __restrict__ k_new, const E* __restrict__ v_new,
                                                                  uint8_t* __restrict__ k_cache, uint8_t* __restrict__ v_cache,
                                                                  uint8_t* __restrict__ k_scale, uint8_t* __restrict__ v_scale,
                                                                  float* __restrict__ k_inv_norm, int tiles) {
  grid_dependency_wait();
  grid_launch_dependents();
  constexpr int LPR = D / 8, RPP = kMxThreads / LPR;  // lanes per row (8 or 16), rows per pass
  const int c = threadIdx.x % LPR, unit = blockIdx.x / tiles, r0 = blockIdx.x % tiles * (UNR * RPP) + threadIdx.x / LPR;
  const int h = unit % P.n_kv, s = unit / P.n_kv;
  const int64_t first = (int64_t)unit * P.chunk;
  const int T = load_input<true>(P.ctx_len + s);
  MxNew<E> kx[UNR], vx[UNR];
#pragma unroll
  for (int j = 0; j < UNR; ++j) {                     // (a row past the chunk reads the last one; it is not written)
    const int64_t row = first + min(r0 + j * RPP, P.chunk - 1);
    kx[j].load(k_new + row * D + c * 8);
    vx[j].load(v_new + row * D + c * 8);
  }
#pragma unroll
  for (int j = 0; j < UNR; ++j) {
    const int r = r0 + j * RPP, t = T + r;
    uint32_t kw[2], vw[2];
    float nn = 0.f, unused;
    const uint32_t kb = mx_quantise8<FMT>(kx[j], kw, k_inv_norm != nullptr, nn), vb = mx_quantise8<FMT>(vx[j], vw, false, unused);
    if (k_inv_norm != nullptr) {
#pragma unroll
      for (int o = LPR / 2; o > 0; o >>= 1) nn += __shfl_xor_sync(0xFFFFFFFFu, nn, o);
    }
    if (r >= P.chunk) continue;
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

// 8 elements of a row (a piece), and the values they stand for.
template <int FMT>
__device__ __forceinline__ uint2 load_piece(const uint8_t* row, int piece) {
  if constexpr (FMT == QUOKA_KV_MXFP8) return load_input<true>(reinterpret_cast<const uint2*>(row) + piece);
  else return make_uint2(load_input<true>(reinterpret_cast<const uint32_t*>(row) + piece), 0u);
}
template <int FMT>
__device__ __forceinline__ void piece_values(uint2 w, float scale, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t code = FMT == QUOKA_KV_MXFP8 ? (i < 4 ? w.x : w.y) >> (8 * (i % 4)) & 0xFFu : w.x >> (4 * i) & 0xFu;
    x[i] = mx_element<FMT>(code) * scale;
  }
}
template <typename E, int FMT>
__device__ __forceinline__ void store_values(E* p, const uint2& w, uint32_t scale) {
  if constexpr (sizeof(E) == 4) {
    float x[8];
    piece_values<FMT>(w, mx_scale(scale), x);
    reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
  } else {
    uint4 v = mx_values_bf16x8<FMT>(w.x, w.y, mx_scale_bf16x2(scale));
    if constexpr (FMT == QUOKA_KV_MXFP8) {
      if (e4m3_has_nan(w.x) || e4m3_has_nan(w.y)) {     // (a cache that other code wrote)
        const auto pair = [](uint32_t x, uint32_t codes) {
          return ((codes & 0x7Fu) == kE4m3Nan ? 0x7FC0u : x & 0xFFFFu) | ((codes >> 8 & 0x7Fu) == kE4m3Nan ? 0x7FC00000u : x & 0xFFFF0000u);
        };
        v = make_uint4(pair(v.x, w.x), pair(v.y, w.x >> 16), pair(v.z, w.y), pair(v.w, w.y >> 16));
      }
    }
    *reinterpret_cast<uint4*>(p) = v;
  }
}

template <typename E, int FMT, int D, int UNR>
__global__ void __launch_bounds__(kMxThreads) read_kv_mx_kernel(DevParams P, const uint8_t* __restrict__ k_cache,
                                                                const uint8_t* __restrict__ v_cache, int first, int n_rows,
                                                                E* __restrict__ k_out, E* __restrict__ v_out, int tiles) {
  grid_dependency_wait();
  grid_launch_dependents();
  constexpr int LPR = D / 8, RPP = kMxThreads / LPR;
  const int c = threadIdx.x % LPR, unit = blockIdx.x / tiles, r0 = blockIdx.x % tiles * (UNR * RPP) + threadIdx.x / LPR;
  const int h = unit % P.n_kv, s = unit / P.n_kv;
  const int T = load_input<true>(P.ctx_len + s);
  const int64_t t0 = first < 0 ? T : first;
  const int64_t rows = min((int64_t)n_rows, (int64_t)T + P.chunk - t0);      // that there are
  if (r0 >= rows) return;
  uint2 kw[UNR], vw[UNR];
  uint8_t kb[UNR], vb[UNR];
#pragma unroll
  for (int j = 0; j < UNR; ++j) {                     // (a row past them reads the last one; it is not written)
    const int t = (int)(t0 + min((int64_t)r0 + j * RPP, rows - 1));
    const int64_t off = kv_row_offset<true>(P, s, h, t) * kMxBits<FMT> / 8;
    const int64_t at = mx_scale_index<D, true>(P, s, h, t) + c / 4;
    kw[j] = load_piece<FMT>(k_cache + off, c);
    kb[j] = load_input<true>(P.k_scale + at);
    if (v_cache) { vw[j] = load_piece<FMT>(v_cache + off, c); vb[j] = load_input<true>(P.v_scale + at); }
  }
#pragma unroll
  for (int j = 0; j < UNR; ++j) {
    if (r0 + j * RPP >= rows) break;
    const int64_t to = ((int64_t)unit * n_rows + r0 + j * RPP) * D + c * 8;
    store_values<E, FMT>(k_out + to, kw[j], kb[j]);
    if (v_cache) store_values<E, FMT>(v_out + to, vw[j], vb[j]);
  }
}

// ---------------------------------------------------------------------------------------------- host
// Rows per thread: four where the CTAs then still make two waves, else one.  One / four, us, 8 KV heads, d 128, MXFP8: append of 8 times 4096 rows 39.3 / 34.7,
// 16 of one row 7.2 / 7.4, read of 8192 rows 12.6 / 7.8, of 2000 rows 5.9 / 6.1, of 4 sequences of 20011 to 32768 rows 162 / 104 (MXFP4 161 / 90).
struct MxGrid { int unr, tiles; int64_t ctas; };
static MxGrid mx_grid(const DevParams& P, int64_t rows) {
  const int64_t units = (int64_t)P.batch * P.n_kv;
  const auto of = [&](int unr) {
    const int per = unr * kMxThreads / (P.d / 8);
    const int64_t tiles = (rows + per - 1) / per;
    return MxGrid{unr, (int)tiles, tiles * units};
  };
  const MxGrid four = of(4);
  return four.ctas >= 2ll * device_sm_count() ? four : of(1);
}

cudaError_t launch_append_kv_mx(const DevParams& P, int dtype, int fmt, const void* k_new, const void* v_new, void* k_cache, void* v_cache,
                                uint8_t* k_scale, uint8_t* v_scale, float* k_inv_norm, cudaStream_t st) {
  const MxGrid g = mx_grid(P, P.chunk);
  if (g.ctas > 0x7FFFFFFFll) return cudaErrorInvalidConfiguration;
  const cudaError_t e = mx_dispatch(dtype, fmt, P.d, [&](auto elem, auto f, auto d) {
    using E = decltype(elem);
    return launch_kernel("append_kv_mx", g.unr == 4 ? append_kv_mx_kernel<E, f.value, d.value, 4> : append_kv_mx_kernel<E, f.value, d.value, 1>, dim3((unsigned)g.ctas),
                         dim3(kMxThreads), 0, st, 1, true, P, (const E*)k_new, (const E*)v_new, (uint8_t*)k_cache, (uint8_t*)v_cache, k_scale, v_scale, k_inv_norm, g.tiles);
  });
  if (e != cudaSuccess) return e;
  count_launch();
  return cudaGetLastError();
}

cudaError_t launch_read_kv_mx(const DevParams& P, int dtype, int fmt, const void* k_cache, const void* v_cache, int first, int n_rows,
                              void* k_out, void* v_out, cudaStream_t st) {
  const MxGrid g = mx_grid(P, n_rows);
  if (g.ctas > 0x7FFFFFFFll) return cudaErrorInvalidConfiguration;
  const cudaError_t e = mx_dispatch(dtype, fmt, P.d, [&](auto elem, auto f, auto d) {
    using E = decltype(elem);
    return launch_kernel("read_kv_mx", g.unr == 4 ? read_kv_mx_kernel<E, f.value, d.value, 4> : read_kv_mx_kernel<E, f.value, d.value, 1>, dim3((unsigned)g.ctas),
                         dim3(kMxThreads), 0, st, 1, true, P, (const uint8_t*)k_cache, (const uint8_t*)v_cache, first, n_rows, (E*)k_out, (E*)v_out, g.tiles);
  });
  if (e != cudaSuccess) return e;
  count_launch();
  return cudaGetLastError();
}

}  // namespace quoka
