// Rows of a microscaled cache as bf16, for the attention of long chunks: the rows that a (sequence, KV head) attends to, [listed or all cached |
// the chunk's own], written one after the other into scratch, which the bf16 kernels then walk as a cache of that length.
//
// The loaders that convert (attn_mx_loader.cuh) do so for every row block anew, on the issue ports that the softmax needs; a long chunk
// has many.  One pass instead reads a byte or half and writes two per element, and most of what it writes is read from L2.
// Listed rows then are consecutive ones: the copy engine fetches them.
// A value block that is not finite becomes zeros, and the first chunk position that sees it goes to v_nan (one word per tile of rows and
// 32 columns), from where the attention kernel's epilogue makes NaN of what sees it.
//
// Bound by memory: 8 KV heads of 34816 rows of 128 columns, MXFP8, 73 MB in and 143 MB out; the call it belongs to, a chunk of 2048 over 32768
// cached rows, takes 944 to 958 us among other work, where the power cap sets the pace (865 to 890 over a bf16 cache), and 825 by itself on a cool card with L2 emptied
// (converted in the loaders 880; MXFP4 809 / 866).
//
// The rule (kUnpackFrom), query rows per KV head; both ways, us, one call after the other, converted in the loaders / unpacked first, MXFP8:
//   listed 3932 of 32768, d 128:  1024 rows 40.2 / 42.5, 2048 57.5 / 55.4, 4096 85.7 / 79.3, 8192 170 / 147
//   listed 3932 of 20011, d 64:   1024 rows 32.9 / 35.2, 2048 49.1 / 47.2, 3108 80.0 / 71.7
//   all of 20011, d 64:           512 rows 57.4 / 61.6, 1024 82.0 / 81.8, 2048 148 / 137, 3108 233 / 214
//   all of 32768, d 128:          1024 rows 148 / 170, 2048 243 / 262, 4096 490 / 491, 8192 969 / 917
// so 2048, and four times that where all of a cache of 128 columns is unpacked.  Scratch is bounded (kMostUnpacked); calls above it, or with
// a workspace that has no room, convert.
#include "api_host.cuh"
#include "attn_tc.cuh"
#include "attn_tc_pair.cuh"
#include "mx_host.cuh"

namespace quoka {

constexpr int kUnpackThreads = 256, kUnpackRowsPerThread = 4;
template <int D>
constexpr int kUnpackTile = kUnpackRowsPerThread * kUnpackThreads / (D / 8);      // rows of a CTA

template <int FMT, int D>
__global__ void __launch_bounds__(kUnpackThreads) unpack_rows_mx_kernel(DevParams P, const uint8_t* __restrict__ kc, const uint8_t* __restrict__ vc,
                                                                       const int32_t* __restrict__ k_idx, const int32_t* __restrict__ k_cnt, int pitch,
                                                                       uint4* __restrict__ k_out, uint4* __restrict__ v_out, int32_t* __restrict__ v_nan) {
  constexpr int LPR = D / 8, UNR = kUnpackRowsPerThread, RPP = kUnpackThreads / LPR, BLOCKS = D / kMxBlock;
  __shared__ int nan_pos[BLOCKS];
  grid_dependency_wait();                             // the list comes from the kernel before
  const int c = threadIdx.x % LPR, unit = blockIdx.x / P.v_nan_tiles, tile = blockIdx.x % P.v_nan_tiles, r0 = tile * kUnpackTile<D> + threadIdx.x / LPR;
  const int h = unit % P.n_kv, s = unit / P.n_kv, T = __ldg(P.ctx_len + s);
  const int cnt = min(k_idx ? __ldcg(k_cnt + s) : T, pitch - P.chunk), rows = cnt + P.chunk;
  if (tile * kUnpackTile<D> >= rows) return;
  if (threadIdx.x < BLOCKS) nan_pos[threadIdx.x] = kNoNan;
  __syncthreads();
  const int32_t* idx = k_idx && !(P.list_of_selection && cnt == T) ? k_idx + (int64_t)unit * P.budget_cap : nullptr;
  int t[UNR];
#pragma unroll
  for (int j = 0; j < UNR; ++j) {                     // (a row past the end reads the last one; it is not written)
    const int r = min(r0 + j * RPP, rows - 1);
    t[j] = r >= cnt ? T + (r - cnt) : idx ? __ldcg(idx + r) : r;
  }
  uint2 kw[UNR], vw[UNR];
  uint32_t kb[UNR], vb[UNR];
#pragma unroll
  for (int j = 0; j < UNR; ++j) {
    const int64_t off = kv_row_offset(P, s, h, t[j]) * kMxBits<FMT> / 8, at = mx_scale_index<D>(P, s, h, t[j]) + c / 4;
    if constexpr (FMT == QUOKA_KV_MXFP8) {
      kw[j] = __ldg(reinterpret_cast<const uint2*>(kc + off) + c);
      vw[j] = __ldg(reinterpret_cast<const uint2*>(vc + off) + c);
    } else {
      kw[j].x = __ldg(reinterpret_cast<const uint32_t*>(kc + off) + c);
      vw[j].x = __ldg(reinterpret_cast<const uint32_t*>(vc + off) + c);
    }
    kb[j] = __ldg(P.k_scale + at);
    vb[j] = __ldg(P.v_scale + at);
  }
#pragma unroll
  for (int j = 0; j < UNR; ++j) {
    const int r = r0 + j * RPP;
    if (r >= rows) break;
    const int64_t to = ((int64_t)unit * pitch + r) * LPR + c;
    k_out[to] = mx_values_bf16x8<FMT>(kw[j].x, kw[j].y, mx_scale_bf16x2(kb[j]));
    const bool bad = vb[j] == kMxNanScale;
    if (bad && c % 4 == 0) atomicMin(nan_pos + c / 4, max(r - cnt, -1));
    v_out[to] = mx_values_bf16x8<FMT>(vw[j].x, vw[j].y, bad ? 0u : mx_scale_bf16x2(vb[j]));
  }
  __syncthreads();
  if (threadIdx.x < BLOCKS) v_nan[(size_t)blockIdx.x * BLOCKS + threadIdx.x] = nan_pos[threadIdx.x];
}

// ---------------------------------------------------------------------------------------------- host
static size_t pad256(size_t n) { return (n + 255) / 256 * 256; }
static int unpack_tile(const quoka_params* p) { return p->head_dim == 128 ? kUnpackTile<128> : kUnpackTile<64>; }
static int64_t unpack_rows(const quoka_params* p, bool listed) { return (int64_t)(listed ? budget_cap_of(p) : p->max_ctx_len) + p->chunk_len; }
static size_t unpack_side(const quoka_params* p, bool listed) {
  return pad256((size_t)p->batch * p->n_kv_heads * unpack_rows(p, listed) * p->head_dim * 2);
}
static int64_t unpack_tiles(const quoka_params* p, bool listed) { return (unpack_rows(p, listed) + unpack_tile(p) - 1) / unpack_tile(p); }

constexpr int kUnpackFrom = 2048;
constexpr size_t kMostUnpacked = (size_t)256 << 20;
size_t attn_unpack_bytes(const quoka_params* p, bool listed) {
#ifdef QUOKA_DEBUG
  return 0;                                           // the loaders' checks of listed rows and pages mask a bad one; a pass before them could not
#endif
  const int64_t rows = (int64_t)p->chunk_len * (p->n_q_heads / p->n_kv_heads);
  if (p->dtype != QUOKA_BF16 || p->impl == QUOKA_IMPL_SIMT || rows < (listed || p->head_dim == 64 ? 1 : 4) * kUnpackFrom) return 0;
  const size_t bytes = 2 * unpack_side(p, listed) + pad256((size_t)p->batch * p->n_kv_heads * unpack_tiles(p, listed) * (p->head_dim / kMxBlock) * 4);
  return bytes <= kMostUnpacked ? bytes : 0;
}

static AttnKernel pick_unpacked_pair(bool sparse, bool parts, bool in_cluster) { return pick_attn_tc_pair<kUnpacked>(sparse, parts, in_cluster); }

quoka_status launch_attn_mx_unpacked(const quoka_params* p, const DevParams& P0, int fmt, const void* q, const void* k, const void* v, const int32_t* k_idx,
                                     const int32_t* k_cnt, void* out, float* lse, void* scratch, cudaStream_t st, bool after_selection, const AttnPlan& plan) {
  const bool listed = k_idx != nullptr;
  const int rows = (int)unpack_rows(p, listed);
  unsigned char* base = static_cast<unsigned char*>(scratch);
  void *ku = base, *vu = base + unpack_side(p, listed);
  int32_t* v_nan = reinterpret_cast<int32_t*>(base + 2 * unpack_side(p, listed));
  DevParams P = attn_of_plan(P0, plan);
  P.list_of_selection = after_selection ? 1 : 0;
  P.v_nan = v_nan;
  P.v_nan_rows = unpack_tile(p);
  P.v_nan_tiles = (int)unpack_tiles(p, listed);
  const unsigned ctas = (unsigned)((long long)P.batch * P.n_kv * P.v_nan_tiles);
  const cudaError_t e = mx_dispatch(QUOKA_BF16, fmt, P.d, [&](auto, auto f, auto d) {
    return launch_kernel("unpack_rows_mx", unpack_rows_mx_kernel<f.value, d.value>, dim3(ctas), dim3(kUnpackThreads), 0, st, 1, after_selection, P, (const uint8_t*)k,
                         (const uint8_t*)v, k_idx, k_cnt, rows, (uint4*)ku, (uint4*)vu, v_nan);
  });
  if (e != cudaSuccess) return QUOKA_ERR_CUDA;
  count_launch();
  // From here on a bf16 cache of `rows` rows, k_cnt of them listed: all, in order.
  quoka_params pu = *p;
  pu.page_size = 0; pu.max_pages_per_seq = 0; pu.block_table = nullptr;
  pu.kv_rows = rows;
  pu.kv_stride_t = p->head_dim; pu.kv_stride_h = (int64_t)rows * p->head_dim; pu.kv_stride_b = pu.kv_stride_h * p->n_kv_heads;
  P.page_size = 0; P.max_pages = 0; P.block_table = nullptr;
  P.kv_rows = rows;
  P.kv_st = pu.kv_stride_t; P.kv_sh = pu.kv_stride_h; P.kv_sb = pu.kv_stride_b;
  if (listed) { P.ctx_len = k_cnt; P.list_of_selection = 1; }
  CUtensorMap tm_q, tm_k, tm_v;
  if (!encode_q_tensor_map(&tm_q, P, q) || !encode_kv_tensor_map(&tm_k, &pu, ku, 64) || !encode_kv_tensor_map(&tm_v, &pu, vu, 64)) return QUOKA_ERR_CUDA;
  const bool pair = plan.ctas == 2, wide = P.d == 128;
  AttnKernel (*const kernel)(bool, bool, bool) = pair ? pick_unpacked_pair : wide ? pick_attn_tc<128, kUnpacked> : pick_attn_tc<64, kUnpacked>;
  return launch_attn_plan(p, P, plan, kernel, pair ? "attn_tc_pair_unpacked" : "attn_tc_unpacked", pair ? 2 : 1, kAttnThreads,
                          pair ? attn_tc_pair_smem<0>(plan) : wide ? attn_tc_smem<128>() : attn_tc_smem<64>(), tm_q, tm_k, tm_v, ku, vu, k_idx, k_cnt, out, lse, st,
                          /*after_selection=*/false);
}

}  // namespace quoka
