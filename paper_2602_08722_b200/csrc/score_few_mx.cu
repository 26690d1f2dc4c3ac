// Key scoring over a microscaled cache against eight retained queries or fewer (a generation step has one): every key is read once for
// a few products, so HBM bounds it, and next to it the instructions that make operands of 8 or 4 bits.  As in decode_mx.cu the keys are the M
// side of fp16 matrix instructions, a warp takes 32 of them at a time from a ring of its own that the copy engine fills, and the granules of
// all (sequence, KV head) make one list that the CTAs share equally.
// The squared norm of a key is the diagonal of K K^T, whose second operand is the first one's registers: two more matrix
// instructions for 16 columns where multiplying and adding up the elements would be a hundred others.
#include <algorithm>

#include "decode_mx.cuh"

namespace quoka {

constexpr int kFewWarps = 16, kFewStages = 3;

template <int FMT, int D>
constexpr uint32_t kFewMeta = (D == 128 ? 256 : 384);      // scale words of 32 rows, inverse norms, head_dim 64 also shifts

template <int FMT, int D, bool OWN_NORM>
__global__ void __launch_bounds__(32 * kFewWarps, 1)
score_few_mx_kernel(DevParams P, DecWork work, const __nv_bfloat16* __restrict__ qbar, const uint8_t* __restrict__ kc, float* __restrict__ scores,
                    const __grid_constant__ CUtensorMap tm_k) {
  typedef DecBytes<FMT, D> B;
  constexpr int WARPS = kFewWarps, ST = kFewStages, KSTEPS = D / 16, KW = B::kKBytes * B::kKPieces / 4;
  extern __shared__ unsigned char few_smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(few_smem_raw) + 1023) & ~(uintptr_t)1023);
  __shared__ int abort_flag;
  grid_launch_dependents();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
  const uint32_t ring = smem_u32(smem) + (uint32_t)warp * (ST * B::kTile);
  const uint32_t metas = smem_u32(smem) + (uint32_t)(WARPS * ST) * B::kTile + (uint32_t)warp * (ST * kFewMeta<FMT, D>);
  uint64_t* landed = reinterpret_cast<uint64_t*>(smem + WARPS * ST * (B::kTile + kFewMeta<FMT, D>)) + warp * ST;
  const WaitCtx wc{&abort_flag, P.status};
  if (threadIdx.x == 0) abort_flag = 0;
  if (lane == 0) {
    for (int i = 0; i < ST; ++i) mbar_init(&landed[i], 1);
    fence_mbar_init();
  }
  __syncthreads();
  // ---- this CTA's share
  const DecTotals all(P, work, 0, lane);
  const long long each = all.share(gridDim.x), lo = min(each * blockIdx.x, all.total), hi = min(lo + each, all.total);
  if (lo == hi) { grid_dependency_wait(); return; }   // (no link of a chain ends without having waited)
  DecPart in(P, work, all, lo, hi, lane);
  DecPart part = in;
  const bool cached = P.k_inv_norm != nullptr && !P.score_dot;
  MxPlaces places(P);
  int pos = in.begin + warp;
  bool more = true;
  const auto fill = [&](int stage) {
    while (more && pos >= in.end) {                   // (the warps take granules of the share in turn, across its parts)
      const int past = pos - in.end;
      more = in.next(P, work);
      pos = in.begin + past;
    }
    if (more) {
      const int first = pos * kDecGranule, t = first + lane < in.lens.cnt ? first + lane : -1;
      uint32_t place, srow;
      int page;
      places.at_head(P, in.s, in.kv);
      places.of(P, t, place, srow, page);
      const uint32_t at = ring + (uint32_t)stage * B::kTile, meta = metas + (uint32_t)stage * kFewMeta<FMT, D> + 4 * lane;
      if (t >= 0) {
        cp_async_4(meta, P.k_scale + (D == 128 ? (size_t)srow * 4 : (size_t)(srow >> 1) * 4));
        if (cached) cp_async_4(meta + 128, P.k_inv_norm + srow);
      } else {
        asm volatile("st.shared.u32 [%0], %1;" ::"r"(meta), "r"(0u) : "memory");
      }
      if (D == 64) asm volatile("st.shared.u32 [%0], %1;" ::"r"(meta + 256), "r"((srow & 1u) * 16) : "memory");
      if (first + kDecGranule <= in.lens.cnt) {
        if (lane == 0) {
          fence_proxy_async_smem();                   // earlier contents of the stage were read, or written, through the generic proxy
          mbar_arrive_expect_tx(&landed[stage], B::kTile);
          tma_load_4d(smem + ((size_t)warp * ST + stage) * B::kTile, &tm_k, &landed[stage], 0, P.page_size != 0 ? first & (kPage - 1) : first, in.kv,
                      P.page_size != 0 ? page : in.s);
        }
      } else {                                        // the last rows of a sequence, zeros behind them
#pragma unroll 1
        for (int i = 0; i < 4 * B::kKPieces; ++i) {
          const int row = g + 8 * (i / B::kKPieces), piece = c * B::kKBytes + 64 * (i % B::kKPieces);
          const uint32_t from = __shfl_sync(0xFFFFFFFFu, place, row);
          cp_async_n<B::kKBytes>(at + B::place(row, piece), kc + (size_t)(from == kNoRow ? 0u : from) * (2 * kMxBits<FMT>) + piece, from != kNoRow);
        }
        if (lane == 0) mbar_arrive(&landed[stage]);
      }
      pos += WARPS;
    }
    cp_async_commit();
  };
#pragma unroll
  for (int i = 0; i < ST; ++i) fill(i);
  grid_dependency_wait();                             // Q-bar comes from the kernel before
  uint32_t qf[2 * KSTEPS];
  float qs[2] = {0.f, 0.f};
  bool wide_q = false;                                // a query has elements that fp16 does not hold beside its largest one
  int stage = 0, s_cur = -1, kv_cur = -1, gr = part.begin + warp;
  uint32_t phase = 0;
  bool ok = true;
  for (bool again = true; again && ok;) {
    if (gr >= part.end) {
      const int past = gr - part.end;
      again = part.next(P, work);
      gr = part.begin + past;
      continue;
    }
    if (part.s != s_cur || part.kv != kv_cur) {       // queries past the retained ones are zeros
      s_cur = part.s; kv_cur = part.kv;
      const __nv_bfloat16* qr = qbar + (((long long)part.s * P.n_kv + part.kv) * P.n_sel + min(g, P.n_sel - 1)) * D;
      uint4 w[D / 32];
      DecMagnitudes mags;
#pragma unroll
      for (int j = 0; j < D / 32; ++j) {
        w[j] = __ldcg(reinterpret_cast<const uint4*>(qr + dec_column<FMT, D>(c, j)));
        if (g >= P.n_sel) w[j] = make_uint4(0, 0, 0, 0);
        const uint32_t x[4] = {w[j].x, w[j].y, w[j].z, w[j].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) mags.take(x[i]);
      }
      uint32_t top = mags.largest();
      top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
      top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
      const int up = min(14 + 127 - (int)(top >> 23), 120);
      wide_q = __any_sync(0xFFFFFFFFu, mags.below_f16(up));
      const float f = __uint_as_float((uint32_t)(127 + up) << 23), back = __uint_as_float((uint32_t)(127 - up) << 23);
#pragma unroll
      for (int j = 0; j < D / 32; ++j) {
        const uint32_t x[4] = {w[j].x, w[j].y, w[j].z, w[j].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) qf[4 * j + i] = f16x2(__uint_as_float(x[i] << 16) * f, __uint_as_float(x[i] & 0xFFFF0000u) * f);
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) qs[e] = __shfl_sync(0xFFFFFFFFu, back, 4 * (2 * c + e));
    }
    float* out = scores + ((long long)part.s * P.n_kv + part.kv) * P.max_ctx;
#pragma unroll 1
    for (; gr < part.end; gr += WARPS) {
      cp_async_wait<ST - 1>();
      if (!mbar_wait_done(&landed[stage], phase, wc)) { ok = false; break; }
      __syncwarp();
      const uint32_t at = ring + (uint32_t)stage * B::kTile, meta = metas + (uint32_t)stage * kFewMeta<FMT, D>;
      const auto row_scales = [&](int row) {
        uint32_t sw;
        asm volatile("ld.shared.u32 %0, [%1];" : "=r"(sw) : "r"(meta + 4 * row) : "memory");
        if (D == 64) {
          uint32_t shift;
          asm volatile("ld.shared.u32 %0, [%1];" : "=r"(shift) : "r"(meta + 256 + 4 * row) : "memory");
          sw = sw >> shift & 0xFFFFu;
        }
        return sw;
      };
      // Scores of 16 keys from their products with queries 2 c and 2 c + 1 (rows g, g + 8), and with themselves.
      const auto write = [&](int h, const float (&sc)[4], const float (&na)[4], const float (&nb)[4], const float (&key)[2], const float (&inv)[2],
                             const bool (&bad)[2]) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float s0 = sc[2 * i], s1 = sc[2 * i + 1];
          float v;
          if (P.agg_mean) {                             // (queries past the retained ones score zero)
            v = s0 + s1;
            v += __shfl_xor_sync(0xFFFFFFFFu, v, 1);
            v += __shfl_xor_sync(0xFFFFFFFFu, v, 2);
            v /= (float)P.n_sel;
          } else {
            v = fmaxf(2 * c < P.n_sel ? s0 : -INFINITY, 2 * c + 1 < P.n_sel ? s1 : -INFINITY);
            v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, 1));
            v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, 2));
          }
          // the key's diagonal element is in the lane with c = g / 2, which writes
          if constexpr (OWN_NORM) {
            const float nn = i == 0 ? (g & 1 ? na[1] : na[0]) : (g & 1 ? nb[3] : nb[2]);
            v = v * key[i] / fmaxf(sqrtf(nn) * key[i], kNormEps);
          } else {
            v = v * key[i] * inv[i];
          }
          if (bad[i] && !P.agg_mean) v = -INFINITY;
          const int t = gr * kDecGranule + 16 * h + 8 * i + g;
          if (c == g >> 1 && t < part.lens.cnt) out[t] = v;
        }
      };
      const auto norms_kept = [&](int row) {
        float inv = 1.f;
        if (cached) asm volatile("ld.shared.f32 %0, [%1];" : "=f"(inv) : "r"(meta + 128 + 4 * row) : "memory");
        return inv;
      };
      DecFactors factors;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float sc[4] = {0.f, 0.f, 0.f, 0.f}, na[4] = {0.f, 0.f, 0.f, 0.f}, nb[4] = {0.f, 0.f, 0.f, 0.f};
        uint32_t w[2][KW], f[2][B::kKPieces];
        bool bad[2];
        float key[2], inv[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int row = g + 16 * h + 8 * i;
#pragma unroll
          for (int p = 0; p < B::kKPieces; ++p) lds_words<B::kKBytes / 4>(at + B::place(row, c * B::kKBytes + 64 * p), w[i] + p * (B::kKBytes / 4));
          const uint32_t sw = row_scales(row);
          inv[i] = norms_kept(row);
          uint32_t top = __vmaxu4(sw, sw >> 16);       // the largest of the row's scale bytes
          top = max(top & 0xFFu, top >> 8 & 0xFFu);
          bad[i] = top == kMxNanScale;
          key[i] = mx_scale(top);
          const int blk = FMT == QUOKA_KV_MXFP4 && D == 128 ? c : c >> 1;
#pragma unroll
          for (int p = 0; p < B::kKPieces; ++p) {
            const float x = pow2_at_most_15((int)(sw >> (8 * (blk + 2 * p)) & 0xFFu) - (int)top);
            f[i][p] = f16x2(x, x);
            factors.take(f[i][p]);
          }
        }
#pragma unroll
        for (int j = 0; j < KW; ++j) {
          constexpr int N = FMT == QUOKA_KV_MXFP8 ? 2 : 4;
          uint32_t a[N], b[N];
          f16_pairs<FMT>(w[0][j], f[0][j / (KW / B::kKPieces)], a);
          f16_pairs<FMT>(w[1][j], f[1][j / (KW / B::kKPieces)], b);
#pragma unroll
          for (int i = 0; i < N / 2; ++i) {
            mma_f16(sc, a[2 * i], b[2 * i], a[2 * i + 1], b[2 * i + 1], qf[N * j + 2 * i], qf[N * j + 2 * i + 1]);
            if constexpr (OWN_NORM) {                  // keys 0-7 of the 16 against all, and 8-15
              mma_f16(na, a[2 * i], b[2 * i], a[2 * i + 1], b[2 * i + 1], a[2 * i], a[2 * i + 1]);
              mma_f16(nb, a[2 * i], b[2 * i], a[2 * i + 1], b[2 * i + 1], b[2 * i], b[2 * i + 1]);
            }
          }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) sc[e] *= qs[e & 1];
        write(h, sc, na, nb, key, inv, bad);
      }
      // Where fp16 operands do not hold the granule: anew, of the values themselves, over what was written.
      const bool below = factors.below_f16<FMT>();
      if (__builtin_expect(__any_sync(0xFFFFFFFFu, below || wide_q), 0)) {
        if (wide_q || __any_sync(0xFFFFFFFFu, dec_key_below_f16<FMT, D>(at, lane, row_scales(lane)))) {
#pragma unroll 1
          for (int h = 0; h < 2; ++h) {
            float sc[1][4] = {{0.f, 0.f, 0.f, 0.f}}, na[4] = {0.f, 0.f, 0.f, 0.f}, nb[4] = {0.f, 0.f, 0.f, 0.f};
            uint32_t sw[2];
            bool bad[2];
            float key[2] = {1.f, 1.f}, inv[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              sw[i] = row_scales(g + 16 * h + 8 * i);
              inv[i] = norms_kept(g + 16 * h + 8 * i);
              bad[i] = __vcmpeq4(sw[i], 0xFFFFFFFFu) != 0u;
            }
            dec_scores_bf16<FMT, D, 1, OWN_NORM>(at, g + 16 * h, c, sw, [&](int, int j) {
              if (g >= P.n_sel) return make_uint4(0, 0, 0, 0);
              return __ldcg(reinterpret_cast<const uint4*>(qbar + (((long long)part.s * P.n_kv + part.kv) * P.n_sel + g) * D + dec_column<FMT, D>(c, j)));
            }, sc, na, nb);
            write(h, sc[0], na, nb, key, inv, bad);
          }
        }
      }
      __syncwarp();                                    // the scale words of this stage have been read
      fill(stage);
      if (++stage == ST) { stage = 0; phase ^= 1; }
    }
  }
  cp_async_wait_all();                                 // nothing of this thread is in flight at exit
}

// ---------------------------------------------------------------------------------------------- host
// The tensor-core kernel takes the same for one query as for 16, 22.5 us over 32768 keys of 8 KV heads; this one 18.5 for one as for eight, the columns of a
// matrix instruction.  16 sequences of 8192 to 32768 rows, one query, cached norms: 84 among other work (4.6 TB/s of MXFP8), one call after the other 80; over a
// bf16 cache 120; the tensor-core kernel 165.  Looking for granules that fp16 does not hold takes 2 of the 80.
bool score_few_mx_applies(const quoka_params* p) { return std::min(p->n_retain, p->chunk_len) <= 8; }

cudaError_t launch_score_few_mx(const DevParams& P, int fmt, const void* qbar, const void* k, float* scores, cudaStream_t st, bool chained) {
  const int sms = device_sm_count();
  if (sms <= 0) return cudaErrorInvalidDevice;
  const long long granules = (long long)P.batch * P.n_kv * ((P.max_ctx + kDecGranule - 1) / kDecGranule);
  const long long ctas = std::min<long long>(sms, granules);
  const DecWork work{1, 0, nullptr};
  const cudaError_t e = mx_dispatch(QUOKA_BF16, fmt, P.d, [&](auto, auto f, auto d) {
    constexpr int FMT = decltype(f)::value, D = decltype(d)::value;
    CUtensorMap tm_k;
    if (!encode_mx_tile_map(&tm_k, P, FMT, k, kDecGranule)) return cudaErrorInvalidValue;
    const size_t smem = 1024 + (size_t)kFewWarps * kFewStages * (DecBytes<FMT, D>::kTile + kFewMeta<FMT, D> + 8);
    const auto kernel = P.k_inv_norm == nullptr && !P.score_dot ? score_few_mx_kernel<FMT, D, true> : score_few_mx_kernel<FMT, D, false>;
    const cudaError_t err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (err != cudaSuccess) return err;
    return launch_kernel("score_few_mx", kernel, dim3((unsigned)ctas), dim3(32 * kFewWarps), smem, st, 1, chained, P, work, (const __nv_bfloat16*)qbar, (const uint8_t*)k,
                         scores, tm_k);
  });
  if (e != cudaSuccess) return e;
  count_launch();
  return cudaGetLastError();
}

}  // namespace quoka
