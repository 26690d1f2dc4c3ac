// Pieces of the kernels that take a few query rows per KV head over a microscaled cache (decode_mx.cu, score_few_mx.cu): fp16 operands of
// matrix instructions from raw rows, and the list of granules of 32 keys that the CTAs share.
#pragma once

#include <cuda_fp16.h>

#include "mx_host.cuh"
#include "mx_rows.cuh"
#include "tensor_kernels.cuh"

namespace quoka {

using namespace ptx;

constexpr int kDecGranule = 32;
constexpr int kDecStages = 2;

// A stage of a warp: 32 rows of K, 32 of V, 16-byte chunks swizzled as the copy engine does for rows of 128, 64 or 32 bytes (a lane's
// reads below then meet no bank twice, or K's of 128-byte rows twice).  A lane reads kKPieces pieces of kKBytes of each of four key rows,
// kVBytes of each of eight value rows.
template <int FMT, int D>
struct DecBytes {
  static constexpr int kRow = D * kMxBits<FMT> / 8;
  static constexpr int kKPieces = kRow == 128 ? 2 : 1, kKBytes = kRow / 4 / kKPieces, kVBytes = kRow / 8;
  static constexpr uint32_t kTile = kDecGranule * kRow;
  static constexpr uint32_t kMeta = D == 128 ? 256 : 384;      // of a stage: scale words of the rows' keys, of their values, head_dim 64 also their shifts
  static constexpr uint32_t kStage = 2 * kTile + kMeta;
  // byte `at` of row `row` of a tile
  static __device__ __forceinline__ uint32_t place(int row, int at) {
    return (uint32_t)(row * kRow + (at ^ (kRow == 128 ? (row & 7) << 4 : kRow == 64 ? (row >> 1 & 3) << 4 : (row >> 2 & 1) << 4)));
  }
};

template <int BYTES>
__device__ __forceinline__ void cp_async_n(uint32_t dst, const void* src, bool valid) {
  if constexpr (BYTES == 16) {
    cp_async_16(dst, src, valid);
  } else {
    const uint32_t n = valid ? (uint32_t)BYTES : 0u;
    asm volatile("cp.async.ca.shared.global [%0], [%1], %3, %2;" ::"r"(dst), "l"(src), "r"(n), "n"(BYTES) : "memory");
  }
}
template <int WORDS>
__device__ __forceinline__ void lds_words(uint32_t at, uint32_t* w) {
  if constexpr (WORDS == 4) asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at) : "memory");
  else if constexpr (WORDS == 2) asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(at) : "memory");
  else asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w[0]) : "r"(at) : "memory");
}
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t f16x2(float lo, float hi) {
  uint32_t d;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  return d;
}
__device__ __forceinline__ uint32_t mul_f16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
// A word of elements as fp16 pairs in order: two of MXFP8, four of MXFP4 (a byte has a pair).
template <int FMT, int N>
__device__ __forceinline__ void f16_pairs(uint32_t w, uint32_t factor2, uint32_t (&o)[N]) {
  static_assert(N == (FMT == QUOKA_KV_MXFP8 ? 2 : 4), "pairs of a word");
  if constexpr (FMT == QUOKA_KV_MXFP8) {
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}" : "=r"(o[0]), "=r"(o[1]) : "r"(w));
  } else {
    asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %4;\n\tcvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, c;\n\tcvt.rn.f16x2.e2m1x2 %3, d;\n\t}" : "=r"(o[0]), "=r"(o[1]), "=r"(o[2]), "=r"(o[3]) : "r"(w));
  }
#pragma unroll
  for (int i = 0; i < N; ++i) o[i] = mul_f16x2(o[i], factor2);
}
// 2^diff, diff <= 15, as an fp16 number (zero below its range).
__device__ __forceinline__ float pow2_at_most_15(int diff) { return __uint_as_float((uint32_t)(max(diff, -60) + 127) << 23); }
// Weight of a result with the reference point m among results whose largest is mx: what has seen nothing weighs nothing.
__device__ __forceinline__ float dec_weight(float m, float mx) { return m == mx ? 1.f : m == -INFINITY ? 0.f : ex2(m - mx); }
constexpr int kDecMaxAbove = 15, kDecHeadroom = 7;       // of a weight's exponent over the reference point, at most and when it is set
constexpr int kDecScaleAbove = 7;                        // of a value block's exponent over O's: 448 * 2^7 is an fp16 number

__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}

// The list of granules: unit = (sequence, KV head, row group), in this order.  CTA i has granules [i share, (i + 1) share), share the
// smallest that reaches.
struct DecWork {
  int groups;              // row groups of a KV head
  int own;                 // keys of a sequence behind the cached ones
  const int32_t* k_cnt;    // listed: rows in the list (device), or null
};
// A sequence's lengths: cached keys attended to (listed or all), cached rows.
struct DecLens {
  int cnt, T;
  __device__ __forceinline__ DecLens(const DevParams& P, const DecWork& w, int s) : T(load_input<true>(P.ctx_len + s)) { cnt = w.k_cnt ? __ldcg(w.k_cnt + s) : T; }
  __device__ __forceinline__ DecLens(int cnt_, int T_) : cnt(cnt_), T(T_) {}
  __device__ __forceinline__ int granules(const DecWork& w) const { return (cnt + w.own + kDecGranule - 1) / kDecGranule; }
};
// Granules of the whole list and of the sequences before s (whole warp; one round trip for up to 32 sequences).
struct DecTotals {
  DecLens lane_lens;       // this lane's sequence of the first 32
  long long total, before;
  __device__ __forceinline__ DecTotals(const DevParams& P, const DecWork& w, int s, int lane) : lane_lens(0, 0), total(0), before(0) {
    for (int s0 = 0; s0 < P.batch; s0 += 32) {
      const bool there = s0 + lane < P.batch;
      const DecLens mine = there ? DecLens(P, w, s0 + lane) : DecLens(0, 0);
      if (s0 == 0) lane_lens = mine;
      const int n = there ? mine.granules(w) : 0;
      total += __reduce_add_sync(0xFFFFFFFFu, n);
      before += __reduce_add_sync(0xFFFFFFFFu, s0 + lane < s ? n : 0);
    }
    total *= P.n_kv * w.groups;
    before *= P.n_kv * w.groups;
  }
  __device__ __forceinline__ long long share(int ctas) const {
    return total < 0x7FFFFFFF ? (long long)(((uint32_t)total + (uint32_t)ctas - 1) / (uint32_t)ctas) : (total + ctas - 1) / ctas;
  }
};
__device__ __forceinline__ int dec_div(long long a, long long b) {      // both small, as a rule
  return (a | b) >> 31 == 0 ? (int)((uint32_t)a / (uint32_t)b) : (int)(a / b);
}
// A CTA's share of the list, part of a unit after part of a unit; identical in every warp.
struct DecPart {
  int s, kv, grp;          // unit
  DecLens lens;
  int n;                   // its granules
  int begin, end;          // granules of this part
  long long left;          // granules of the share behind this part
  // the share [lo, hi)
  __device__ __forceinline__ DecPart(const DevParams& P, const DecWork& w, const DecTotals& all, long long lo, long long hi, int lane)
      : lens(all.lane_lens), left(hi - lo) {
    const int heads = P.n_kv * w.groups;
    for (s = 0;; s += 32) {                           // the sequence that lo is in
      const DecLens mine = s == 0 ? all.lane_lens : s + lane < P.batch ? DecLens(P, w, s + lane) : DecLens(0, 0);
      const long long here = s + lane < P.batch ? (long long)mine.granules(w) * heads : 0;
      long long incl = here;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const long long v = __shfl_up_sync(0xFFFFFFFFu, incl, o);
        if (lane >= o) incl += v;
      }
      const uint32_t hit = __ballot_sync(0xFFFFFFFFu, incl > lo);
      if (hit != 0) {
        const int src = __ffs(hit) - 1;
        lo -= __shfl_sync(0xFFFFFFFFu, incl - here, src);
        lens = DecLens(__shfl_sync(0xFFFFFFFFu, mine.cnt, src), __shfl_sync(0xFFFFFFFFu, mine.T, src));
        s += src;
        break;
      }
      lo -= __shfl_sync(0xFFFFFFFFu, incl, 31);
    }
    n = lens.granules(w);
    const int unit = dec_div(lo, n);
    kv = unit / w.groups;
    grp = unit % w.groups;
    begin = (int)(lo - (long long)unit * n);
    cut();
  }
  // one whole unit
  __device__ __forceinline__ DecPart(const DevParams& P, const DecWork& w, int unit)
      : s(unit / (P.n_kv * w.groups)), kv(unit / w.groups % P.n_kv), grp(unit % w.groups), lens(P, w, unit / (P.n_kv * w.groups)), begin(0), left(0) {
    n = end = lens.granules(w);
  }
  __device__ __forceinline__ void cut() {
    end = (int)min((long long)n, begin + left);
    left -= end - begin;
  }
  // false: that was the last
  __device__ __forceinline__ bool next(const DevParams& P, const DecWork& w) {
    if (left <= 0) { begin = end; return false; }
    if (++grp == w.groups) {
      grp = 0;
      if (++kv == P.n_kv) {
        kv = 0;
        lens = DecLens(P, w, ++s);
        n = lens.granules(w);
      }
    }
    begin = 0;
    cut();
    return true;
  }
};

}  // namespace quoka
