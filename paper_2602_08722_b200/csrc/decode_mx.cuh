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
// The same as bf16 pairs, whatever the scale.
template <int FMT, int N>
__device__ __forceinline__ void bf16_pairs(uint32_t w, uint32_t factor2, uint32_t (&o)[N]) {
  uint32_t x[4];
  mx_bits_bf16x8<FMT>(w, 0u, x);
#pragma unroll
  for (int i = 0; i < N; ++i) o[i] = mul_bf16x2(mul_bf16x2(x[i], FMT == QUOKA_KV_MXFP8 ? 0x7B807B80u : 0x7E807E80u), factor2);
}
__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t bf16x2(float lo, float hi) {
  uint32_t d;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  return d;
}
// 2^diff, -126 <= diff <= 15 (below: 2^-126).
__device__ __forceinline__ float pow2_at_most_15(int diff) { return __uint_as_float((uint32_t)(max(diff, -126) + 127) << 23); }

// ---- What fp16 operands hold, and what is done where they do not.
// A key's row goes into the product divided by its largest block's scale: elements of a block that is kDecKeyWindow powers of two below it
// are fp16 numbers still (multiples of 2^-9 or 2^-1; fp16's are multiples of 2^-24).  A row with a block below that, of elements that are not all
// zero, and a query whose smallest element fp16 does not hold beside its largest one, take bf16 products of the values as they are
// (dec_scores_bf16): exact, as those of a bf16 cache, for three times the instructions.
template <int FMT>
constexpr int kDecKeyWindow = FMT == QUOKA_KV_MXFP8 ? 15 : 23;
template <int FMT>
constexpr uint32_t kMagnitudeBits = FMT == QUOKA_KV_MXFP8 ? 0x7F7F7F7Fu : 0x77777777u;     // of a word of elements
// Columns of a query row, 8 at a time, that go with a lane's pieces of key rows.
template <int FMT, int D>
__device__ __forceinline__ int dec_column(int c, int j) { return FMT == QUOKA_KV_MXFP8 && D == 128 ? 16 * c + 8 * j + (j >= 2 ? 48 : 0) : c * (D / 4) + 8 * j; }
// Magnitudes of a query row's elements, pairs of bf16 bits: the largest, and one less than the smallest but zero (by halves of a word).
struct DecMagnitudes {
  uint32_t most = 0u, low = 0xFFFFFFFFu;
  __device__ __forceinline__ void take(uint32_t x) {
    const uint32_t m = x & 0x7FFF7FFFu;
    most = __vmaxu2(most, m);
    low = __viaddmin_u16x2(m, 0xFFFFFFFFu, low);
  }
  // bits of the largest, as a float's
  __device__ __forceinline__ uint32_t largest() const { return max(most & 0xFFFF0000u, most << 16); }
  // whether the smallest, times 2^up, has its last bit below 2^-24 (a number with exponent field e ends at 2^(max(e, 1) - 134))
  __device__ __forceinline__ bool below_f16(int up) const {
    const int from = 110 - up;
    return from > 1 && (int)min(low & 0xFFFFu, low >> 16) + 1 < (from << 7);
  }
};
// Whether the factors 2^diff of a lane's pieces of keys, fp16 pairs, have one of a block that far below its row's largest.
struct DecFactors {
  uint32_t least = 0xFFFFFFFFu;
  __device__ __forceinline__ void take(uint32_t f) { least = __vminu2(least, f); }
  template <int FMT>
  __device__ __forceinline__ bool below_f16() const { return (least & 0xFFFFu) < (FMT == QUOKA_KV_MXFP8 ? 0x0200u : 0x0002u); }      // 2^-kDecKeyWindow
};
// Whether key row `row` of the tile at `at` (scale word sw) has such a block, not zero.  (A block of zeros has the smallest scale; heads of 80 or 96
// columns padded to 128 have one in every row: sixteen sequences of 20000 rows 130 us, 119 without, 141 by a loop over the blocks.)
template <int FMT, int D>
__device__ __forceinline__ bool dec_key_below_f16(uint32_t at, int row, uint32_t sw) {
  constexpr int kBytes = 4 * kMxBits<FMT>;             // of a block: 16-byte chunks of the swizzle
  uint32_t top = __vmaxu4(sw, sw >> 16);
  top = max(top & 0xFFu, top >> 8 & 0xFFu);
  uint32_t far = top == kMxNanScale ? 0u : __vcmpltu4(sw, (uint32_t)max((int)top - kDecKeyWindow<FMT>, 0) * 0x01010101u) & (D == 128 ? 0xFFFFFFFFu : 0xFFFFu);
  uint32_t any = 0;
  while (far != 0u) {
    const int b = (__ffs((int)far) - 1) / 8;
    far &= ~(0xFFu << (8 * b));
#pragma unroll
    for (int i = 0; i < kBytes; i += 16) {
      uint32_t w[4];
      lds_words<4>(at + DecBytes<FMT, D>::place(row, kBytes * b + i), w);
      any |= w[0] | w[1] | w[2] | w[3];
    }
  }
  return (any & kMagnitudeBits<FMT>) != 0;
}
// Products of 16 keys (rows row0 and row0 + 8 of the tile at `at` are this lane's, with scale words sw) and 8 NT query rows, bf16: sc, and of
// the keys with themselves, where NORM.  load_q(nt, j): the lane's 8 columns of its query row.  A block that is not finite makes its key's NaN.
template <int FMT, int D, int NT, bool NORM, typename LoadQ>
__device__ __forceinline__ void dec_scores_bf16(uint32_t at, int row0, int c, const uint32_t (&sw)[2], LoadQ&& load_q, float (&sc)[NT][4], float (&na)[4],
                                                float (&nb)[4]) {
  typedef DecBytes<FMT, D> B;
  const int blk = FMT == QUOKA_KV_MXFP4 && D == 128 ? c : c >> 1;
#pragma unroll 1                                       // (few instructions: hardly ever taken)
  for (int j = 0; j < D / 32; ++j) {
    const int p = j * kMxBits<FMT> / B::kKBytes, within = j * kMxBits<FMT> % B::kKBytes;
    uint32_t k[2][4];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      uint32_t w[2] = {0u, 0u};
      lds_words<kMxBits<FMT> / 4>(at + B::place(row0 + 8 * i, c * B::kKBytes + 64 * p) + within, w);
      const uint32_t f = mx_scale_bf16x2(sw[i] >> (8 * (blk + 2 * p)) & 0xFFu);
      mx_bits_bf16x8<FMT>(w[0], w[1], k[i]);
#pragma unroll
      for (int e = 0; e < 4; ++e) k[i][e] = mul_bf16x2(mul_bf16x2(k[i][e], FMT == QUOKA_KV_MXFP8 ? 0x7B807B80u : 0x7E807E80u), f);
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const uint4 q = load_q(nt, j);
      mma_bf16(sc[nt], k[0][0], k[1][0], k[0][1], k[1][1], q.x, q.y);
      mma_bf16(sc[nt], k[0][2], k[1][2], k[0][3], k[1][3], q.z, q.w);
    }
    if constexpr (NORM) {
#pragma unroll
      for (int e = 0; e < 4; e += 2) {
        mma_bf16(na, k[0][e], k[1][e], k[0][e + 1], k[1][e + 1], k[0][e], k[0][e + 1]);
        mma_bf16(nb, k[0][e], k[1][e], k[0][e + 1], k[1][e + 1], k[1][e], k[1][e + 1]);
      }
    }
  }
}
// Weight of a result with the reference point m among results whose largest is mx: what has seen nothing weighs nothing.
__device__ __forceinline__ float dec_weight(float m, float mx) { return m == mx ? 1.f : m == -INFINITY ? 0.f : ex2(m - mx); }
constexpr int kDecMaxAbove = 15, kDecHeadroom = 7;       // of a weight's exponent over the reference point, at most and when it is set
constexpr int kDecScaleAbove = 7;                        // of a value block's exponent over O's: 448 * 2^7 is an fp16 number
// Of the largest over the smallest exponent of value blocks that fp16 weights and values are used for.  It keeps the values exact (their
// exponents are 9 below O's at most), and weights that fp16 does not hold, 2^-32 of the largest one and less, from mattering: 2^-23 of the
// output for each of them.
constexpr int kDecValueWindow = 9;

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
