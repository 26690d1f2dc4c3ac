// Rows of a microscaled cache as bf16 tiles in shared memory, for the tensor-core kernels.
//
// A tile holds the cache's values times 2^-16: an element's bits at the place of a bf16 exponent and fraction are the value
// divided by 2^120 (2^126 for 4 bits), one multiplication by 2^(104 + e) (2^(110 + e)) applies the block's scale 2^e, and 2^-16 keeps that
// factor a bf16 number for every e that a cache has.  All of it is exact; who uses the tile takes 2^-16 back.
#pragma once

#include <type_traits>

#include "attn_tiles.cuh"
#include "mx.cuh"

namespace quoka {

constexpr int kMxShift = 16;                         // tiles hold values times 2^-kMxShift
constexpr float kMxUnshift = 65536.f;

// 16 elements of a row.
template <int FMT> struct MxUnit;
template <> struct MxUnit<QUOKA_KV_MXFP8> { uint4 w; };
template <> struct MxUnit<QUOKA_KV_MXFP4> { uint2 w; };

// bf16 pair 2^(104 + e) or 2^(110 + e) of a scale byte.
template <int FMT>
__device__ __forceinline__ uint32_t mx_factor2(uint32_t b) { return ((b + (FMT == QUOKA_KV_MXFP8 ? 120u - kMxShift : 126u - kMxShift)) << 7) * 0x10001u; }
constexpr uint32_t kBf16Nan2 = 0x7FC07FC0u;

// The 8 elements of half a unit (two words of MXFP8, one of MXFP4) as four bf16 pairs, in the order in which their bits are reached by
// shifts and masks alone: 0 2 1 3 4 6 5 7, or 0 4 1 5 2 6 3 7 (mx_place).  Queries are put in the same order once per CTA, so that products
// are the same; the columns of O come out in it, and the epilogues take them from there.  Against the plain order, by byte
// permutations, it saves a third of the conversion's instructions on the integer pipe, which the softmax warps need too.
// A word of elements in that order: two pairs of MXFP8, four of MXFP4.
template <int FMT, int N>
__device__ __forceinline__ void mx_to_pairs(uint32_t w, uint32_t factor2, uint32_t (&o)[N]) {
  static_assert(N == (FMT == QUOKA_KV_MXFP8 ? 2 : 4), "pairs of a word");
  if constexpr (FMT == QUOKA_KV_MXFP8) {
    o[0] = (w << 8 & 0x80008000u) | (w << 4 & 0x07F007F0u);
    o[1] = (w & 0x80008000u) | (w >> 4 & 0x07F007F0u);
  } else {
    o[0] = (w << 12 & 0x80008000u) | (w << 6 & 0x01C001C0u);
    o[1] = (w << 8 & 0x80008000u) | (w << 2 & 0x01C001C0u);
    o[2] = (w << 4 & 0x80008000u) | (w >> 2 & 0x01C001C0u);
    o[3] = (w & 0x80008000u) | (w >> 6 & 0x01C001C0u);
  }
#pragma unroll
  for (int i = 0; i < N; ++i) o[i] = mul_bf16x2(o[i], factor2);
}
// PLAIN: in the plain order.
template <int FMT, bool PLAIN = false>
__device__ __forceinline__ uint4 mx_to_bf16x8(uint32_t w0, uint32_t w1, uint32_t factor2) {
  uint32_t o[4];
  if constexpr (PLAIN) {
    mx_bits_bf16x8<FMT>(w0, w1, o);
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = mul_bf16x2(o[i], factor2);
  } else if constexpr (FMT == QUOKA_KV_MXFP8) {
    uint32_t a[2], b[2];
    mx_to_pairs<FMT>(w0, factor2, a);
    mx_to_pairs<FMT>(w1, factor2, b);
    o[0] = a[0]; o[1] = a[1]; o[2] = b[0]; o[3] = b[1];
  } else {
    mx_to_pairs<FMT>(w0, factor2, o);
  }
  return make_uint4(o[0], o[1], o[2], o[3]);
}

// 8 bf16 numbers in plain order, put in that order.
template <int FMT>
__device__ __forceinline__ uint4 mx_order(uint4 w) {
  const uint32_t a = FMT == QUOKA_KV_MXFP8 ? w.y : w.z, b = FMT == QUOKA_KV_MXFP8 ? w.z : w.y;     // what goes with x, and with w
  return make_uint4(__byte_perm(w.x, a, 0x5410), __byte_perm(w.x, a, 0x7632), __byte_perm(b, w.w, 0x5410), __byte_perm(b, w.w, 0x7632));
}
// An item is ROWS cache rows, COLS columns of each: raw in a stage of shared memory, [ROWS][COLS * bits / 8 bytes] and a word of
// scale bytes per row, then bf16 in a tile, [64-column halves][ROWS][128 B] with 16-byte pieces swizzled by row.  What fills stages (the
// copy engine where rows follow one another, else cp.async) and what converts them are different warps: each of the two alone, one
// after the other in the same warps, took longer than a step of the attention kernel.
template <int FMT, int D, int ROWS, int COLS>
struct MxItem {
  static constexpr int U = COLS / 16;                                  // units of 16 elements per row
  static constexpr int RPI = 32 / U;                                   // rows per warp instruction
  static constexpr int kRows = ROWS, kHalves = U / 4;
  static_assert(U == 8 || U == 4, "64 or 128 columns");
  static constexpr int kUnitBytes = 2 * kMxBits<FMT>, kRowBytes = U * kUnitBytes;
  static constexpr uint32_t kRaw = ROWS * kRowBytes, kStage = kRaw + ROWS * 4;     // of a stage
  static constexpr uint32_t kHalf = ROWS * 128;
  typedef decltype(MxUnit<FMT>::w) W;

  // ---- filling, one of NW warps: lane l looks after rows row(0, l), row(1, l) ..
  template <int NW> static constexpr int kMine = (ROWS / NW + 31) / 32;      // (1 or 2)
  template <int NW> static __device__ __forceinline__ int row(int w, int i, int lane) {
    const int p = 32 * i + lane;
    return p < ROWS / NW ? (w + p / RPI * NW) * RPI + p % RPI : ROWS;
  }
  // this lane's copies: its pieces of the warp's rows, whose places (in units from `base`, kNoRow: zeros) the lanes that look after them have
  template <int NW>
  static __device__ __forceinline__ void copy(const W* base, const uint32_t (&place)[kMine<NW>], uint32_t stage, int w, int lane) {
    base += lane % U;
#pragma unroll 2                                     // (as for the conversion: few instructions)
    for (int i = 0; i < ROWS / (RPI * NW); ++i) {
      const int p = i * RPI + lane / U;
      const uint32_t at = __shfl_sync(0xFFFFFFFFu, kMine<NW> == 1 || i * RPI < 32 ? place[0] : place[kMine<NW> - 1], p & 31);
      const uint32_t dst = stage + (uint32_t)((w + i * NW) * RPI * kRowBytes + lane * kUnitBytes);
      const W* src = base + (at == kNoRow ? 0u : at);
      if constexpr (kUnitBytes == 16) {
        cp_async_16(dst, src, at != kNoRow);
      } else {
        const uint32_t n = at != kNoRow ? 8u : 0u;
        asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
      }
    }
  }
  // a row's scale bytes, and their word of the stage
  static __device__ __forceinline__ uint32_t load_scales(const uint8_t* scale, uint32_t srow) {
    return D == 128 ? __ldg(reinterpret_cast<const uint32_t*>(scale) + srow) : __ldg(reinterpret_cast<const uint16_t*>(scale) + srow);
  }
  static __device__ __forceinline__ void put_scales(uint32_t stage, int row, uint32_t word) {
    asm volatile("st.shared.u32 [%0], %1;" ::"r"(stage + kRaw + 4 * row), "r"(word) : "memory");
  }
};

// Converting, one of NW warps: an item of `rows` rows of 64 or 128 columns (halves 1, 2) at row_bytes a row, in half tiles of half_bytes;
// scales: the item's first scale byte of its first row; blocks that are not finite become `nan2`.  A warp instruction takes 64 columns of
// eight rows, of the odd ones the other half: no two lanes of a quarter then meet in a bank, neither reading nor writing.
// A loop, one step ahead with its loads, and the same few instructions for every kind of item: unrolled per kind they had to be
// fetched anew for every item, beside those of the softmax (2048 queries of 32 heads over 16384 rows 610 us, 501 as a loop).
template <int FMT, int NW, bool PLAIN>
__device__ __forceinline__ void mx_convert(uint32_t stage, uint32_t scales, int rows, int halves, int row_bytes, uint32_t nan2, unsigned char* tile,
                                           uint32_t half_bytes, int w, int lane) {
  constexpr int kUnitBytes = 2 * kMxBits<FMT>;
  typename std::remove_const<decltype(MxUnit<FMT>::w)>::type raw;
  uint32_t b;
  const int sub = lane >> 2, u = lane & 3, odd = sub & 1;
  uint32_t src = stage + (uint32_t)((8 * w + sub) * row_bytes + u * kUnitBytes), sc = scales + (uint32_t)(4 * (8 * w + sub) + (u >> 1));
  unsigned char* dst = tile + (uint32_t)(8 * w + sub) * 128u + ((uint32_t)(2 * u ^ sub) << 4);
  const uint32_t second = (sub & 1) ? (uint32_t)-16 : 16u;     // the unit's other piece: 2 u + 1, swizzled
  int steps = rows / (8 * NW) * halves, h = halves == 2 ? odd : 0;
  const auto fetch = [&](int half) {
    asm volatile("ld.shared.u8 %0, [%1];" : "=r"(b) : "r"(sc + 2 * half) : "memory");
    const uint32_t at = src + (uint32_t)(half * 4 * kUnitBytes);
    if constexpr (FMT == QUOKA_KV_MXFP8)
      asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(raw.x), "=r"(raw.y), "=r"(raw.z), "=r"(raw.w) : "r"(at) : "memory");
    else
      asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(raw.x), "=r"(raw.y) : "r"(at) : "memory");
  };
  fetch(h);
#pragma unroll 1
  for (;;) {
    const auto now = raw;
    const uint32_t f = b == kMxNanScale ? nan2 : mx_factor2<FMT>(b);
    unsigned char* to = dst + (h ? half_bytes : 0u);
    // the next step: the other half of these rows, or the next eight rows of this warp
    if (halves == 2) h ^= 1;
    if (halves == 1 || h == odd) {
      src += 8 * NW * (uint32_t)row_bytes;
      sc += 8 * NW * 4;
      dst += 8 * NW * 128;
    }
    if (--steps > 0) fetch(h);
    if constexpr (FMT == QUOKA_KV_MXFP8) {
      *reinterpret_cast<uint4*>(to) = mx_to_bf16x8<FMT, PLAIN>(now.x, now.y, f);
      *reinterpret_cast<uint4*>(to + (int)second) = mx_to_bf16x8<FMT, PLAIN>(now.z, now.w, f);
    } else {
      *reinterpret_cast<uint4*>(to) = mx_to_bf16x8<FMT, PLAIN>(now.x, 0u, f);
      *reinterpret_cast<uint4*>(to + (int)second) = mx_to_bf16x8<FMT, PLAIN>(now.y, 0u, f);
    }
    if (steps <= 0) break;
  }
}

// mbarrier: more bytes to come, without an arrival
__device__ __forceinline__ void mbar_expect_tx(uint64_t* bar, uint32_t bytes) {
  asm volatile("mbarrier.expect_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(bar)), "r"(bytes) : "memory");
}

// Where row t of a (sequence, KV head) is: its place in units of 16 elements from the cache's first, and its index among the rows of
// scales.  (The host refuses caches of 2^32 - 1 units or rows and more.)
struct MxPlaces {
  uint32_t head, st, sb, srow0, page_rows;
  const int32_t* table;
  __device__ __forceinline__ MxPlaces(const DevParams& P) : st((uint32_t)(P.kv_st >> 4)), sb((uint32_t)(P.kv_sb >> 4)), page_rows((uint32_t)(P.n_kv * kPage)) {}
  __device__ __forceinline__ void at_head(const DevParams& P, int s, int kv) {
    head = (uint32_t)(((P.page_size == 0 ? (long long)s * P.kv_sb : 0ll) + (long long)kv * P.kv_sh) >> 4);
    srow0 = P.page_size == 0 ? (uint32_t)(((long long)s * P.n_kv + kv) * P.kv_rows) : (uint32_t)kv * kPage;
    table = P.block_table + (long long)s * P.max_pages;
  }
  // t < 0: kNoRow
  __device__ __forceinline__ void of(const DevParams& P, int t, uint32_t& place, uint32_t& srow) const { int page; of(P, t, place, srow, page); }
  __device__ __forceinline__ void of(const DevParams& P, int t, uint32_t& place, uint32_t& srow, int& page) const {
    page = 0;
    const int tc = max(t, 0);
    uint32_t off = (uint32_t)tc * st;
    srow = srow0 + (uint32_t)tc;
    if (P.page_size != 0) {
      page = __ldg(table + (tc >> 6));
#ifdef QUOKA_DEBUG
      // debug build: a page id outside the pool is recorded and the row treated as absent
      if (page < 0 || (long long)page >= P.kv_rows) {
        if (t >= 0) atomicExch(P.status, (int32_t)QUOKA_ERR_BAD_INDEX);
        t = -1;
        page = 0;
      }
#endif
      off = (uint32_t)page * sb + (uint32_t)(tc & (kPage - 1)) * st;
      srow = (uint32_t)page * page_rows + srow0 + (uint32_t)(tc & (kPage - 1));
    }
    place = t < 0 ? kNoRow : head + off;
  }
};

}  // namespace quoka
