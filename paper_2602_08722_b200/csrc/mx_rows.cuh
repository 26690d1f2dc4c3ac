// Rows of a microscaled cache as bf16 tiles in shared memory, for the tensor-core kernels.
//
// A tile holds the cache's values times 2^-16: an element's bits at the place of a bf16 exponent and fraction are the value
// divided by 2^120 (2^126 for 4 bits), one multiplication by 2^(104 + e) (2^(110 + e)) applies the block's scale 2^e, and 2^-16 keeps that
// factor a bf16 number for every e that a cache has.  All of it is exact; who uses the tile takes 2^-16 back.
#pragma once

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

__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
// The 8 elements of half a unit (two words of MXFP8, one of MXFP4) as four bf16 pairs, in the order in which their bits are reached by
// shifts and masks alone: 0 2 1 3 4 6 5 7, or 0 4 1 5 2 6 3 7 (mx_place).  Queries are put in the same order once per CTA, so that products
// are the same; the columns of O come out in it, and the epilogues take them from there.  Against the plain order, by byte
// permutations, it saves a third of the conversion's instructions on the integer pipe, which the softmax warps need too.
// PLAIN: in the plain order.
template <int FMT, bool PLAIN = false>
__device__ __forceinline__ uint4 mx_to_bf16x8(uint32_t w0, uint32_t w1, uint32_t factor2) {
  uint32_t o[4];
  if constexpr (PLAIN) {
    if constexpr (FMT == QUOKA_KV_MXFP8) {
      o[0] = __byte_perm(w0, w0, 0x1100); o[1] = __byte_perm(w0, w0, 0x3322);
      o[2] = __byte_perm(w1, w1, 0x1100); o[3] = __byte_perm(w1, w1, 0x3322);
    } else {
      const uint32_t lo = w0 << 4;
      o[0] = __byte_perm(lo, w0, 0x4400); o[1] = __byte_perm(lo, w0, 0x5511);
      o[2] = __byte_perm(lo, w0, 0x6622); o[3] = __byte_perm(lo, w0, 0x7733);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)                        // (what stands below an element's bits is masked off)
      o[i] = (o[i] & 0x80008000u) | (FMT == QUOKA_KV_MXFP8 ? o[i] >> 4 & 0x07F007F0u : o[i] >> 6 & 0x01C001C0u);
  } else if constexpr (FMT == QUOKA_KV_MXFP8) {
    o[0] = (w0 << 8 & 0x80008000u) | (w0 << 4 & 0x07F007F0u);
    o[1] = (w0 & 0x80008000u) | (w0 >> 4 & 0x07F007F0u);
    o[2] = (w1 << 8 & 0x80008000u) | (w1 << 4 & 0x07F007F0u);
    o[3] = (w1 & 0x80008000u) | (w1 >> 4 & 0x07F007F0u);
  } else {
    o[0] = (w0 << 12 & 0x80008000u) | (w0 << 6 & 0x01C001C0u);
    o[1] = (w0 << 8 & 0x80008000u) | (w0 << 2 & 0x01C001C0u);
    o[2] = (w0 << 4 & 0x80008000u) | (w0 >> 2 & 0x01C001C0u);
    o[3] = (w0 & 0x80008000u) | (w0 >> 6 & 0x01C001C0u);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = mul_bf16x2(o[i], factor2);
  return make_uint4(o[0], o[1], o[2], o[3]);
}

// One of NLW warps that bring items of cache rows into shared memory as bf16: of the ROWS tile rows from row0 on, or 128, the columns from
// col0 on.  An item is [64-column halves][rows][128 B], 16-byte pieces swizzled by row.
// The raw elements come in with cp.async, some items ahead of their conversion, into stages whose every piece is read by the
// lane that copied it (8 or 16 bytes: a unit of 16 elements); a row's scale bytes by the lane that looks after the row.
template <int FMT, int D, int ROWS, int COLS, int NLW, bool PLAIN>
struct MxItem {
  static constexpr int U = COLS / 16;                                  // units per row
  static constexpr int RPI = 32 / U;                                   // rows per warp instruction
  static constexpr int GROUPS = ROWS / (RPI * NLW);                    // row groups of this warp
  static constexpr int kRows = GROUPS * RPI;                           // its rows, a lane each
  static constexpr int kUnitBytes = 2 * kMxBits<FMT>;
  static constexpr uint32_t kRaw = GROUPS * 32 * kUnitBytes;           // of a stage: this warp's units
  static constexpr uint32_t kHalf = ROWS * 128;
  static_assert(kRows <= 32 && GROUPS >= 1 && GROUPS * RPI * NLW == ROWS, "a lane per row");
  typedef decltype(MxUnit<FMT>::w) W;

  // this lane's row of the item
  static __device__ __forceinline__ int row(int lw, int lane) { return (lw + lane / RPI * NLW) * RPI + lane % RPI; }

  // The copies of one item: `place` is this lane's row in units of 16 elements from `base` (kNoRow: zeros), `srow` its index among the
  // rows of scales; raw: shared memory of this warp's units; meta: 32 scale words, head_dim 64 also 32 shifts.
  static __device__ __forceinline__ void copy(const W* base, uint32_t place, const uint8_t* scale, uint32_t srow, uint32_t raw, uint32_t meta, int lane) {
    if (place != kNoRow)                              // (head_dim 64: the word that has the scales of two rows)
      cp_async_4(meta + 4 * lane, scale + (D == 128 ? (size_t)srow * 4 : (size_t)(srow >> 1) * 4));
    else
      asm volatile("st.shared.u32 [%0], %1;" ::"r"(meta + 4 * lane), "r"(0u) : "memory");
    if (D == 64) asm volatile("st.shared.u32 [%0], %1;" ::"r"(meta + 128 + 4 * lane), "r"((srow & 1u) * 16) : "memory");
    base += lane % U;
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) {
      const uint32_t at = __shfl_sync(0xFFFFFFFFu, place, i * RPI + lane / U), dst = raw + (uint32_t)(i * 32 + lane) * kUnitBytes;
      const W* src = base + (at == kNoRow ? 0u : at);
      if constexpr (kUnitBytes == 16) {
        cp_async_16(dst, src, at != kNoRow);
      } else {
        const uint32_t n = at != kNoRow ? 8u : 0u;
        asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
      }
    }
  }
  // the scale bytes of this lane's row, landed
  static __device__ __forceinline__ uint32_t scales(uint32_t meta, int lane) {
    uint32_t w;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w) : "r"(meta + 4 * lane) : "memory");
    if (D == 64) {
      uint32_t shift;
      asm volatile("ld.shared.u32 %0, [%1];" : "=r"(shift) : "r"(meta + 128 + 4 * lane) : "memory");
      w = w >> shift & 0xFFFFu;
    }
    return w;
  }
  // The item as bf16; `mine`: scales(), block0: the item's first block of a row; blocks that are not finite become `nan2`.
  static __device__ __forceinline__ void convert(uint32_t raw_at, uint32_t mine, int block0, uint32_t nan2, unsigned char* item, int lw, int lane) {
    const int u = lane % U, rsub = lane / U;
    const int sw = U == 8 ? u >> 2 : 0;               // lanes of the second half store their second piece first: other banks
    W raw[GROUPS];
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) {
      const uint32_t at = raw_at + (uint32_t)(i * 32 + lane) * kUnitBytes;
      if constexpr (FMT == QUOKA_KV_MXFP8)
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(raw[i].x), "=r"(raw[i].y), "=r"(raw[i].z), "=r"(raw[i].w) : "r"(at) : "memory");
      else
        asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(raw[i].x), "=r"(raw[i].y) : "r"(at) : "memory");
    }
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) {
      const uint32_t b = __shfl_sync(0xFFFFFFFFu, mine, i * RPI + rsub) >> (8 * (block0 + (u >> 1))) & 0xFFu;
      const uint32_t f = b == kMxNanScale ? nan2 : mx_factor2<FMT>(b);
      const int r = (lw + i * NLW) * RPI + rsub;
      unsigned char* dst = item + (uint32_t)(u >> 2) * kHalf + (uint32_t)r * 128u;
      const uint32_t p0 = (uint32_t)(((2 * (u & 3) + sw) ^ r) & 7) << 4;
      uint4 first, second;
      if constexpr (FMT == QUOKA_KV_MXFP8) {
        first = mx_to_bf16x8<FMT, PLAIN>(sw ? raw[i].z : raw[i].x, sw ? raw[i].w : raw[i].y, f);
        second = mx_to_bf16x8<FMT, PLAIN>(sw ? raw[i].x : raw[i].z, sw ? raw[i].y : raw[i].w, f);
      } else {
        first = mx_to_bf16x8<FMT, PLAIN>(sw ? raw[i].y : raw[i].x, 0u, f);
        second = mx_to_bf16x8<FMT, PLAIN>(sw ? raw[i].x : raw[i].y, 0u, f);
      }
      *reinterpret_cast<uint4*>(dst + p0) = first;
      *reinterpret_cast<uint4*>(dst + (p0 ^ 16u)) = second;
    }
  }
};

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
  __device__ __forceinline__ void of(const DevParams& P, int t, uint32_t& place, uint32_t& srow) const {
    const int tc = max(t, 0);
    uint32_t off = (uint32_t)tc * st;
    srow = srow0 + (uint32_t)tc;
    if (P.page_size != 0) {
      int page = __ldg(table + (tc >> 6));
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
