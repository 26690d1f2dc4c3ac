// Loader warps of the tensor-core attention kernels over a microscaled cache: rows of 8- or 4-bit elements come in through
// registers, become bf16 there and go to the ring's shared-memory tiles in the layout the operand descriptors expect; the rest
// of those kernels does not know the difference.
//
// A tile holds the cache's values times 2^-16: an element's bits at the place of a bf16 exponent and fraction are the value
// divided by 2^120 (2^126 for 4 bits), one multiplication by 2^(104 + e) (2^(110 + e)) applies the block's scale 2^e, and 2^-16 keeps that
// factor a bf16 number for every e that a cache has.  The softmax scale and the division by the row sum take it back.
// All of it is exact.
//
// Values that are not finite (scale byte 255): a key's block becomes NaN, its column of S with it, and rows that do not see the
// column set it to minus infinity.  A value's block becomes zeros, as its products with weights of zero would reach rows that do not see
// it; the first chunk position that sees one is kept per block of columns, and the epilogue makes NaN of what is at or behind it.
//
// What bounds it: instructions, about four a pair of elements; copies run two or three
// items ahead of the conversion.
#pragma once

#include <type_traits>

#include "attn_tiles.cuh"
#include "mx.cuh"

namespace quoka {

// 512 threads: the roles of the bf16 kernels in the first 12 warps but for the loaders, which are the last four, one on each
// sub-partition's issue port.  A thread may then have 128 registers; the softmax warps take 168 and the others give them.
constexpr int kMxAttnThreads = 512, kMxLoaderWarps = 4, kMxFirstLoader = 12;
constexpr int kMxSoftmaxRegs = 168, kMxOtherRegs = 88;
static_assert(256 * kMxSoftmaxRegs + 256 * kMxOtherRegs == kMxAttnThreads * 128, "what the block is launched with");

constexpr int kMxShift = 16;                         // tiles hold values times 2^-kMxShift
constexpr float kMxUnshift = 65536.f;
constexpr int kNoNan = 0x7FFFFFFF;

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
template <int FMT>
__device__ __forceinline__ uint4 mx_to_bf16x8(uint32_t w0, uint32_t w1, uint32_t factor2) {
  uint32_t o[4];
  if constexpr (FMT == QUOKA_KV_MXFP8) {
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
// 8 bf16 numbers in plain order, put in that order.
template <int FMT>
__device__ __forceinline__ uint4 mx_order(uint4 w) {
  const uint32_t a = FMT == QUOKA_KV_MXFP8 ? w.y : w.z, b = FMT == QUOKA_KV_MXFP8 ? w.z : w.y;     // what goes with x, and with w
  return make_uint4(__byte_perm(w.x, a, 0x5410), __byte_perm(w.x, a, 0x7632), __byte_perm(b, w.w, 0x5410), __byte_perm(b, w.w, 0x7632));
}
// The CTA's Q tiles in that order, in place: by the loader warps, behind their first copies; `ready` gets an arrival of each warp.
template <int FMT>
__device__ __forceinline__ bool mx_order_q(unsigned char* q_smem, int bytes, int thread, int threads, uint64_t* q_full, uint64_t* ready, const WaitCtx& wc) {
  if (!mbar_wait(q_full, 0, wc)) return false;
  uint4* q = reinterpret_cast<uint4*>(q_smem);
#pragma unroll 4
  for (int i = thread; i < bytes / 16; i += threads) q[i] = mx_order<FMT>(q[i]);
  fence_proxy_async_smem();
  __syncwarp();
  if ((thread & 31) == 0) mbar_arrive(ready);
  return true;
}

// One loader warp of NLW.  A K item of the ring is ROWS_K tile rows from row k_row0 on, all D columns; a V item all 128 rows, VC columns
// from v_col0 on.  Both are [64-column halves][rows][128 B], 16-byte pieces swizzled by row.
// The raw elements come in with cp.async, NST items ahead of their conversion, into stages whose every piece is read by the
// lane that copied it (8 or 16 bytes: a unit of 16 elements); a row's scale bytes by the lane that looks after the row.
template <int FMT, int D, int ROWS_K, int VC, bool SPARSE, int NLW, int SLOTS, int NST>
struct MxLoader {
  static constexpr int KU = D / 16, VU = VC / 16;                      // units per row
  static constexpr int K_RPI = 32 / KU, V_RPI = 32 / VU;               // rows per warp instruction
  static constexpr int K_GROUPS = ROWS_K / (K_RPI * NLW), V_GROUPS = 128 / (V_RPI * NLW);     // row groups of this warp
  static constexpr int K_ROWS = K_GROUPS * K_RPI, V_ROWS = V_GROUPS * V_RPI;                  // rows of this warp, a lane each
  static constexpr int kUnitBytes = 2 * kMxBits<FMT>;
  static constexpr int kGroups = K_GROUPS > V_GROUPS ? K_GROUPS : V_GROUPS;
  static constexpr uint32_t kWarpRaw = kGroups * 32 * kUnitBytes;      // a stage: this warp's units, 32 scale words, their shifts
  static constexpr uint32_t kWarpStage = kWarpRaw + (D == 128 ? 128 : 256);
  static constexpr uint32_t kStageBytes = NST * NLW * kWarpStage;      // shared memory of all of them
  static_assert(K_ROWS <= 32 && V_ROWS <= 32 && K_GROUPS >= 1 && V_GROUPS >= 1, "a lane per row");
  typedef decltype(MxUnit<FMT>::w) W;
  // One of the two streams of items: the tile that is copied next, and the number of this lane's row in it (if it has one; looked
  // at only when the copies are issued, an item later than it is asked for)
  struct Stream { int tile, n; };

  const DevParams& P;
  int s, kv, lw, lane, k_row0, v_col0, T;
  uint32_t head, st, sb, srow0, stage0;              // stage0: shared-memory address of this warp's first stage
  const int32_t *table, *idx;
  const W *kc, *vc;
  int* v_nan;

  __device__ __forceinline__ MxLoader(const DevParams& P_, int s_, int kv_, int lw_, int lane_, int k_row0_, int v_col0_, int T_, const void* k,
                                      const void* v, const int32_t* k_idx, int* v_nan_, unsigned char* stages)
      : P(P_), s(s_), kv(kv_), lw(lw_), lane(lane_), k_row0(k_row0_), v_col0(v_col0_), T(T_), v_nan(v_nan_) {
    // (the host refuses caches of 2^32 - 1 units or rows and more)
    st = (uint32_t)(P.kv_st >> 4);
    sb = (uint32_t)(P.kv_sb >> 4);
    head = (uint32_t)(((P.page_size == 0 ? (long long)s * P.kv_sb : 0ll) + (long long)kv * P.kv_sh) >> 4);
    srow0 = P.page_size == 0 ? (uint32_t)(((long long)s * P.n_kv + kv) * P.kv_rows) : (uint32_t)kv * kPage;
    table = P.block_table + (long long)s * P.max_pages;
    idx = SPARSE ? k_idx + ((long long)s * P.n_kv + kv) * P.budget_cap : nullptr;
    kc = static_cast<const W*>(k);
    vc = static_cast<const W*>(v);
    stage0 = smem_u32(stages) + (uint32_t)lw * (NST * kWarpStage);
  }

  // this lane's row in a tile (of K: in the whole tile, not the item)
  template <bool V> __device__ __forceinline__ int tile_row() const {
    constexpr int RPI = V ? V_RPI : K_RPI;
    return (V ? 0 : k_row0) + (lw + lane / RPI * NLW) * RPI + lane % RPI;
  }
  // its number in the cache; of a listed one a load
  template <bool V> __device__ __forceinline__ int number(const AttnGeom& g, int tile) const {
    const TileRows tr = tile_rows<SPARSE>(g, tile);
    const int rr = tile_row<V>();
    if (SPARSE && tr.from_list) return __ldcg(idx + tr.first + max(min(rr, min(tr.count, kKeyTile) - 1), 0));    // written by the kernel before: L2
    return tr.first + rr;
  }
  // whether there is such a row
  template <bool V> __device__ __forceinline__ bool exists(const AttnGeom& g, int tile) const {
    return lane < (V ? V_ROWS : K_ROWS) && tile_row<V>() < min(tile_rows<SPARSE>(g, tile).count, kKeyTile);
  }
  // The copies of the next item of a stream into a stage, one group (empty past the known tiles); then the next row number.
  template <bool V> __device__ __forceinline__ void copy(const AttnGeom& g, Stream& next, int stage) const {
    constexpr int GROUPS = V ? V_GROUPS : K_GROUPS, RPI = V ? V_RPI : K_RPI, U = V ? VU : KU;
    if (next.tile < g.n_known) {
      int t = exists<V>(g, next.tile) ? next.n : -1;
#ifdef QUOKA_DEBUG
      if (SPARSE && tile_rows<SPARSE>(g, next.tile).from_list && (t < -1 || t >= T)) { atomicExch(P.status, (int32_t)QUOKA_ERR_BAD_INDEX); t = -1; }
#endif
      const int tc = max(t, 0);
      uint32_t off = (uint32_t)tc * st, srow = srow0 + (uint32_t)tc;
      if (P.page_size != 0) {
        int page = __ldg(table + (tc >> 6));
#ifdef QUOKA_DEBUG
        if (page < 0 || (long long)page >= P.kv_rows) {
          if (t >= 0) atomicExch(P.status, (int32_t)QUOKA_ERR_BAD_INDEX);
          t = -1;
          page = 0;
        }
#endif
        off = (uint32_t)page * sb + (uint32_t)(tc & (kPage - 1)) * st;
        srow = (uint32_t)page * (uint32_t)(P.n_kv * kPage) + srow0 + (uint32_t)(tc & (kPage - 1));
      }
      const uint32_t dst = stage0 + (uint32_t)stage * kWarpStage;
      const uint8_t* sc = (V ? P.v_scale : P.k_scale);
      if (t >= 0) {
        // (head_dim 64: the word that has the scales of two rows)
        cp_async_4(dst + kWarpRaw + 4 * lane, sc + (D == 128 ? (size_t)srow * 4 : (size_t)(srow >> 1) * 4));
      } else {
        asm volatile("st.shared.u32 [%0], %1;" ::"r"(dst + kWarpRaw + 4 * lane), "r"(0u) : "memory");
      }
      if (D == 64) asm volatile("st.shared.u32 [%0], %1;" ::"r"(dst + kWarpRaw + 128 + 4 * lane), "r"((srow & 1u) * 16) : "memory");
      const uint32_t place = t < 0 ? kNoRow : head + off;
      const W* base = (V ? vc : kc) + (V ? (uint32_t)v_col0 >> 4 : 0u) + lane % U;
#pragma unroll
      for (int i = 0; i < GROUPS; ++i) {
        const uint32_t at = __shfl_sync(0xFFFFFFFFu, place, i * RPI + lane / U);
        cp_async_unit(dst + (uint32_t)(i * 32 + lane) * kUnitBytes, base + (at == kNoRow ? 0u : at), at != kNoRow);
      }
      ++next.tile;
      if (next.tile < g.n_known) next.n = number<V>(g, next.tile);
    }
    cp_async_commit();
  }
  static __device__ __forceinline__ void cp_async_unit(uint32_t dst, const W* src, bool valid) {
    if constexpr (kUnitBytes == 16) {
      cp_async_16(dst, src, valid);
    } else {
      const uint32_t n = valid ? 8u : 0u;
      asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
    }
  }
  // A stage's item as bf16 into the ring; for V, the first position that sees a value that is not finite, per 32 columns.
  template <bool V> __device__ __forceinline__ void convert(const AttnGeom& g, int tile, int stage, unsigned char* item) const {
    constexpr int GROUPS = V ? V_GROUPS : K_GROUPS, RPI = V ? V_RPI : K_RPI, U = V ? VU : KU;
    constexpr uint32_t kHalf = (V ? 128 : ROWS_K) * 128;
    const uint32_t src = stage0 + (uint32_t)stage * kWarpStage;
    const int u = lane % U, rsub = lane / U;
    const int sw = U == 8 ? u >> 2 : 0;               // lanes of the second half store their second piece first: other banks
    uint32_t mine;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(mine) : "r"(src + kWarpRaw + 4 * lane) : "memory");
    if (D == 64) {
      uint32_t shift;
      asm volatile("ld.shared.u32 %0, [%1];" : "=r"(shift) : "r"(src + kWarpRaw + 128 + 4 * lane) : "memory");
      mine = mine >> shift & 0xFFFFu;
    }
    if (V && lane < V_ROWS && __vcmpeq4(mine, 0xFFFFFFFFu) != 0) {
      const TileRows tr = tile_rows<SPARSE>(g, tile);
#pragma unroll
      for (int b = 0; b < D / kMxBlock; ++b)
        if ((mine >> (8 * b) & 0xFFu) == kMxNanScale) atomicMin(v_nan + b, tr.causal ? max(tr.col0 + tile_row<true>(), -1) : -1);
    }
    W raw[GROUPS];
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) {
      const uint32_t at = src + (uint32_t)(i * 32 + lane) * kUnitBytes;
      if constexpr (FMT == QUOKA_KV_MXFP8)
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(raw[i].x), "=r"(raw[i].y), "=r"(raw[i].z), "=r"(raw[i].w) : "r"(at) : "memory");
      else
        asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(raw[i].x), "=r"(raw[i].y) : "r"(at) : "memory");
    }
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) {
      const uint32_t word = __shfl_sync(0xFFFFFFFFu, mine, i * RPI + rsub);
      const uint32_t b = word >> (8 * ((V ? v_col0 / kMxBlock : 0) + (u >> 1))) & 0xFFu;
      const uint32_t f = b == kMxNanScale ? (V ? 0u : kBf16Nan2) : mx_factor2<FMT>(b);
      const int row = (lw + i * NLW) * RPI + rsub;
      unsigned char* dst = item + (uint32_t)(u >> 2) * kHalf + (uint32_t)row * 128u;
      const uint32_t p0 = (uint32_t)(((2 * (u & 3) + sw) ^ row) & 7) << 4;
      uint4 first, second;
      if constexpr (FMT == QUOKA_KV_MXFP8) {
        first = mx_to_bf16x8<FMT>(sw ? raw[i].z : raw[i].x, sw ? raw[i].w : raw[i].y, f);
        second = mx_to_bf16x8<FMT>(sw ? raw[i].x : raw[i].z, sw ? raw[i].y : raw[i].w, f);
      } else {
        first = mx_to_bf16x8<FMT>(sw ? raw[i].y : raw[i].x, 0u, f);
        second = mx_to_bf16x8<FMT>(sw ? raw[i].x : raw[i].y, 0u, f);
      }
      *reinterpret_cast<uint4*>(dst + p0) = first;
      *reinterpret_cast<uint4*>(dst + (p0 ^ 16u)) = second;
    }
  }

  // All tiles of this CTA's walk (until a wait gives up).
  template <typename Learn, typename Begun>
  __device__ __forceinline__ void run(AttnGeom& g, int t_lo, unsigned char* ring, uint32_t slot_bytes, uint64_t* full, uint64_t* empty,
                                      const WaitCtx& wc, Learn&& learn, Begun&& begun) {
    bool first = true;
    int tile = t_lo, slot = 0, stage = 0;
    uint32_t phase = 0;
    Stream k{t_lo, -1}, v{t_lo, -1};
    const auto one = [&](auto is_v) -> bool {         // the next item: conversion, and copies into the stage it leaves
      constexpr bool V = decltype(is_v)::value;
      cp_async_wait<NST - 1>();
      __syncwarp();
      if (!mbar_wait_done(&empty[slot], phase ^ 1, wc)) return false;
      convert<V>(g, tile, stage, ring + (size_t)slot * slot_bytes);
      fence_proxy_async_smem();                       // these stores, before products read the slot
      __syncwarp();
      if (lane == 0) mbar_arrive(&full[slot]);
      if (++slot == SLOTS) { slot = 0; phase ^= 1; }
      if constexpr (NST % 2 == 0) copy<V>(g, V ? v : k, stage);
      else copy<!V>(g, V ? k : v, stage);
      if (++stage == NST) stage = 0;
      return true;
    };
    for (;;) {
      if (tile == g.n_known) {                        // end of what is known: the list length, or the end
        if (!g.resolved) learn();
        if (tile == g.n_known) {
          if (first) begun();                         // (a part without tiles)
          break;
        }
      }
      k.tile = v.tile = tile;                         // (all copies have been converted)
      k.n = number<false>(g, tile);
      v.n = number<true>(g, tile);
#pragma unroll
      for (int i = 0; i < NST; ++i) {
        const int at = stage + i < NST ? stage + i : stage + i - NST;
        if (i % 2 == 0) copy<false>(g, k, at); else copy<true>(g, v, at);
      }
      if (first && !begun()) break;
      first = false;
      for (; tile < g.n_known; ++tile)
        if (!one(std::false_type{}) || !one(std::true_type{})) goto out;
    }
  out:
    cp_async_wait_all();                              // nothing of this thread is in flight at exit
  }
};

}  // namespace quoka
