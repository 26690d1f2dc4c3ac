// Loader warps of the tensor-core attention kernels over a microscaled cache: rows of 8- or 4-bit elements come in through
// registers, become bf16 there and go to the ring's shared-memory tiles in the layout the operand descriptors expect; the rest
// of those kernels does not know the difference.
//
// The conversion is in mx_rows.cuh.  Tiles hold the cache's values times 2^-16; the softmax scale and the division by the row sum take
// that back.
//
// Values that are not finite (scale byte 255): a key's block becomes NaN, its column of S with it, and rows that do not see the
// column set it to minus infinity.  A value's block becomes zeros, as its products with weights of zero would reach rows that do not see
// it; the first chunk position that sees one is kept per block of columns, and the epilogue makes NaN of what is at or behind it.
//
// What bounds it: instructions, about four a pair of elements; copies run two or three
// items ahead of the conversion.
#pragma once

#include <type_traits>

#include "mx_rows.cuh"

namespace quoka {

// 512 threads: the roles of the bf16 kernels in the first 12 warps but for the loaders, which are the last four, one on each
// sub-partition's issue port.  A thread may then have 128 registers; the softmax warps take 168 and the others give them.
constexpr int kMxAttnThreads = 512, kMxLoaderWarps = 4, kMxFirstLoader = 12;
constexpr int kMxSoftmaxRegs = 168, kMxOtherRegs = 88;
static_assert(256 * kMxSoftmaxRegs + 256 * kMxOtherRegs == kMxAttnThreads * 128, "what the block is launched with");

constexpr int kNoNan = 0x7FFFFFFF;

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
// from v_col0 on.  NST items are on their way or landed and not converted yet.
template <int FMT, int D, int ROWS_K, int VC, bool SPARSE, int NLW, int SLOTS, int NST>
struct MxLoader {
  typedef MxItem<FMT, D, ROWS_K, D, NLW, false> K;
  typedef MxItem<FMT, D, 128, VC, NLW, false> V;
  typedef typename K::W W;
  static constexpr uint32_t kWarpRaw = K::kRaw > V::kRaw ? K::kRaw : V::kRaw;
  static constexpr uint32_t kWarpStage = kWarpRaw + (D == 128 ? 128 : 256);
  static constexpr uint32_t kStageBytes = NST * NLW * kWarpStage;      // shared memory of all stages
  // One of the two streams of items: the tile that is copied next, and the number of this lane's row in it (if it has one; looked
  // at only when the copies are issued, an item later than it is asked for)
  struct Stream { int tile, n; };

  const DevParams& P;
  int lw, lane, k_row0, v_col0, T;
  uint32_t stage0;                                   // shared-memory address of this warp's first stage
  MxPlaces places;
  const int32_t* idx;
  const W *kc, *vc;
  int* v_nan;

  __device__ __forceinline__ MxLoader(const DevParams& P_, int s, int kv, int lw_, int lane_, int k_row0_, int v_col0_, int T_, const void* k,
                                      const void* v, const int32_t* k_idx, int* v_nan_, unsigned char* stages)
      : P(P_), lw(lw_), lane(lane_), k_row0(k_row0_), v_col0(v_col0_), T(T_), places(P_), v_nan(v_nan_) {
    places.at_head(P, s, kv);
    idx = SPARSE ? k_idx + ((long long)s * P.n_kv + kv) * P.budget_cap : nullptr;
    kc = static_cast<const W*>(k);
    vc = static_cast<const W*>(v);
    stage0 = smem_u32(stages) + (uint32_t)lw * (NST * kWarpStage);
  }

  // this lane's row in a tile (of K: in the whole tile, not the item)
  template <bool IS_V> __device__ __forceinline__ int tile_row() const { return IS_V ? V::row(lw, lane) : k_row0 + K::row(lw, lane); }
  // its number in the cache; of a listed one a load
  template <bool IS_V> __device__ __forceinline__ int number(const AttnGeom& g, int tile) const {
    const TileRows tr = tile_rows<SPARSE>(g, tile);
    const int rr = tile_row<IS_V>();
    if (SPARSE && tr.from_list) return __ldcg(idx + tr.first + max(min(rr, min(tr.count, kKeyTile) - 1), 0));    // written by the kernel before: L2
    return tr.first + rr;
  }
  // whether there is such a row
  template <bool IS_V> __device__ __forceinline__ bool exists(const AttnGeom& g, int tile) const {
    return lane < (IS_V ? V::kRows : K::kRows) && tile_row<IS_V>() < min(tile_rows<SPARSE>(g, tile).count, kKeyTile);
  }
  // The copies of the next item of a stream into a stage, one group (empty past the known tiles); then the next row number.
  template <bool IS_V> __device__ __forceinline__ void copy(const AttnGeom& g, Stream& next, int stage) const {
    if (next.tile < g.n_known) {
      int t = exists<IS_V>(g, next.tile) ? next.n : -1;
#ifdef QUOKA_DEBUG
      if (SPARSE && tile_rows<SPARSE>(g, next.tile).from_list && (t < -1 || t >= T)) { atomicExch(P.status, (int32_t)QUOKA_ERR_BAD_INDEX); t = -1; }
#endif
      uint32_t place, srow;
      places.of(P, t, place, srow);
      const uint32_t raw = stage0 + (uint32_t)stage * kWarpStage, meta = raw + kWarpRaw;
      if constexpr (IS_V) V::copy(vc + ((uint32_t)v_col0 >> 4), place, P.v_scale, srow, raw, meta, lane);
      else K::copy(kc, place, P.k_scale, srow, raw, meta, lane);
      ++next.tile;
      if (next.tile < g.n_known) next.n = number<IS_V>(g, next.tile);
    }
    cp_async_commit();
  }
  // A stage's item as bf16 into the ring; for V, the first position that sees a value that is not finite, per 32 columns.
  template <bool IS_V> __device__ __forceinline__ void convert(const AttnGeom& g, int tile, int stage, unsigned char* item) const {
    const uint32_t raw = stage0 + (uint32_t)stage * kWarpStage;
    const uint32_t mine = K::scales(raw + kWarpRaw, lane);
    if constexpr (IS_V) {
      if (lane < V::kRows && __vcmpeq4(mine, 0xFFFFFFFFu) != 0) {
        const TileRows tr = tile_rows<SPARSE>(g, tile);
#pragma unroll
        for (int b = 0; b < D / kMxBlock; ++b)
          if ((mine >> (8 * b) & 0xFFu) == kMxNanScale) atomicMin(v_nan + b, tr.causal ? max(tr.col0 + tile_row<true>(), -1) : -1);
      }
      V::convert(raw, mine, v_col0 / kMxBlock, 0u, item, lw, lane);
    } else {
      K::convert(raw, mine, 0, kBf16Nan2, item, lw, lane);
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
      constexpr bool IS_V = decltype(is_v)::value;
      cp_async_wait<NST - 1>();
      __syncwarp();
      if (!mbar_wait_done(&empty[slot], phase ^ 1, wc)) return false;
      convert<IS_V>(g, tile, stage, ring + (size_t)slot * slot_bytes);
      fence_proxy_async_smem();                       // these stores, before products read the slot
      __syncwarp();
      if (lane == 0) mbar_arrive(&full[slot]);
      if (++slot == SLOTS) { slot = 0; phase ^= 1; }
      if constexpr (NST % 2 == 0) copy<IS_V>(g, IS_V ? v : k, stage);
      else copy<!IS_V>(g, IS_V ? k : v, stage);
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
