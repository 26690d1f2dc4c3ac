// Loader warps of the tensor-core attention kernels over a microscaled cache.  Two warps bring raw rows of 8- or 4-bit elements, and their
// scale words, into stages of shared memory: whole tiles of consecutive rows by the copy engine, listed rows and ragged tiles by cp.async.  Four
// others take them from there, make them bf16 and put them into the ring's tiles in the layout the operand descriptors expect; the rest of
// those kernels does not know the difference.
//
// The conversion is in mx_rows.cuh.  Tiles hold the cache's values times 2^-16; the softmax scale and the division by the row sum take
// that back.
//
// Values that are not finite (scale byte 255): a key's block becomes NaN, its column of S with it, and rows that do not see the
// column set it to minus infinity.  A value's block becomes zeros, as its products with weights of zero would reach rows that do not see
// it; the first chunk position that sees one is kept per block of columns, and the epilogue makes NaN of what is at or behind it.
//
// What bounds it: the conversion's instructions, which share the issue ports with the softmax.
#pragma once

#include <type_traits>

#include "mx_rows.cuh"

namespace quoka {

// 512 threads: the roles of the bf16 kernels in the first 12 warps, where the loaders only bring raw rows in; the last four, one on
// each sub-partition's issue port, convert them.  A thread may then have 128 registers; the softmax warps take 168 and the others give them.
constexpr int kMxAttnThreads = 512, kMxLoaderWarps = 4, kMxFirstLoader = 12;
constexpr int kMxSoftmaxRegs = 168, kMxOtherRegs = 88;
static_assert(256 * kMxSoftmaxRegs + 256 * kMxOtherRegs == kMxAttnThreads * 128, "what the block is launched with");


// The CTA's Q tiles in the order of converted rows, in place, by the converting warps before their first item; `ready` gets an arrival of each warp.
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

// A K item of the ring is ROWS_K tile rows from row k_row0 on, all D columns; a V item all 128 rows, VC columns from v_col0 on.  Two warps
// (`fill`) bring items into NST stages, four (`convert`) take them from there to the ring's slots; the barriers raw_full, raw_empty [NST]
// are between them.
constexpr int kMxCopyWarps = 2;
template <int FMT, int D, int ROWS_K, int VC, bool SPARSE, int SLOTS, int NST>
struct MxLoader {
  typedef MxItem<FMT, D, ROWS_K, D> K;
  typedef MxItem<FMT, D, 128, VC> V;
  typedef typename K::W W;
  static constexpr uint32_t kStage = ((K::kStage > V::kStage ? K::kStage : V::kStage) + 127) / 128 * 128;
  static constexpr uint32_t kBytes = NST * kStage;                     // shared memory of all stages
  static constexpr int kFullArrivals = kMxCopyWarps * 33;              // every lane when its copies have landed, a lane for the scale words

  const DevParams& P;
  int s, kv, lane, k_row0, v_col0;
  unsigned char* stages;
  uint64_t *raw_full, *raw_empty;

  // ---- filling
  // numbers of this lane's rows in a tile, of listed ones loads (whether there are such rows is asked later)
  template <typename I> __device__ __forceinline__ void numbers(const AttnGeom& g, int tile, int row0, int w, const int32_t* idx,
                                                                int (&n)[I::template kMine<kMxCopyWarps>]) const {
    if (tile >= g.n_known) return;
    const TileRows tr = tile_rows<SPARSE>(g, tile);
#pragma unroll
    for (int i = 0; i < I::template kMine<kMxCopyWarps>; ++i) {
      const int rr = row0 + I::template row<kMxCopyWarps>(w, i, lane);
      n[i] = SPARSE && tr.from_list ? __ldcg(idx + tr.first + max(min(rr, min(tr.count, kKeyTile) - 1), 0)) : tr.first + rr;   // (written by the kernel before: L2)
    }
  }
  // An item's rows of this lane: where they are, and their scale words (on their way until the item is finished).
  template <typename I> struct Mine { uint32_t place[I::template kMine<kMxCopyWarps>], word[I::template kMine<kMxCopyWarps>]; };
  template <typename I>
  __device__ __forceinline__ void prepare(const TileRows& tr, int row0, int w, const MxPlaces& places, const int (&n)[I::template kMine<kMxCopyWarps>], const uint8_t* scale,
                                          Mine<I>& m) const {
#pragma unroll
    for (int i = 0; i < I::template kMine<kMxCopyWarps>; ++i) {
      const int r = I::template row<kMxCopyWarps>(w, i, lane);
      int t = r < (int)(I::kHalf / 128) && row0 + r < min(tr.count, kKeyTile) ? n[i] : -1;
#ifdef QUOKA_DEBUG
      if (SPARSE && tr.from_list && (t < -1 || t >= __ldg(P.ctx_len + s))) { atomicExch(P.status, (int32_t)QUOKA_ERR_BAD_INDEX); t = -1; }
#endif
      uint32_t srow;
      places.of(P, t, m.place[i], srow);
      m.word[i] = 0u;
      if (m.place[i] != kNoRow) m.word[i] = I::load_scales(scale, srow);
    }
  }
  template <typename I>
  __device__ __forceinline__ void bring(const TileRows& tr, int row0, int w, const MxPlaces& places, const Mine<I>& m, const W* cache, const CUtensorMap* tm, int col_bytes,
                                        int stage) const {
    // A whole tile of consecutive rows (page-aligned in a paged cache) comes through the copy engine as 64-row boxes.
    if (!tr.from_list && tr.count >= kKeyTile && (P.page_size == 0 || (tr.first & (kPage - 1)) == 0)) {
      if (w == 0 && lane == 0) {
        fence_proxy_async_smem();                     // earlier contents of the stage were read, or written, through the generic proxy
        mbar_expect_tx(&raw_full[stage], I::kRaw);
#pragma unroll
        for (int sub = 0; sub < (int)(I::kHalf / 8192); ++sub) {
          int c1 = tr.first + row0 + sub * 64, c3 = s;
          if (P.page_size != 0) { c3 = __ldg(places.table + (c1 >> 6)); c1 = 0; }
          tma_load_4d(stages + (uint32_t)stage * kStage + sub * 64 * I::kRowBytes, tm, &raw_full[stage], col_bytes, c1, kv, c3);
        }
      }
    } else {
      I::template copy<kMxCopyWarps>(cache, m.place, smem_u32(stages) + (uint32_t)stage * kStage, w, lane);
    }
    cp_async_mbar_arrive_noinc(&raw_full[stage]);
  }
  template <typename I> __device__ __forceinline__ void finish(int w, const Mine<I>& m, int stage) const {
#pragma unroll
    for (int i = 0; i < I::template kMine<kMxCopyWarps>; ++i) {
      const int r = I::template row<kMxCopyWarps>(w, i, lane);
      if (r < (int)(I::kHalf / 128)) I::put_scales(smem_u32(stages) + (uint32_t)stage * kStage, r, m.word[i]);
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(&raw_full[stage]);
  }
  template <typename Learn>
  __device__ __forceinline__ void fill(AttnGeom& g, int t_lo, int w, const void* kc, const void* vc, const int32_t* k_idx, const CUtensorMap* tm_k,
                                       const CUtensorMap* tm_v, const WaitCtx& wc, Learn&& learn) const {
    MxPlaces places(P);
    places.at_head(P, s, kv);
    const int32_t* idx = SPARSE ? k_idx + ((long long)s * P.n_kv + kv) * P.budget_cap : nullptr;
    int kn[K::template kMine<kMxCopyWarps>], vn[V::template kMine<kMxCopyWarps>];
    Mine<K> mk;
    Mine<V> mv;
    int stage = 0;
    uint32_t phase = 0;
    TileRows tr;
    const auto next_stage = [&]() { if (++stage == NST) { stage = 0; phase ^= 1; } };
    // What an item needs is asked for an item or more before it is looked at: row numbers (listed: loads), then scale words.
    const auto begin = [&](int tile) {
      tr = tile_rows<SPARSE>(g, tile);
      numbers<K>(g, tile, k_row0, w, idx, kn);
      numbers<V>(g, tile, 0, w, idx, vn);
      prepare<K>(tr, k_row0, w, places, kn, P.k_scale, mk);
      numbers<K>(g, tile + 1, k_row0, w, idx, kn);
    };
    if (t_lo < g.n_known) begin(t_lo);
    for (int tile = t_lo;; ++tile) {
      if (tile == g.n_known) {                        // end of what is known: the list length, or the end
        if (g.resolved) break;
        learn();
        if (tile == g.n_known) break;
        begin(tile);
      }
      prepare<V>(tr, 0, w, places, vn, P.v_scale, mv);
      numbers<V>(g, tile + 1, 0, w, idx, vn);
      if (!mbar_wait(&raw_empty[stage], phase ^ 1, wc)) break;
      bring<K>(tr, k_row0, w, places, mk, static_cast<const W*>(kc), tm_k, 0, stage);
      finish<K>(w, mk, stage);
      next_stage();
      TileRows tn = tr;
      if (tile + 1 < g.n_known) {
        tn = tile_rows<SPARSE>(g, tile + 1);
        prepare<K>(tn, k_row0, w, places, kn, P.k_scale, mk);
        numbers<K>(g, tile + 2, k_row0, w, idx, kn);
      }
      if (!mbar_wait(&raw_empty[stage], phase ^ 1, wc)) break;
      bring<V>(tr, 0, w, places, mv, static_cast<const W*>(vc) + (v_col0 >> 4), tm_v, v_col0 / 16 * V::kUnitBytes, stage);
      finish<V>(w, mv, stage);
      next_stage();
      tr = tn;
    }
    cp_async_wait_all();                              // nothing of this thread is in flight at exit
  }

  // ---- converting
  template <typename Learn>
  __device__ __forceinline__ void convert(AttnGeom& g, int t_lo, int w, unsigned char* ring, uint32_t slot_bytes, uint64_t* full, uint64_t* empty, int* v_nan,
                                          const WaitCtx& wc, Learn&& learn) const {
    int slot = 0, stage = 0;
    uint32_t phase = 0, raw_phase = 0;
    const auto one = [&](bool is_v, int tile) -> bool {
      if (!mbar_wait(&raw_full[stage], raw_phase, wc) || !mbar_wait_done(&empty[slot], phase ^ 1, wc)) return false;
      const uint32_t at = smem_u32(stages) + (uint32_t)stage * kStage;
      if (is_v) {
        uint32_t mine;                                // this lane's row: the first position that sees a value that is not finite, per 32 columns
        const int r = 32 * w + lane;
        asm volatile("ld.shared.u32 %0, [%1];" : "=r"(mine) : "r"(at + V::kRaw + 4 * r) : "memory");
        if (__vcmpeq4(mine, 0xFFFFFFFFu) != 0) {
          const TileRows tr = tile_rows<SPARSE>(g, tile);
          for (int b = 0; b < D / kMxBlock; ++b)
            if ((mine >> (8 * b) & 0xFFu) == kMxNanScale) atomicMin(v_nan + b, tr.causal ? max(tr.col0 + r, -1) : -1);
        }
      }
      mx_convert<FMT, kMxLoaderWarps, false>(at, at + (is_v ? V::kRaw + v_col0 / kMxBlock : K::kRaw), is_v ? V::kRows : K::kRows, is_v ? V::kHalves : K::kHalves,
                                             is_v ? V::kRowBytes : K::kRowBytes, is_v ? 0u : kBf16Nan2, ring + (size_t)slot * slot_bytes,
                                             is_v ? V::kHalf : K::kHalf, w, lane);
      fence_proxy_async_smem();                       // these stores, before products read the slot
      __syncwarp();
      if (lane == 0) { mbar_arrive(&full[slot]); mbar_arrive(&raw_empty[stage]); }
      if (++slot == SLOTS) { slot = 0; phase ^= 1; }
      if (++stage == NST) { stage = 0; raw_phase ^= 1; }
      return true;
    };
    for (int tile = t_lo;; ++tile) {
      if (tile == g.n_known) {
        if (g.resolved) break;
        learn();
        if (tile == g.n_known) break;
      }
      bool ok = true;
#pragma unroll 1
      for (int i = 0; i < 2 && ok; ++i) ok = one(i != 0, tile);
      if (!ok) break;
    }
  }
};

}  // namespace quoka
