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
// What bounds it: instructions.  Five a pair of elements, 16 elements a lane and copy; loads run one copy group (4 of 16 elements a
// lane) ahead of the conversion.
#pragma once

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
// Elements whose bits stand at the top of each half of h, as bf16 numbers times 2^-120 or 2^-126.
template <int FMT>
__device__ __forceinline__ uint32_t mx_spread(uint32_t h) {
  if constexpr (FMT == QUOKA_KV_MXFP8) return (h & 0x80008000u) | (h >> 4 & 0x07F007F0u);
  else return (h & 0x80008000u) | (h >> 6 & 0x01C001C0u);
}
// The 8 elements of half a unit (two words of MXFP8, one of MXFP4) as four bf16 pairs.
template <int FMT>
__device__ __forceinline__ uint4 mx_to_bf16x8(uint32_t w0, uint32_t w1, uint32_t factor2) {
  uint32_t o[4];
  if constexpr (FMT == QUOKA_KV_MXFP8) {
    o[0] = __byte_perm(w0, w0, 0x1100); o[1] = __byte_perm(w0, w0, 0x3322);
    o[2] = __byte_perm(w1, w1, 0x1100); o[3] = __byte_perm(w1, w1, 0x3322);
  } else {
    const uint32_t lo = w0 << 4;                     // (what stands below an element's bits is masked off)
    o[0] = __byte_perm(lo, w0, 0x4400); o[1] = __byte_perm(lo, w0, 0x5511);
    o[2] = __byte_perm(lo, w0, 0x6622); o[3] = __byte_perm(lo, w0, 0x7733);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = mul_bf16x2(mx_spread<FMT>(o[i]), factor2);
  return make_uint4(o[0], o[1], o[2], o[3]);
}

// One loader warp of NLW.  A K item of the ring is ROWS_K tile rows from row k_row0 on, all D columns; a V item all 128 rows, VC columns
// from v_col0 on.  Both are [64-column halves][rows][128 B], 16-byte pieces swizzled by row.
template <int FMT, int D, int ROWS_K, int VC, bool SPARSE, int NLW, int SLOTS>
struct MxLoader {
  static constexpr int KU = D / 16, VU = VC / 16;                      // units per row
  static constexpr int K_RPI = 32 / KU, V_RPI = 32 / VU;               // rows per warp instruction
  static constexpr int K_GROUPS = ROWS_K / (K_RPI * NLW), V_GROUPS = 128 / (V_RPI * NLW);     // row groups of this warp
  static constexpr int SUB = 4;                                        // of them at a time
  static constexpr int KSUB = K_GROUPS / SUB, VSUB = V_GROUPS / SUB;
  static constexpr int K_REGS = (K_GROUPS * K_RPI + 31) / 32, V_REGS = (V_GROUPS * V_RPI + 31) / 32;     // (a lane may be left over)
  static_assert(K_GROUPS % SUB == 0 && V_GROUPS % SUB == 0 && (KSUB + VSUB) % 2 == 0, "whole groups, alternating buffers");
  // a row's number, its offset in units of 16 elements (kNoRow: no such row) and its scale bytes; lane l looks after rows p = l, 32 + l
  // of this warp's rows, p = group * rows per instruction + row of the instruction
  template <int R> struct Rows { int t[R]; uint32_t off[R], scale[R]; };
  typedef decltype(MxUnit<FMT>::w) W;

  const DevParams& P;
  int s, kv, lw, lane, k_row0, v_col0, T;
  uint32_t head, st, sb, srow0;
  const int32_t *table, *idx;
  const W *kc, *vc;
  int* v_nan;

  __device__ __forceinline__ MxLoader(const DevParams& P_, int s_, int kv_, int lw_, int lane_, int k_row0_, int v_col0_, int T_, const void* k,
                                      const void* v, const int32_t* k_idx, int* v_nan_)
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
  }

  template <bool V> __device__ __forceinline__ int tile_row(int r) const {
    constexpr int RPI = V ? V_RPI : K_RPI;
    const int p = 32 * r + lane;
    return (V ? 0 : k_row0) + (lw + p / RPI * NLW) * RPI + p % RPI;
  }
  // row numbers of tile tr (-1 past its end); listed ones are loads
  template <bool V, int R> __device__ __forceinline__ void numbers(const TileRows& tr, int (&t)[R]) const {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int rr = 32 * r + lane < (V ? V_GROUPS * V_RPI : K_GROUPS * K_RPI) ? tile_row<V>(r) : 128;
      if (SPARSE && tr.from_list) {
        const int last = min(tr.count, kKeyTile) - 1;
        const int n = last >= 0 ? __ldcg(idx + tr.first + min(rr, last)) : -1;     // written by the kernel before: L2
        t[r] = rr <= last ? n : -1;
      } else {
        t[r] = rr < min(tr.count, kKeyTile) ? tr.first + rr : -1;
      }
    }
  }
  template <bool V, int R> __device__ __forceinline__ void places(const TileRows& tr, Rows<R>& rows) const {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      int t = rows.t[r];
#ifdef QUOKA_DEBUG
      if (SPARSE && tr.from_list && (t < -1 || t >= T)) { atomicExch(P.status, (int32_t)QUOKA_ERR_BAD_INDEX); t = -1; }
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
      rows.off[r] = t < 0 ? kNoRow : head + off;
      const uint8_t* sc = (V ? P.v_scale : P.k_scale) + (size_t)srow * (D / kMxBlock);
      uint32_t w = 0;
      if (t >= 0) w = D == 128 ? __ldg(reinterpret_cast<const uint32_t*>(sc)) : __ldg(reinterpret_cast<const uint16_t*>(sc));
      rows.scale[r] = w;
    }
  }
  // the first position that sees a value that is not finite, per block of 32 columns
  __device__ __forceinline__ void note_nan(const TileRows& tr, const Rows<V_REGS>& rows) const {
#pragma unroll
    for (int r = 0; r < V_REGS; ++r)
      if (rows.off[r] != kNoRow && __vcmpeq4(rows.scale[r], 0xFFFFFFFFu) != 0) {
#pragma unroll
        for (int b = 0; b < D / kMxBlock; ++b)
          if ((rows.scale[r] >> (8 * b) & 0xFFu) == kMxNanScale) atomicMin(v_nan + b, tr.causal ? max(tr.col0 + tile_row<true>(r), -1) : -1);
      }
  }
  template <bool V, int R> __device__ __forceinline__ void load(const Rows<R>& rows, int sub, W (&buf)[SUB]) const {
    constexpr int RPI = V ? V_RPI : K_RPI, U = V ? VU : KU;
    const W* base = (V ? vc : kc) + (V ? (uint32_t)v_col0 >> 4 : 0u) + lane % U;
#pragma unroll
    for (int i = 0; i < SUB; ++i) {
      const int p = (sub * SUB + i) * RPI;
      const uint32_t off = __shfl_sync(0xFFFFFFFFu, rows.off[p / 32], (p + lane / U) & 31);
      W w = {};
      if (off != kNoRow) w = __ldg(base + off);
      buf[i] = w;
    }
  }
  template <bool V, int R> __device__ __forceinline__ void store(const Rows<R>& rows, int sub, const W (&buf)[SUB], unsigned char* item) const {
    constexpr int RPI = V ? V_RPI : K_RPI, U = V ? VU : KU;
    constexpr uint32_t kHalf = (V ? 128 : ROWS_K) * 128;
    const int u = lane % U, rsub = lane / U;
    const int sw = U == 8 ? u >> 2 : 0;               // lanes of the second half store their second piece first: other banks
#pragma unroll
    for (int i = 0; i < SUB; ++i) {
      const int p = (sub * SUB + i) * RPI;
      const uint32_t word = __shfl_sync(0xFFFFFFFFu, rows.scale[p / 32], (p + rsub) & 31);
      const uint32_t b = word >> (8 * ((V ? v_col0 / kMxBlock : 0) + (u >> 1))) & 0xFFu;
      const uint32_t f = b == kMxNanScale ? (V ? 0u : kBf16Nan2) : mx_factor2<FMT>(b);
      const int row = (lw + (sub * SUB + i) * NLW) * RPI + rsub;
      unsigned char* dst = item + (uint32_t)(u >> 2) * kHalf + (uint32_t)row * 128u;
      const uint32_t p0 = (uint32_t)(((2 * (u & 3) + sw) ^ row) & 7) << 4;
      uint4 first, second;
      if constexpr (FMT == QUOKA_KV_MXFP8) {
        first = mx_to_bf16x8<FMT>(sw ? buf[i].z : buf[i].x, sw ? buf[i].w : buf[i].y, f);
        second = mx_to_bf16x8<FMT>(sw ? buf[i].x : buf[i].z, sw ? buf[i].y : buf[i].w, f);
      } else {
        first = mx_to_bf16x8<FMT>(sw ? buf[i].y : buf[i].x, 0u, f);
        second = mx_to_bf16x8<FMT>(sw ? buf[i].x : buf[i].y, 0u, f);
      }
      *reinterpret_cast<uint4*>(dst + p0) = first;
      *reinterpret_cast<uint4*>(dst + (p0 ^ 16u)) = second;
    }
  }

  // All tiles of this CTA's walk; false when a wait gave up.
  template <typename Learn>
  __device__ __forceinline__ bool run(AttnGeom& g, int t_lo, unsigned char* ring, uint32_t slot_bytes, uint64_t* full, uint64_t* empty,
                                      const WaitCtx& wc, Learn&& learn) {
    int tile = t_lo, slot = 0;
    uint32_t phase = 0;
    if (tile == g.n_known) {
      if (!g.resolved) learn();
      if (tile == g.n_known) return true;
    }
    Rows<K_REGS> k;
    Rows<V_REGS> v;
    W buf[2][SUB];
    TileRows tr = tile_rows<SPARSE>(g, tile);
    const auto whole = [&]() {                        // everything about tile tr, and its first loads
      numbers<false>(tr, k.t);
      numbers<true>(tr, v.t);
      places<false>(tr, k);
      places<true>(tr, v);
      load<false>(k, 0, buf[0]);
    };
    whole();
    for (;;) {
      const bool next = tile + 1 < g.n_known;
      TileRows tn = tr;
      int kt[K_REGS], vt[V_REGS];
      if (next) {
        tn = tile_rows<SPARSE>(g, tile + 1);
        numbers<false>(tn, kt);
        numbers<true>(tn, vt);
      }
      note_nan(tr, v);
#pragma unroll
      for (int sub = 0; sub < KSUB + VSUB; ++sub) {
        // the next group's loads, then this one's conversion; a K tile of the next row numbers behind the last V group
        if (sub + 1 == KSUB + VSUB) {
          if (next) {
#pragma unroll
            for (int r = 0; r < K_REGS; ++r) k.t[r] = kt[r];
            places<false>(tn, k);
            load<false>(k, 0, buf[(sub + 1) & 1]);
          }
        } else if (sub + 1 < KSUB) {
          load<false>(k, sub + 1, buf[(sub + 1) & 1]);
        } else {
          load<true>(v, sub + 1 - KSUB, buf[(sub + 1) & 1]);
        }
        if (sub == 0 || sub == KSUB)
          if (!mbar_wait_done(&empty[slot], phase ^ 1, wc)) return false;
        unsigned char* item = ring + (size_t)slot * slot_bytes;
        if (sub < KSUB) store<false>(k, sub, buf[sub & 1], item);
        else store<true>(v, sub - KSUB, buf[sub & 1], item);
        if (sub == KSUB - 1 || sub == KSUB + VSUB - 1) {
          fence_proxy_async_smem();                   // these stores, before products read the slot
          __syncwarp();
          if (lane == 0) mbar_arrive(&full[slot]);
          if (++slot == SLOTS) { slot = 0; phase ^= 1; }
        }
      }
      ++tile;
      if (next) {
#pragma unroll
        for (int r = 0; r < V_REGS; ++r) v.t[r] = vt[r];
        tr = tn;
        places<true>(tr, v);
      } else {
        if (g.resolved) return true;
        learn();
        if (tile == g.n_known) return true;
        tr = tile_rows<SPARSE>(g, tile);
        whole();
      }
    }
  }
};

}  // namespace quoka
