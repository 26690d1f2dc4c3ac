// Flash-style attention on the 5th-generation tensor cores over
//   [selected cached rows | the chunk's own causal rows]      (Algorithm 2's attention line, Eq. 2)
// or, without an index list, over every cached row (Eq. 2, dense chunk attention).  bf16 in, fp32
// softmax and accumulation, P rounded to bf16 for the PV product.
//
// This file: the kernel whose row blocks are those of one CTA (attn_tc_pair.cuh has the one of pairs, for head_dim 128; attn_tc.cu
// the plan and the launches of both).  A CTA owns two Q tiles (A, B) of 128 rows, or one, chunk positions of all heads of a KV group, and walks the key
// tiles (128 keys) once for both.  Roles:
//   warps 0-3 / 4-7  softmax of Q tile A / B: one thread per query row, S read from tensor memory,
//                    running max / sum in registers, P written back to tensor memory, lazy rescale of
//                    the O accumulator (only when the max grew by more than 2^32), final
//                    normalisation and the global store.
//   warps 8-9        loaders: every K / V row of a tile is fetched with 16-byte cp.async straight
//                    into the 128-byte-swizzled layout the MMA descriptors expect.  The row address
//                    comes from the selected-index list (the gather), the chunk offset, or the page
//                    table, so no compacted copy of K or V is ever made; rows past the end are
//                    zero-filled.  A slot's "full" barrier is armed by the copies themselves.
//   warp 10          issues O += P V (P from tensor memory, V in shared memory, MN-major)
//   warp 11          issues S = Q K^T (both operands in shared memory)
// Where S and P live and what the products wait for: "order of the products" in attn_tiles.cuh.
// K and V tiles share one ring of shared-memory slots in the order K0 V0 K1 V1 ...
// 384 threads and no register re-balancing between roles: every thread may use 168 registers, a thirteenth warp would
// leave it 128.  Sixteen softmax warps with half a row each (96 registers) were slower: 121 us where these take 100
// (777 queries of 32 heads over 5000 listed rows, head_dim 64, the whole call).
#pragma once

#include "attn_mx_loader.cuh"
#include "attn_tiles.cuh"

namespace quoka {

template <int D, int FMT = 0>
constexpr int kSlotsOf = D == 64 ? 8 : kIsMx<FMT> ? 4 : 5;     // of 16 KB, 32 KB
template <int D, int FMT>
constexpr int kMxStagesOf = D == 64 ? 4 : FMT == QUOKA_KV_MXFP8 ? 2 : 3;      // raw items of 16 KB beside four slots, or smaller ones
template <int D, int FMT, bool SPARSE>
using MxTileLoader = MxLoader<FMT, D, 128, D, SPARSE, kSlotsOf<D, FMT>, kMxStagesOf<D, FMT>>;
template <int D, int FMT = 0>
constexpr size_t attn_tc_smem() {
  size_t n = 1024 + (size_t)(2 + kSlotsOf<D, FMT>) * (D / 64) * 16384 + 512;
  if constexpr (kIsMx<FMT>) n += MxTileLoader<D, FMT, false>::kBytes;
  return n;
}

template <int D, bool SPARSE, bool SPLIT, int FMT = 0>
__global__ void __launch_bounds__(kIsMx<FMT> ? kMxAttnThreads : kAttnThreads, 1)
attn_tc_kernel(DevParams P, const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
               const __grid_constant__ CUtensorMap tm_v, const __nv_bfloat16* __restrict__ kc,
               const __nv_bfloat16* __restrict__ vc, const int32_t* __restrict__ k_idx,
               const int32_t* __restrict__ k_cnt, __nv_bfloat16* __restrict__ out, float* __restrict__ lse) {
  constexpr int kSlots = kSlotsOf<D, FMT>, HALVES = D / 64;
  constexpr bool MX = kIsMx<FMT>;                              // a microscaled cache: kc, vc are its bytes
  constexpr int kThreads = MX ? kMxAttnThreads : kAttnThreads;
  constexpr uint32_t kHalfBytes = 128 * 128;                 // 128 rows x 128 B
  constexpr uint32_t kTileBytes = HALVES * kHalfBytes;       // one Q / K / V tile
  // tensor memory (see "order of the products"): S | S | S | O_A | O_B, head_dim 128: S | S | O_A | O_B; P in place
  constexpr int NBUF = D == 64 ? 3 : 2;
  constexpr uint32_t O_COL = NBUF * 128;                     // (Q tile B's O is D columns on)
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  unsigned char* q_smem = smem;                               // [2][HALVES][128][128 B]
  unsigned char* kv_smem = smem + 2 * kTileBytes;             // [kSlots][HALVES][128][128 B]
  uint64_t* bars = reinterpret_cast<uint64_t*>(kv_smem + (size_t)kSlots * kTileBytes);
  uint64_t* kv_full = bars;                 // [kSlots]  the loader threads' cp.async arrivals
  uint64_t* kv_empty = bars + kSlots;       // [kSlots]  MMA commit
  uint64_t* s_full = bars + 2 * kSlots;     // [NBUF]    MMA commit
  uint64_t* p_full = s_full + NBUF;         // [NBUF][2] 4 softmax warps arrive, per half of the key tile
  uint64_t* p_done = p_full + 2 * NBUF;     // [NBUF]    MMA commit: P has been multiplied, the buffer is free
  uint64_t* o_full = p_done + NBUF;         // [2]       MMA commit after the last PV
  uint64_t* q_full = o_full + 2;            // TMA
  uint64_t* q_ready = q_full + 1;           // MX: the Q tiles are in the order of the converted rows, 4 loader warps
  uint64_t* raw_full = q_ready + 1;         // MX: [2][kMxStages] raw items, full and empty
  constexpr int kMxStages = kMxStagesOf<D, FMT>;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(raw_full + 2 * kMxStages);
  __shared__ int abort_flag;
  __shared__ int v_nan[D / kMxBlock];       // MX

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const WaitCtx wc{&abort_flag, P.status};
  // grid = (head groups, row blocks, batch): head groups vary fastest, the row blocks run heaviest (most causal tiles)
  // first, lightest last, the sequences longest first
  const int s = longest_first(P, blockIdx.z), hg = blockIdx.x;
  // (SPLIT: grid.y = row blocks times the parts a row block's key tiles are cut into)
  const int n_parts = SPLIT ? P.attn_parts : 1;
  const int rb = (SPLIT ? P.attn_split_rb : P.attn_row_blocks) - 1 - blockIdx.y / n_parts;
  const QRows qr(P, hg, rb, 0, 1);
  const int kv = qr.head0 / P.group;
  AttnGeom g = make_geom<SPARSE>(P, s, qr.p0, 1);
  // SPLIT: this CTA walks the tiles [t_lo, t_hi) of the row block's sequence only and leaves, per row, a partial
  // result; the part that finishes last adds the parts up.  The list length has to be known before the range is, so
  // nothing of the walk starts before the selection has ended.
  int t_lo = 0;
  if (SPLIT) {
    if (SPARSE) { if (P.attn_after_whole) learn_count(g, k_cnt, s); else resolve(g, k_cnt, s); }
    const int part = blockIdx.y % n_parts;
    t_lo = (int)(((long long)part * g.n_known) / n_parts);
    g.n_known = (int)(((long long)(part + 1) * g.n_known) / n_parts);
  }

  if (threadIdx.x == 0) {
    abort_flag = 0;
    for (int i = 0; i < kSlots; ++i) { mbar_init(&kv_full[i], MX ? kMxLoaderWarps : kLoaderWarps * 32); mbar_init(&kv_empty[i], 1); }
    for (int i = 0; i < NBUF; ++i) { mbar_init(&s_full[i], 1); mbar_init(&p_done[i], 1); }
    for (int i = 0; i < 2 * NBUF; ++i) mbar_init(&p_full[i], 4);
    for (int i = 0; i < 2; ++i) mbar_init(&o_full[i], 1);
    mbar_init(q_full, 1);
    mbar_init(q_ready, kMxLoaderWarps);
    tma_prefetch_desc(&tm_q);
    tma_prefetch_desc(&tm_k);
    tma_prefetch_desc(&tm_v);
    if constexpr (MX) {
      for (int i = 0; i < D / kMxBlock; ++i) v_nan[i] = kNoNan;
      for (int i = 0; i < kMxStages; ++i) { mbar_init(&raw_full[i], kMxCopyWarps * 33); mbar_init(&raw_full[kMxStages + i], kMxLoaderWarps); }
    }
    fence_mbar_init();
  }
  if constexpr (FMT == kUnpacked) attn_load_nan<D>(P, v_nan, s, kv, g.T + P.chunk);
  if (warp == kQkWarp) tmem_alloc(tmem_slot, 512);
  zero_spare_q_rows<D>(P, q_smem, threadIdx.x, kThreads);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  if (!SPARSE && !SPLIT) grid_launch_dependents();

  if constexpr (MX) {
    if (warp < 8) setmaxnreg_inc<kMxSoftmaxRegs>(); else setmaxnreg_dec<kMxOtherRegs>();
  }
  if (warp < 8) {
    // ================================================================== softmax + epilogue
    const int x = warp >> 2;                                  // Q tile A (0) or B (1)
    const int quarter = warp & 3;
    const int row_in_tile = quarter * 32 + lane;
    const int row = qr.position(P, x, row_in_tile);           // chunk position
    const uint32_t lane_addr = tmem_base + ((uint32_t)(quarter * 32) << 16);
    const uint32_t o_addr = lane_addr + O_COL + x * D;
    const float scale_log2 = P.scale * 1.4426950408889634f * (MX ? kMxUnshift : 1.f);
    float m_run = -INFINITY, l_run = 0.f;
    // S buffers go by items: the first of this Q tile's is item 0, or 1 where the other comes first, the next one `step` on
    uint32_t phase = 0;
    int buf = (x ? t_lo >= g.skip_a : g.skip_a > t_lo) ? 1 : 0;
    const int step = g.active_b ? 2 : 1;
    bool ok = true;
    const int skip_x = max(x ? 0 : g.skip_a, t_lo);         // first tile this Q tile takes part in
    const bool active_x = (x ? g.active_b : true) && (!SPLIT || skip_x < g.n_known);
    VisibleCols<SPARSE> vis(g, skip_x, row);
    for (int t = skip_x; active_x; ++t, vis.advance()) {
      if (t == g.n_known) {                                   // end of what is known: the list length, or the end
        if (g.resolved) break;
        resolve(g, k_cnt, s);
        if (t == g.n_known) break;
      }
      vis.at(g, t, row);
      const bool masked = !__all_sync(0xFFFFFFFFu, vis.lim >= kKeyTile);
      if (!mbar_wait(&s_full[buf], phase, wc)) { ok = false; break; }
      tc_fence_after();
      const uint32_t s_addr = lane_addr + buf * 128;
      ok = attn_softmax_tile<D, false>(
          s_addr, s_addr, o_addr, vis.lim, masked, scale_log2, t == skip_x, lane, m_run, l_run, []() {}, []() { return true; },
          [&]() {                                             // products of this Q tile's item before
            const int before = buf - step;
            if (!mbar_wait_done(&p_done[before < 0 ? before + NBUF : before], before < 0 ? phase ^ 1 : phase, wc)) return false;
            tc_fence_after();
            return true;
          },
          [&](int half) { mbar_arrive(&p_full[2 * buf + half]); });
      if (!ok) break;
      buf += step;
      if (buf >= NBUF) { phase ^= 1; buf -= NBUF; }
    }
    // ---- epilogue: O / l -> bf16 -> global
    if constexpr (!SPLIT) {
      if (ok && active_x && mbar_wait(&o_full[x], 0, wc)) {
        tc_fence_after();
        attn_store_row<D, FMT>(P, o_addr, m_run, l_run, s, qr.head(P, row_in_tile), row, row_in_tile < qr.count(P, x), out, lse, v_nan);
      }
    } else {
      const bool have = ok && active_x && mbar_wait(&o_full[x], 0, wc);
      if (have) tc_fence_after();
      attn_split_epilogue<D, FMT>(P, (s * QRows::groups(P) + hg) * P.attn_split_rb + rb, blockIdx.y % n_parts, n_parts, x, quarter, lane,
                             row_in_tile, row, row_in_tile < qr.count(P, x), have, o_addr, m_run, l_run, s, qr.head(P, row_in_tile),
                             out, lse, v_nan);
    }
  } else if (MX && warp >= kMxFirstLoader) {
    // ================================================================== microscaled cache: rows converted
    if constexpr (MX) {
      MxTileLoader<D, FMT, SPARSE> loader{P, s, kv, lane, 0, 0, reinterpret_cast<unsigned char*>(bars) + 512, raw_full, raw_full + kMxStages};
      if (mx_order_q<FMT>(q_smem, P.attn_qtiles * (int)kTileBytes, threadIdx.x - 32 * kMxFirstLoader, 32 * kMxLoaderWarps, q_full, q_ready, wc))
        loader.convert(g, t_lo, warp - kMxFirstLoader, kv_smem, kTileBytes, kv_full, kv_empty, v_nan, wc, [&]() { resolve(g, k_cnt, s); });
    }
  } else if (warp < 8 + kLoaderWarps) {
    // ================================================================== K / V row loaders (gather)
    // One warp instruction copies four whole rows (eight lanes x 16 bytes cover a 128-byte row; head_dim 128: two); the row
    // groups of a tile are dealt round-robin to the loader warps.
    if constexpr (MX) {
      MxTileLoader<D, FMT, SPARSE> loader{P, s, kv, lane, 0, 0, reinterpret_cast<unsigned char*>(bars) + 512, raw_full, raw_full + kMxStages};
      loader.fill(g, t_lo, warp - 8, kc, vc, k_idx, &tm_k, &tm_v, wc, [&]() { resolve(g, k_cnt, s); });
    } else {
    const int lw = warp - 8;
    constexpr int PIECES = D / 8;                             // 16-byte pieces per row (16 or 8)
    constexpr int ROWS_PER_INSTR = 32 / PIECES;               // 2 or 4
    constexpr int GROUPS = kKeyTile / ROWS_PER_INSTR;         // 64 or 32 row groups per tile
    constexpr int RPT = GROUPS / kLoaderWarps;                // row groups per warp
    const int c16 = lane % PIECES;                            // this thread's piece of the row
    const int rsub = lane / PIECES;
    // a thread's rows are 8 apart and have the same swizzle, or 4 apart, and it is turned by 4 rows for every second one
    static_assert(kLoaderWarps * ROWS_PER_INSTR == (HALVES == 1 ? 8 : 4), "rows of a thread");
    const int lrow = lw * ROWS_PER_INSTR + rsub;
    const uint32_t thread_dst = (uint32_t)((c16 >> 3) * kHalfBytes + lrow * 128 + (((c16 & 7) ^ lrow) << 4));
    const auto row_dst = [](uint32_t dst, int i) {
      return (HALVES == 1 || (i & 1) == 0 ? dst : dst ^ 64u) + (uint32_t)(i * kLoaderWarps * ROWS_PER_INSTR * 128);
    };
    const int32_t* idx = SPARSE ? k_idx + ((long long)s * P.n_kv + kv) * P.budget_cap : nullptr;
    uint32_t phase = 0;
    int slot = 0;
    const uint32_t kv_base = smem_u32(kv_smem);
    // Row addressing in 16-byte units, 32 bits wide (the host refuses caches of 2^32 - 1 units and more; strides are
    // multiples of 8 elements): sequence/head base plus this thread's piece, row stride, page stride.
    const uint32_t st16 = (uint32_t)(P.kv_st >> 3), sb16 = (uint32_t)(P.kv_sb >> 3);
    const uint32_t base16 = (uint32_t)(((P.page_size == 0 ? (long long)s * P.kv_sb : 0ll) + (long long)kv * P.kv_sh) >> 3) +
                            (uint32_t)c16;
    const int32_t* table = P.block_table + (long long)s * P.max_pages;
    // The warp's RPT * ROWS_PER_INSTR rows of a tile are numbered p = i * ROWS_PER_INSTR + rsub (i = its i-th row group); lane
    // l looks after rows p = l and p = 32 + l: their row numbers (-1 past the end), for listed rows fetched when the
    // previous tile's copies have been issued and looked at when this tile's are, and their offsets, worked out once per
    // tile.  The thread that copies a row fetches its offset by shuffle.  The per-row code is kept free of branches: a branch
    // per row costs a single warp far more than the arithmetic it skips.
    constexpr int LIST_REGS = RPT * ROWS_PER_INSTR / 32;
    static_assert(GROUPS % kLoaderWarps == 0 && RPT * ROWS_PER_INSTR % 32 == 0, "whole registers of rows");
    int rows[LIST_REGS], rr_of[LIST_REGS];
    uint32_t offs[LIST_REGS];
    bool all_rows = false;
#pragma unroll
    for (int k = 0; k < LIST_REGS; ++k) {
      const int pp = 32 * k + lane;
      rr_of[k] = (lw + (pp / ROWS_PER_INSTR) * kLoaderWarps) * ROWS_PER_INSTR + pp % ROWS_PER_INSTR;
      rows[k] = -1;
      offs[k] = kNoRow;
    }
    auto list_rows = [&](int base, int count) {
      const int last = min(count, kKeyTile) - 1;                   // last valid row of the tile
      if (last >= 0) {
#pragma unroll
        for (int k = 0; k < LIST_REGS; ++k) {
          const int v = __ldcg(idx + base + min(rr_of[k], last));  // written by the kernel before: L2, not the read-only path
          rows[k] = rr_of[k] <= last ? v : -1;
        }
      }
    };
    for (int tile = t_lo;; ++tile) {
      if (tile == g.n_known) {                                // end of what is known: the list length, or the end
        if (g.resolved) break;
        resolve(g, k_cnt, s);
        if (tile == g.n_known) break;
      }
      const TileRows tr = tile_rows<SPARSE>(g, tile);
      bool stop = false;
#pragma unroll 1
      for (int kvi = 0; kvi < 2; ++kvi) {                     // the tile's K rows, then its V rows
        if (!mbar_wait_done(&kv_empty[slot], phase ^ 1, wc)) { stop = true; break; }
        // A whole tile of consecutive rows (page-aligned in a paged cache) is fetched by the copy engine as 64-row
        // boxes: one thread issues them, the others only keep the barrier's arrival count.  Ragged tiles (rows past
        // the end must read as zeros, not as whatever the cache holds there) and listed rows take the copies below.
        if (!tr.from_list && tr.count >= kKeyTile && (P.page_size == 0 || (tr.first & (kPage - 1)) == 0)) {
          if (lw == 0 && lane == 0) {
            fence_proxy_async_smem();             // earlier contents of the slot were written through the generic proxy
            mbar_arrive_expect_tx(&kv_full[slot], kTileBytes);
            unsigned char* dst = kv_smem + (size_t)slot * kTileBytes;
            const CUtensorMap* tm = kvi ? &tm_v : &tm_k;
#pragma unroll
            for (int sub = 0; sub < 2; ++sub) {
              int c1 = tr.first + sub * 64, c3 = s;
              if (P.page_size != 0) { c1 = 0; c3 = __ldg(table + (tr.first >> 6) + sub); }
#pragma unroll
              for (int hh = 0; hh < HALVES; ++hh)
                tma_load_4d(dst + hh * kHalfBytes + sub * 64 * 128, tm, &kv_full[slot], hh * 64, c1, kv, c3);
            }
          } else {
            mbar_arrive(&kv_full[slot]);
          }
          if (++slot == kSlots) { slot = 0; phase ^= 1; }
          continue;
        }
        if (kvi == 0) {
          if (tr.from_list && tile == max(g.n_chunk, t_lo)) list_rows(tr.first, tr.count);   // first list tile
#pragma unroll
          for (int k = 0; k < LIST_REGS; ++k) {
            if (!tr.from_list) rows[k] = rr_of[k] < tr.count ? tr.first + rr_of[k] : -1;
            offs[k] = kv_row_off16(P, table, st16, sb16, rows[k], tr.from_list, g.T);
            all_rows = (k == 0 || all_rows) && offs[k] != kNoRow;
          }
          all_rows = warp_all(all_rows);
        }
        const uint4* src_base = reinterpret_cast<const uint4*>(kvi ? vc : kc) + base16;
        const uint32_t dst = kv_base + slot * kTileBytes + thread_dst;
        if (all_rows) {                                           // no size to select
#pragma unroll
          for (int i = 0; i < RPT; ++i) {
            const uint32_t off = __shfl_sync(0xFFFFFFFFu, offs[(i * ROWS_PER_INSTR) / 32], (i * ROWS_PER_INSTR + rsub) & 31);
            cp_async_16(row_dst(dst, i), src_base + off);
          }
        } else {
#pragma unroll
          for (int i = 0; i < RPT; ++i) {
            const uint32_t off = __shfl_sync(0xFFFFFFFFu, offs[(i * ROWS_PER_INSTR) / 32], (i * ROWS_PER_INSTR + rsub) & 31);
            cp_async_16(row_dst(dst, i), src_base + (off == kNoRow ? 0u : off), off != kNoRow);
          }
        }
        // this thread's share of the slot is signalled by the copy engine itself when the bytes have landed:
        // no wait in the loader, every slot of the ring can be in flight
        cp_async_mbar_arrive_noinc(&kv_full[slot]);
        if (kvi == 1 && tr.from_list) list_rows(tr.first + kKeyTile, tr.count - kKeyTile);   // next list tile
        if (++slot == kSlots) { slot = 0; phase ^= 1; }
      }
      if (stop) break;
    }
    cp_async_wait_all();                                      // nothing of this thread is in flight at exit
    }
  } else {
    // ================================================================== warp 11: QK^T, warp 10: PV
    if (warp == kQkWarp && lane == 0) load_q_tiles<D>(P, qr, q_smem, &tm_q, q_full, s);
    __syncwarp();
    const bool leader = elect_one();
    const uint32_t tmem = (uint32_t)warp_uniform((int)tmem_base);
    t_lo = warp_uniform(t_lo);
    uniform_geom(g);
    const uint32_t kv_base = smem_u32(kv_smem);
    const auto acquire = [&](int sl, uint32_t phase) {
      if (!warp_all(mbar_poll(&kv_full[sl], phase, wc))) return false;
      fence_proxy_async_smem();               // cp.async wrote through the generic proxy, the MMA reads through the async one
      tc_fence_after();
      return true;
    };
    const auto release = [&](int sl) { if (leader) mma_commit(&kv_empty[sl]); };
    // Operand descriptors are built once; a tile, slot or k-step offset is an addition to the 16-byte-unit
    // address field (shared memory addresses stay far below the field's 14 bits).
    // The sparse sequence's length is learnt (resolve) just before the walk past the chunk's own tiles.
    if (warp == kQkWarp) {
      const uint32_t idesc_qk = idesc_bf16_f32(128, kKeyTile, false, false);
      const uint64_t desc_q = smem_desc_sw128(smem_u32(q_smem), 16, 1024);
      const uint64_t desc_k = smem_desc_sw128(kv_base, 16, 1024);            // K-major rows (K tiles)
      if (warp_all(mbar_poll(MX ? q_ready : q_full, 0, wc)))
        attn_issue_qk<NBUF, kSlots>(
            g, t_lo, [&]() { resolve(g, k_cnt, s); uniform_geom(g); grid_launch_dependents(); }, acquire,
            [&](unsigned buf, uint32_t parity) {
              if (!warp_all(mbar_poll(&p_done[buf], parity, wc))) return false;
              tc_fence_after();
              return true;
            },
            [&](int x, unsigned buf, int ks) {
              const uint64_t da = desc_q + (uint64_t)(x * (kTileBytes >> 4));
              const uint64_t db = desc_k + (uint64_t)((uint32_t)ks * (kTileBytes >> 4));
#pragma unroll
              for (int hh = 0; hh < HALVES; ++hh)
#pragma unroll
                for (int kk = 0; kk < 4; ++kk) {
                  const uint64_t o = (uint64_t)((hh * kHalfBytes + kk * 32) >> 4);
                  if (leader) mma_ss(tmem + buf * 128, da + o, db + o, idesc_qk, (hh | kk) ? 1u : 0u);
                }
              if (leader) mma_commit(&s_full[buf]);
            },
            release);
    } else {
      const uint32_t idesc_pv = idesc_bf16_f32(128, D, false, true);
      const uint64_t desc_v = smem_desc_sw128(kv_base, HALVES == 1 ? 16 : kHalfBytes, 1024);      // MN-major rows (V tiles)
      uint32_t p_phase = 0;
      attn_issue_pv<NBUF, kSlots>(
          g, t_lo, [&]() { resolve(g, k_cnt, s); uniform_geom(g); }, acquire,
          [&](int x, int half, unsigned buf, int vs, bool add) {
            if (!warp_all(mbar_poll(&p_full[2 * buf + half], (p_phase >> buf) & 1u, wc))) return false;
            tc_fence_after();
            const uint64_t dv = desc_v + (uint64_t)((uint32_t)vs * (kTileBytes >> 4) + half * 4 * (2048 >> 4));
            const uint32_t pa = tmem + buf * 128 + half * 32, oa = tmem + O_COL + x * D;
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)             // 16 keys per MMA: 8 packed columns of P, 16 rows of V
              if (leader) mma_ts(oa, pa + kk * 8, dv + (uint64_t)(kk * (2048 >> 4)), idesc_pv, add || kk ? 1u : 0u);
            if (half) {
              if (leader) mma_commit(&p_done[buf]);
              p_phase ^= 1u << buf;
            }
            return true;
          },
          release, [&](int x) { if (leader) mma_commit(&o_full[x]); });
    }
  }
  if constexpr (MX) {
    // As launched, once every warp has had its share: a warp that took registers back before would keep a softmax warp from
    // ever getting its own.
    __syncthreads();
    if (warp < 8) setmaxnreg_dec<128>(); else setmaxnreg_inc<128>();
  }
  if (SPLIT && attn_last_cta()) grid_dependency_wait();       // this grid's end is the whole row blocks' end too
  tc_fence_before();
  __syncthreads();
  if (warp == kQkWarp) tmem_dealloc(tmem_base, 512);
}

template <int D, int FMT>
AttnKernel pick_attn_tc(bool sparse, bool parts, bool) {
  if (parts) return sparse ? attn_tc_kernel<D, true, true, FMT> : attn_tc_kernel<D, false, true, FMT>;
  return sparse ? attn_tc_kernel<D, true, false, FMT> : attn_tc_kernel<D, false, false, FMT>;
}

}  // namespace quoka
