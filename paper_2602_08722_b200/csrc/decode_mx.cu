// Attention of a few query rows per KV head over a microscaled cache: generation steps, and the few positions of a speculated
// continuation.  The C chunk positions of the G heads of a KV group are R = C G query rows, taken 8 or 16 at a time.
//
// What bounds it: HBM (every row of the cache is read once and used for a dozen multiplications), and next to it the instructions
// that turn 8 or 4 bits into operands.  So the products are matrix instructions with the keys on the M side (m16n8k16: the query
// rows fill the 8 columns, a 128-row tcgen05 tile would have 4 or 8 rows of use in 128), whose operands a lane builds in registers from raw
// bytes:
//   S^T = K Q^T   a lane reads 16-byte pieces of key rows; which columns they are does not matter to the sum, Q's fragment has the same
//   O^T = V^T P^T a lane reads the same 8 or 16 columns of value rows and interleaves the rows of a pair
// P^T comes out of S^T by 8 x 8 transpositions (movmatrix).  The rows come into a ring of shared memory that a warp has for itself: 32
// consecutive ones by the copy engine, of which lane 0 asks for a box and every lane waits on the barrier; others by cp.async of all lanes, each
// waiting for its own and then for the warp.
//
// The operands are fp16, which the conversion instructions make of 8 and 4 bits at once (by shifts and masks, as bf16, it took twice
// the instructions: 637 for 16 keys of 128 columns, 171 us for a step of 16 sequences of 8K to 32K rows):
//   K  each row is divided by its largest block's scale, which goes into the row's score in fp32;
//   Q  each row is multiplied by a power of two to 2^14 .. 2^15, taken off the score in fp32;
//   V  blocks are divided by a scale of O's columns, which follows the largest one met;
//   P  weights 2^(x - m), m a reference point that the largest exponent x exceeds by 7 when it is set and by 15 at most.
// Products are exact as long as fp16 holds the operands: blocks of a key 2^15 (4-bit elements 2^23) below its largest, elements of a query
// 2^31 below its largest, blocks of values 2^9 below the largest of their columns.  Where a granule of 32 keys has others, and only there, its
// scores or its weighted values are taken from bf16 operands, which hold every value of a cache: so what a key of no weight, or one that a row
// does not see, is worth has no part in the row's rounding.  Weights are fp16 otherwise; those 2^-32 times the largest and less then vanish, against
// values 2^9 times the others' at most.  To look for such granules takes 1 % of the time (sixteen long sequences in a warm loop: 133.0 us, without 132.4), with the code
// for them out of line (in line 135.7).  What they cost, sixteen sequences of 20000 rows, 119 us: values of zero, or far from the others', in every granule 144, keys
// or queries 2^30 below their largest 333 to 357.
//
// Split: units are (sequence, KV head, row group).  Few keys: a CTA per unit, or a cluster of CTAs with an equal share of the unit's granules of
// 32 keys each, whose results are added up through distributed shared memory.  Else the granules of all units are one list, cut into equal contiguous
// shares, one per CTA, and a second kernel adds up the units that several CTAs share: long lists are balanced whatever the sequences' lengths
// are.  Inside a CTA the warps take granules in turn, each with a running maximum, sum and output of its own, added up at the end of a unit's part.
// All parts are added up in order.  Weights are rounded to fp16 (bf16) for the product and divided by their sum as rounded, so that they add up to
// one; the log-sum-exp is that of the weights before.
//
// Measured, MXFP8, us: 16 sequences of 8192 to 32768 rows, 8 KV heads of 4, d 128, one position: 148 among other work (735 MB: 5.0 TB/s), 134 one
// call after the other (5.5 TB/s; over a bf16 cache 557); one of 4003 rows 14.4; 5 positions of 8 heads, d 64, MXFP4, three
// sequences of 9001 to 20011 rows 39.4.  Before granules were looked at for their range, one call after the other, MXFP8 / MXFP4: one sequence of 131072
// rows 63 / 59, of 32768 29 / 27; over 131072 rows 867 instructions per 32 keys, the issue ports busy for 48 % of the cycles, the integer pipe for 47 %.
#include <algorithm>
#include <atomic>

#include "decode_mx.cuh"

namespace quoka {

// Warps of a CTA: what registers (168 for twelve) leave room for.  Those from kDecLast on hand their results to the others before these
// are added up, which halves the shared memory for it: twelve rings of 8-bit rows leave 29 KB.
template <int NT>
constexpr int kDecWarps = NT == 1 ? 12 : 8;
constexpr int kDecAtOnce = 8;                          // parts of a cluster whose results a thread has on their way
template <int NT>
constexpr int kDecLast = NT == 1 ? 6 : 8;
template <int FMT, int D, int NT>
__global__ void __launch_bounds__(32 * kDecWarps<NT>, 1)
decode_mx_kernel(DevParams P, DecWork work, const __nv_bfloat16* __restrict__ q, const uint8_t* __restrict__ kc, const uint8_t* __restrict__ vc,
                 const int32_t* __restrict__ k_idx, __nv_bfloat16* __restrict__ out, float* __restrict__ lse, float* __restrict__ parts, int per_unit,
                 const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v) {
  typedef DecBytes<FMT, D> B;
  constexpr int WARPS = kDecWarps<NT>, LAST = kDecLast<NT>, ST = kDecStages, ROWS = 8 * NT, TILES = D / 16, KSTEPS = D / 16;
  constexpr int KW = B::kKBytes * B::kKPieces / 4, VW = B::kVBytes / 4;      // words of a lane per row
  constexpr int LD = D + 4;                                                  // floats of a row of the merge buffer
  extern __shared__ unsigned char dec_smem_raw[];
  unsigned char* dec_smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(dec_smem_raw) + 1023) & ~(uintptr_t)1023);
  grid_dependency_wait();
  grid_launch_dependents();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
  const uint32_t ring = smem_u32(dec_smem) + (uint32_t)warp * (ST * 2 * B::kTile);               // [WARPS][ST][K | V], then [WARPS][ST] scale words
  const uint32_t metas = smem_u32(dec_smem) + (uint32_t)(WARPS * ST * 2) * B::kTile + (uint32_t)warp * (ST * B::kMeta);
  uint64_t* landed = reinterpret_cast<uint64_t*>(dec_smem + WARPS * ST * B::kStage) + warp * ST;     // [WARPS][ST]
  float* merge = reinterpret_cast<float*>(dec_smem + WARPS * ST * (B::kStage + 8));              // [LAST][ROWS][LD], then m, l, lx [LAST][ROWS]
  float* merge_ml = merge + LAST * ROWS * LD;
  __shared__ int abort_flag;
  const WaitCtx wc{&abort_flag, P.status};
  // ---- this CTA's share
  const auto share = [&]() -> DecPart {
    if (per_unit > 0) {
      DecPart p(P, work, blockIdx.x / per_unit);
      const int rank = blockIdx.x % per_unit;
      p.begin = (int)((long long)p.n * rank / per_unit);
      p.end = (int)((long long)p.n * (rank + 1) / per_unit);
      return p;
    }
    const DecTotals all(P, work, 0, lane);
    const long long each = all.share(gridDim.x), lo = min(each * blockIdx.x, all.total);
    if (lo == all.total) { DecPart none(P, work, 0); none.end = 0; return none; }
    return DecPart(P, work, all, lo, min(lo + each, all.total), lane);
  };
  DecPart in = share();
  if (in.begin >= in.end && per_unit <= 1) return;    // (nothing of the list is left for this CTA)
  DecPart part = in;
  if (threadIdx.x == 0) abort_flag = 0;
  if (lane == 0) {
    for (int i = 0; i < ST; ++i) mbar_init(&landed[i], 1);
    fence_mbar_init();
  }
  __syncthreads();
  // ---- copies: granules begin + warp, + WARPS .. of every part.  A lane looks after a row: its number two granules ahead, its place one.
  // 32 consecutive rows come through the copy engine (16-byte cp.async alone, about 20 bytes a clock and SM, held a list of 131072 rows at
  // 4.1 TB/s); listed ones, and the last of a sequence, whose tiles end in zeros, by cp.async.
  MxPlaces places(P);
  int pos = in.begin + warp;
  bool more = true;
  int n_next, s_next = 0, kv_next = 0;                // of the granule whose places are worked out next
  bool live_next = false, run_next = false;
  int first_next = 0;                                 // run: the first of its consecutive rows
  uint32_t place = kNoRow, srow = 0;                  // of the granule that is copied next
  bool live = false, run = false;
  int first = 0, s_fill = 0, kv_fill = 0, page = 0;
  const auto ask = [&]() {
    while (more && pos >= in.end) { more = in.next(P, work); pos = in.begin + warp; }
    live_next = more;
    s_next = in.s; kv_next = in.kv;
    n_next = -1;
    run_next = false;
    if (more) {
      first_next = pos * kDecGranule;
      run_next = !k_idx && first_next + kDecGranule <= in.lens.cnt + P.chunk;
      const int u = pos * kDecGranule + lane;
      if (u < in.lens.cnt) n_next = k_idx ? __ldcg(k_idx + ((long long)in.s * P.n_kv + in.kv) * P.budget_cap + u) : u;
      else if (u < in.lens.cnt + P.chunk) n_next = in.lens.T + (u - in.lens.cnt);
    }
    pos += WARPS;
  };
  int s_at = -1, kv_at = -1;
  const auto locate = [&]() {
    live = live_next;
    if (!live) return;
    run = run_next; first = first_next; s_fill = s_next; kv_fill = kv_next;
    int t = n_next;
#ifdef QUOKA_DEBUG
    if (t < -1 || t >= __ldg(P.ctx_len + s_next) + P.chunk) { atomicExch(P.status, (int32_t)QUOKA_ERR_BAD_INDEX); t = -1; }
#endif
    if (s_next != s_at || kv_next != kv_at) { places.at_head(P, s_next, kv_next); s_at = s_next; kv_at = kv_next; }
    places.of(P, t, place, srow, page);
  };
  const auto fill = [&](int stage) {
    if (live) {
      const uint32_t at = ring + (uint32_t)stage * (2 * B::kTile), meta = metas + (uint32_t)stage * B::kMeta + 4 * lane;
      if (place != kNoRow) {
        const size_t word = D == 128 ? (size_t)srow * 4 : (size_t)(srow >> 1) * 4;
        cp_async_4(meta, P.k_scale + word);
        cp_async_4(meta + 128, P.v_scale + word);
      } else {
        asm volatile("st.shared.u32 [%0], %2;\n\tst.shared.u32 [%1], %2;" ::"r"(meta), "r"(meta + 128), "r"(0u) : "memory");
      }
      if (D == 64) asm volatile("st.shared.u32 [%0], %1;" ::"r"(meta + 256), "r"((srow & 1u) * 16) : "memory");
      if (run) {
        if (lane == 0) {
          fence_proxy_async_smem();                   // earlier contents of the stage were read, or written, through the generic proxy
          mbar_arrive_expect_tx(&landed[stage], 2 * B::kTile);
          int c1 = first, c3 = s_fill;
          if (P.page_size != 0) { c3 = page; c1 = first & (kPage - 1); }
          unsigned char* dst = dec_smem + ((size_t)warp * ST + stage) * (2 * B::kTile);
          tma_load_4d(dst, &tm_k, &landed[stage], 0, c1, kv_fill, c3);
          tma_load_4d(dst + B::kTile, &tm_v, &landed[stage], 0, c1, kv_fill, c3);
        }
      } else {
        constexpr int kUnit = 2 * kMxBits<FMT>;
#pragma unroll 1                                     // (few instructions: this is not the long lists' path, or it waits for memory)
        for (int i = 0; i < 8; ++i) {
          const int rv = 2 * c + (i & 1) + 8 * (i >> 1);           // keys 2 c, 2 c + 1, and 8 on, of both halves of the granule
          const uint32_t row = __shfl_sync(0xFFFFFFFFu, place, rv);
          cp_async_n<B::kVBytes>(at + B::kTile + B::place(rv, g * B::kVBytes), vc + (size_t)(row == kNoRow ? 0u : row) * kUnit + g * B::kVBytes, row != kNoRow);
          const int rk = g + 8 * (i >> 1), piece = c * B::kKBytes + 64 * (i & 1);
          const uint32_t rowk = __shfl_sync(0xFFFFFFFFu, place, rk);
          if (i % 2 < B::kKPieces)                     // (pieces 64 bytes apart: a warp asks for every sector once)
            cp_async_n<B::kKBytes>(at + B::place(rk, piece), kc + (size_t)(rowk == kNoRow ? 0u : rowk) * kUnit + piece, rowk != kNoRow);
        }
        if (lane == 0) mbar_arrive(&landed[stage]);
      }
    }
    cp_async_commit();
    locate();
    ask();
  };
  ask();
  locate();
  ask();
#pragma unroll
  for (int i = 0; i < ST; ++i) fill(i);

  uint32_t qf[NT][2 * KSTEPS];
  float qs[NT][2];                                    // to log2 units of the logits, of the rows of this lane's columns
  float o[NT][TILES][4], m[NT][2], l[NT][2], lx[NT][2];    // lx: the sum of the weights before they are rounded
  int stage = 0, s_cur = -1, kv_cur = -1, grp_cur = -1;
  uint32_t phase = 0;
  bool wide_q = false;                                // a query row has elements that fp16 does not hold beside its largest one
  for (bool again = true; again;) {
    const int first_row = part.grp * ROWS, n_rows = min(ROWS, P.chunk * P.group - first_row);
    // ---- the part's query rows
    if (part.s != s_cur || part.kv != kv_cur || part.grp != grp_cur) {
      s_cur = part.s; kv_cur = part.kv; grp_cur = part.grp;
      bool below = false;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const int row = 8 * nt + g, r = first_row + row;
        const __nv_bfloat16* qr = q + (long long)part.s * P.q_sb + (long long)(part.kv * P.group + r % P.group) * P.q_sh + (long long)(r / P.group) * P.q_st;
        uint4 w[D / 32];
        DecMagnitudes mags;
#pragma unroll
        for (int j = 0; j < D / 32; ++j) {             // 8 columns of the lane's D / 4
          w[j] = make_uint4(0, 0, 0, 0);
          if (row < n_rows) w[j] = load_input<true>(reinterpret_cast<const uint4*>(qr + dec_column<FMT, D>(c, j)));
          const uint32_t x[4] = {w[j].x, w[j].y, w[j].z, w[j].w};
#pragma unroll
          for (int i = 0; i < 4; ++i) mags.take(x[i]);
        }
        uint32_t top = mags.largest();
        top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
        top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
        const int up = min(14 + 127 - (int)(top >> 23), 120);          // (an element that is not finite stays so)
        below |= mags.below_f16(up);
        const float f = __uint_as_float((uint32_t)(127 + up) << 23), back = __uint_as_float((uint32_t)(127 - up) << 23);
#pragma unroll
        for (int j = 0; j < D / 32; ++j) {
          const uint32_t x[4] = {w[j].x, w[j].y, w[j].z, w[j].w};
#pragma unroll
          for (int i = 0; i < 4; ++i) qf[nt][4 * j + i] = f16x2(__uint_as_float(x[i] << 16) * f, __uint_as_float(x[i] & 0xFFFF0000u) * f);
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) qs[nt][e] = __shfl_sync(0xFFFFFFFFu, back, 4 * (2 * c + e)) * (P.scale * 1.4426950408889634f);
      }
      wide_q = __any_sync(0xFFFFFFFFu, below);
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int e = 0; e < 2; ++e) { m[nt][e] = -INFINITY; l[nt][e] = lx[nt][e] = 0.f; }
#pragma unroll
      for (int t = 0; t < TILES; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[nt][t][e] = 0.f;
    }
    // Scale bytes of this lane's columns (all of one block of 32): O's; one less than the smallest of a block of values so far, and the
    // largest that neither minds, in both halves of a word; whether blocks of values have differed too much for fp16 (in some lane).
    int ov = 0;
    uint32_t least = 0xFFFFFFFFu, passed = 0u;
    bool wide_v = false;
    const int v_shift = 8 * (D == 128 ? g >> 1 : g >> 2);
    int nan_u = kNoNan;                                // first key, in the order of visibility, with a value that is not finite in this lane's columns
    // keys that the rows of this lane's columns see: 2 c and 2 c + 1 of each tile
    int sees[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int e = 0; e < 2; ++e) sees[nt][e] = part.lens.cnt + min(first_row + 8 * nt + 2 * c + e, P.chunk * P.group - 1) / P.group + 1;
    const int all_see = part.lens.cnt + first_row / P.group + 1;       // keys that every row sees
#pragma unroll 1
    for (int gr = part.begin + warp; gr < part.end; gr += WARPS) {
      cp_async_wait<ST - 1>();
      if (!mbar_wait_done(&landed[stage], phase, wc)) break;
      __syncwarp();
      const uint32_t at = ring + (uint32_t)stage * (2 * B::kTile), meta = metas + (uint32_t)stage * B::kMeta;
      // scale bytes of the i-th row's keys (0) or values (128)
      const auto scale_word = [&](int what, int i) {
        uint32_t w;
        asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w) : "r"(meta + what + 4 * i) : "memory");
        if (D == 64) {
          uint32_t shift;
          asm volatile("ld.shared.u32 %0, [%1];" : "=r"(shift) : "r"(meta + 256 + 4 * i) : "memory");
          w = w >> shift & 0xFFFFu;
        }
        return w;
      };
      // ---- scale bytes of the lane's eight values in its block of columns, two to a word
      uint32_t ve[4], ve_most = passed, ve_low = least;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t e0 = scale_word(128, 2 * c + 8 * i) >> v_shift & 0xFFu, e1 = scale_word(128, 2 * c + 1 + 8 * i) >> v_shift & 0xFFu;
        ve[i] = e0 | e1 << 16;
        ve_most = __vmaxu2(ve_most, ve[i]);
        ve_low = __viaddmin_u16x2(ve[i], 0xFFFFFFFFu, ve_low);         // (one less: a row that is not there has 0, and does not count)
      }
      const bool values_met = ve_most == passed && ve_low == least;
      // ---- S^T = K Q^T, 16 keys at a time
      float sc[2][NT][4];
      DecFactors factors;
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 4; ++e) sc[h][nt][e] = 0.f;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint32_t w[2][KW], f[2][B::kKPieces];
        float key[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
#pragma unroll
          for (int p = 0; p < B::kKPieces; ++p)
            lds_words<B::kKBytes / 4>(at + B::place(g + 16 * h + 8 * i, c * B::kKBytes + 64 * p), w[i] + p * (B::kKBytes / 4));
          const uint32_t sw = scale_word(0, g + 16 * h + 8 * i);
          uint32_t top = __vmaxu4(sw, sw >> 16);       // the largest of the row's scale bytes (head_dim 64: of two)
          top = max(top & 0xFFu, top >> 8 & 0xFFu);
          key[i] = mx_scale(top);                      // (NaN where a block is not finite)
          // the lane's block(s): 32 columns from c * D / 4 on, two of 16 columns at 8 bits and head_dim 128
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
          for (int i = 0; i < N / 2; ++i)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
              mma_f16(sc[h][nt], a[2 * i], b[2 * i], a[2 * i + 1], b[2 * i + 1], qf[nt][N * j + 2 * i], qf[nt][N * j + 2 * i + 1]);
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 4; ++e) sc[h][nt][e] *= key[e >> 1] * qs[nt][e & 1];
      }
      // ---- softmax: a lane has keys g, g + 8, g + 16, g + 24 of rows 2 c and 2 c + 1; logits in log2 units
      const int u0 = gr * kDecGranule;
      float top[NT][2];
      const auto see = [&]() {                          // masks, maxima; whether the reference point of the exponentials is set, or moves
        if (u0 + kDecGranule > all_see) {
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (u0 + 16 * h + g + 8 * (e >> 1) >= sees[nt][e & 1]) sc[h][nt][e] = -INFINITY;
        }
        bool grow = false;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            top[nt][e] = fmaxf(fmaxf(sc[0][nt][e], sc[0][nt][e + 2]), fmaxf(sc[1][nt][e], sc[1][nt][e + 2]));
            grow |= top[nt][e] > m[nt][e] + (float)kDecMaxAbove;
          }
        return grow;
      };
      // ---- do fp16 operands hold the granule, and the reference point: one vote, rarely with something to do
      const bool keys_below = factors.below_f16<FMT>() || wide_q;
      bool grow = see();
      if (__builtin_expect(__any_sync(0xFFFFFFFFu, grow || keys_below || !values_met), 0)) {
        if (__any_sync(0xFFFFFFFFu, !values_met)) {
          int most = 0, low = (int)(ve_low & 0xFFFFu) + 1;
          low = min(low, (int)(ve_low >> 16) + 1);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const uint32_t e = ve[i / 2] >> (16 * (i & 1)) & 0xFFFFu;
            if (e == kMxNanScale) {                     // a block that is not finite counts as zeros, who sees it is told by nan_u
              nan_u = min(nan_u, u0 + 2 * c + (i & 1) + 8 * (i >> 1));
              ve[i / 2] &= i & 1 ? 0xFFFFu : 0xFFFF0000u;
            } else {
              most = max(most, (int)e);
            }
          }
#pragma unroll
          for (int sh = 1; sh < 4; sh <<= 1) {
            most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, sh));
            low = min(low, __shfl_xor_sync(0xFFFFFFFFu, low, sh));
          }
          wide_v |= __any_sync(0xFFFFFFFFu, max(most, ov) > low + kDecValueWindow) != 0;
          if (most > ov + kDecScaleAbove || ov == 0) {  // O's scale is set, or moves
            if (ov != 0) {
              const float down = pow2_at_most_15(ov - most);
#pragma unroll
              for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int t = 0; t < TILES; ++t)
#pragma unroll
                  for (int i = 0; i < 4; ++i) o[nt][t][i] *= down;
            }
            ov = max(most, 1);
          }
          // (where they have differed too much already, only what O's scale minds)
          least = (wide_v ? 0u : (uint32_t)(low - 1)) * 0x10001u;
          passed = (uint32_t)(wide_v ? ov + kDecScaleAbove : min(ov + kDecScaleAbove, low + kDecValueWindow)) * 0x10001u;
        }
        if (__builtin_expect(__any_sync(0xFFFFFFFFu, keys_below), 0)) {
          if (wide_q || __any_sync(0xFFFFFFFFu, dec_key_below_f16<FMT, D>(at, lane, scale_word(0, lane)))) {       // the scores anew, of the values themselves
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
              for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) sc[h][nt][e] = 0.f;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              uint32_t sw[2];
              float none[4];
#pragma unroll
              for (int i = 0; i < 2; ++i) sw[i] = scale_word(0, g + 16 * h + 8 * i);
              dec_scores_bf16<FMT, D, NT, false>(at, g + 16 * h, c, sw, [&](int nt, int j) {
                const int r = first_row + 8 * nt + g;
                if (8 * nt + g >= n_rows) return make_uint4(0, 0, 0, 0);
                return load_input<true>(reinterpret_cast<const uint4*>(q + (long long)part.s * P.q_sb + (long long)(part.kv * P.group + r % P.group) * P.q_sh +
                                                                       (long long)(r / P.group) * P.q_st + dec_column<FMT, D>(c, j)));
              }, sc[h], none, none);
#pragma unroll
              for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) sc[h][nt][e] *= P.scale * 1.4426950408889634f;
            }
            grow = see();
          }
        }
        if (__any_sync(0xFFFFFFFFu, grow)) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float mx = top[nt][e];
#pragma unroll
            for (int sh = 4; sh < 32; sh <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, sh));
            mx = fmaxf(m[nt][e], mx - (float)kDecHeadroom);
            const float alpha = m[nt][e] == mx ? 1.f : ex2(m[nt][e] - mx);
            m[nt][e] = mx;
            l[nt][e] *= alpha;
            lx[nt][e] *= alpha;
#pragma unroll
            for (int t = 0; t < TILES; ++t) { o[nt][t][e] *= alpha; o[nt][t][e + 2] *= alpha; }
          }
        }
      }
      // ---- weights, and O^T += V^T P^T, on fp16 operands or bf16 ones
      const auto weigh = [&](auto is_wide) {
        constexpr bool WIDE = decltype(is_wide)::value;
        const auto pairs = [](uint32_t w, uint32_t factor2, auto& x) { if constexpr (WIDE) bf16_pairs<FMT>(w, factor2, x); else f16_pairs<FMT>(w, factor2, x); };
        const auto mma = [](float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
          if constexpr (WIDE) mma_bf16(d, a0, a1, a2, a3, b0, b1); else mma_f16(d, a0, a1, a2, a3, b0, b1);
        };
        uint32_t pf[2][NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const float m0 = m[nt][0] == -INFINITY ? 0.f : m[nt][0], m1 = m[nt][1] == -INFINITY ? 0.f : m[nt][1];
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const float p0 = ex2(sc[h][nt][2 * i] - m0), p1 = ex2(sc[h][nt][2 * i + 1] - m1);
              const uint32_t w = WIDE ? bf16x2(p0, p1) : f16x2(p0, p1);
              const float2 back = WIDE ? make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)) : __half22float2(*reinterpret_cast<const __half2*>(&w));
              lx[nt][0] += p0;
              lx[nt][1] += p1;
              l[nt][0] += back.x;
              l[nt][1] += back.y;
              pf[h][nt][i] = transpose8x8(w);
            }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t f[2], v[4][VW];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            // 2^(e - ov) of both: exponent fields (zero for what is not there, and elements of zero)
            const int bias = (WIDE ? 127 : 15) - ov;
            f[i] = (uint32_t)__viaddmax_s16x2_relu(ve[2 * h + i], ((uint32_t)bias & 0xFFFFu) * 0x10001u, 0u) << (WIDE ? 7 : 10);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) lds_words<VW>(at + B::kTile + B::place(16 * h + 2 * c + (i & 1) + 8 * (i >> 1), g * B::kVBytes), v[i]);
#pragma unroll
          for (int w = 0; w < VW; ++w) {
            // the word's columns, the rows of a pair side by side: x those of keys 2 c and 2 c + 1, y 8 on
            if constexpr (FMT == QUOKA_KV_MXFP8) {
#pragma unroll
              for (int half = 0; half < 2; ++half) {
                uint32_t x[2], y[2];
                pairs(__byte_perm(v[0][w], v[1][w], half ? 0x7362 : 0x5140), f[0], x);
                pairs(__byte_perm(v[2][w], v[3][w], half ? 0x7362 : 0x5140), f[1], y);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) mma(o[nt][2 * w + half], x[0], x[1], y[0], y[1], pf[h][nt][0], pf[h][nt][1]);
              }
            } else {
              constexpr uint32_t kLow = 0x0F0F0F0Fu;
              uint32_t x0[4], x1[4], y0[4], y1[4];        // even columns, odd columns
              pairs((v[0][w] & kLow) | (v[1][w] << 4 & ~kLow), f[0], x0);
              pairs((v[0][w] >> 4 & kLow) | (v[1][w] & ~kLow), f[0], x1);
              pairs((v[2][w] & kLow) | (v[3][w] << 4 & ~kLow), f[1], y0);
              pairs((v[2][w] >> 4 & kLow) | (v[3][w] & ~kLow), f[1], y1);
#pragma unroll
              for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) mma(o[nt][4 * w + i], x0[i], x1[i], y0[i], y1[i], pf[h][nt][0], pf[h][nt][1]);
            }
          }
        }
      };
      if (__builtin_expect(!wide_v, 1)) weigh(std::false_type{}); else weigh(std::true_type{});
      __syncwarp();                                    // the scale words of this stage have been read
      fill(stage);
      if (++stage == ST) { stage = 0; phase ^= 1; }
    }
    // ---- the warps' results of this part
    nan_u = min(nan_u, __shfl_xor_sync(0xFFFFFFFFu, nan_u, 1));
    nan_u = min(nan_u, __shfl_xor_sync(0xFFFFFFFFu, nan_u, 2));
    const float ov_scale = mx_scale((uint32_t)ov);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
#pragma unroll
        for (int sh = 4; sh < 32; sh <<= 1) {
          l[nt][e] += __shfl_xor_sync(0xFFFFFFFFu, l[nt][e], sh);
          lx[nt][e] += __shfl_xor_sync(0xFFFFFFFFu, lx[nt][e], sh);
        }
        const bool bad = nan_u < sees[nt][e];
#pragma unroll
        for (int t = 0; t < TILES; ++t)
#pragma unroll
          for (int i = 0; i < 2; ++i) o[nt][t][e + 2 * i] = bad ? __uint_as_float(0x7FC00000u) : o[nt][t][e + 2 * i] * ov_scale;
      }
    __syncthreads();                                   // (the buffer's last part has been read)
    if constexpr (WARPS > LAST) {                      // warp w + LAST's to warp w, lane by lane
      constexpr int kValues = NT * 4 * TILES;
      static_assert(kValues * 32 <= ROWS * LD, "what a warp's rows take below");
      float* hand = merge + (warp % LAST) * (kValues * 32) + lane;
      float* hand_ml = merge_ml + warp % LAST * ROWS + 2 * c;
      if (warp >= LAST) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          if (g == 0) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              hand_ml[8 * nt + e] = m[nt][e]; hand_ml[LAST * ROWS + 8 * nt + e] = l[nt][e]; hand_ml[2 * LAST * ROWS + 8 * nt + e] = lx[nt][e];
            }
          }
#pragma unroll
          for (int t = 0; t < TILES; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) hand[((nt * TILES + t) * 4 + e) * 32] = o[nt][t][e];
        }
      }
      __syncthreads();
      if (warp < LAST) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float other = hand_ml[8 * nt + e], mx = fmaxf(m[nt][e], other), w0 = dec_weight(m[nt][e], mx), w1 = dec_weight(other, mx);
            m[nt][e] = mx;
            l[nt][e] = fmaf(w1, hand_ml[LAST * ROWS + 8 * nt + e], w0 * l[nt][e]);
            lx[nt][e] = fmaf(w1, hand_ml[2 * LAST * ROWS + 8 * nt + e], w0 * lx[nt][e]);
#pragma unroll
            for (int t = 0; t < TILES; ++t)
#pragma unroll
              for (int i = 0; i < 2; ++i) o[nt][t][e + 2 * i] = fmaf(w1, hand[((nt * TILES + t) * 4 + e + 2 * i) * 32], w0 * o[nt][t][e + 2 * i]);
          }
      }
      __syncthreads();
    }
    if (warp < LAST) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int row = 8 * nt + 2 * c + e;
          if (g == 0) { merge_ml[warp * ROWS + row] = m[nt][e]; merge_ml[(LAST + warp) * ROWS + row] = l[nt][e]; merge_ml[(2 * LAST + warp) * ROWS + row] = lx[nt][e]; }
          float2* to = reinterpret_cast<float2*>(merge + (warp * ROWS + row) * LD + g * (D / 8));
#pragma unroll
          for (int t = 0; t < TILES; ++t) to[t] = make_float2(o[nt][t][e], o[nt][t][e + 2]);
        }
    }
    __syncthreads();
    const auto store = [&](int row, int col, const float4& acc, float mx, float sum, float sumx) {
      const int r = first_row + row, h = part.kv * P.group + r % P.group, pos_r = r / P.group;
      const float inv = 1.f / sum;
      const __nv_bfloat162 a = __floats2bfloat162_rn(acc.x * inv, acc.y * inv), b = __floats2bfloat162_rn(acc.z * inv, acc.w * inv);
      *reinterpret_cast<uint2*>(out + (long long)part.s * P.o_sb + (long long)h * P.o_sh + (long long)pos_r * P.o_st + col) =
          make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
      if (lse && col == 0) lse[((long long)part.s * P.n_q + h) * P.chunk + pos_r] = (mx + log2f(sumx)) * 0.6931471805599453f;
    };
    const bool is_whole = per_unit <= 1 && part.begin == 0 && part.end == part.n;
    const int slot = blockIdx.x * 2 + (part.begin == 0 ? 1 : 0);
    for (int i = threadIdx.x; i < n_rows * (D / 4); i += 32 * WARPS) {
      const int row = i / (D / 4), col = i % (D / 4) * 4;
      float mx = -INFINITY;
#pragma unroll
      for (int w = 0; w < LAST; ++w) mx = fmaxf(mx, merge_ml[w * ROWS + row]);
      float sum = 0.f, sumx = 0.f;
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < LAST; ++w) {
        const float wt = dec_weight(merge_ml[w * ROWS + row], mx);
        const float4 v = *reinterpret_cast<const float4*>(merge + (w * ROWS + row) * LD + col);
        sum = fmaf(wt, merge_ml[(LAST + w) * ROWS + row], sum);
        sumx = fmaf(wt, merge_ml[(2 * LAST + w) * ROWS + row], sumx);
        acc.x = fmaf(wt, v.x, acc.x); acc.y = fmaf(wt, v.y, acc.y); acc.z = fmaf(wt, v.z, acc.z); acc.w = fmaf(wt, v.w, acc.w);
      }
      if (is_whole) {
        store(row, col, acc, mx, sum, sumx);
      } else {
        float* to = per_unit > 1 ? reinterpret_cast<float*>(dec_smem) : parts + (size_t)slot * ROWS * (D + 3);        // (the rings are empty by then)
        *reinterpret_cast<float4*>(to + row * D + col) = acc;
        if (col == 0) { to[ROWS * D + row] = mx; to[ROWS * (D + 1) + row] = sum; to[ROWS * (D + 2) + row] = sumx; }
      }
    }
    if (per_unit > 1) {                                // one part: the cluster's are added up, in order, each CTA a share of the outputs
      cluster_sync_all();
      const uint32_t mine = smem_u32(dec_smem);
      const int rank = blockIdx.x % per_unit, items = n_rows * (D / 4);
      for (int i = rank + per_unit * (int)threadIdx.x; i < items; i += per_unit * 32 * WARPS) {
        const int row = i / (D / 4), col = i % (D / 4) * 4;
        float mx = -INFINITY, sum = 0.f, sumx = 0.f;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
        for (int p0 = 0; p0 < per_unit; p0 += kDecAtOnce) {
          float pm[kDecAtOnce], pl[kDecAtOnce], plx[kDecAtOnce];
          float4 v[kDecAtOnce];
#pragma unroll
          for (int j = 0; j < kDecAtOnce; ++j) {
            const uint32_t from = map_to_cta(mine, (uint32_t)min(p0 + j, per_unit - 1));
            v[j] = ld_cluster_f4(from + 4u * (uint32_t)(row * D + col));
            pm[j] = ld_cluster_f(from + 4u * (uint32_t)(ROWS * D + row));
            pl[j] = ld_cluster_f(from + 4u * (uint32_t)(ROWS * (D + 1) + row));
            plx[j] = ld_cluster_f(from + 4u * (uint32_t)(ROWS * (D + 2) + row));
          }
#pragma unroll
          for (int j = 0; j < kDecAtOnce; ++j)
            if (p0 + j < per_unit) {
              const float top = fmaxf(mx, pm[j]), w0 = dec_weight(mx, top), w1 = dec_weight(pm[j], top);
              mx = top;
              sum = fmaf(w1, pl[j], sum * w0);
              sumx = fmaf(w1, plx[j], sumx * w0);
              acc.x = fmaf(w1, v[j].x, acc.x * w0); acc.y = fmaf(w1, v[j].y, acc.y * w0); acc.z = fmaf(w1, v[j].z, acc.z * w0); acc.w = fmaf(w1, v[j].w, acc.w * w0);
            }
        }
        store(row, col, acc, mx, sum, sumx);
      }
      cluster_sync_all();                              // (nobody leaves while its shared memory is read)
    }
    again = part.next(P, work);
  }
  cp_async_wait_all();                                 // nothing of this thread is in flight at exit
}

// Units that several CTAs of the list share, a CTA per query row: its warps take parts in turn, all loads of a warp's parts at once as a rule
// (a loop over the parts by one warp took 15 us for 20 of them), and add them up in a fixed order.
constexpr int kJoinWarps = 4, kJoinAtOnce = 6;
template <int D, int NT>
__global__ void __launch_bounds__(32 * kJoinWarps) decode_mx_join_kernel(DevParams P, DecWork work, const float* __restrict__ parts, int ctas,
                                                                         __nv_bfloat16* __restrict__ out, float* __restrict__ lse) {
  constexpr int ROWS = 8 * NT, PER = D / 32;
  __shared__ float sm[kJoinWarps][3], so[kJoinWarps][D];
  grid_dependency_wait();
  grid_launch_dependents();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, unit = blockIdx.x, per_s = P.n_kv * work.groups, s = unit / per_s;
  const int row = blockIdx.y, r = unit % work.groups * ROWS + row;
  if (r >= P.chunk * P.group) return;
  const DecTotals all(P, work, s, lane);
  const int n = DecLens(P, work, s).granules(work);
  const long long each = all.share(ctas), a = all.before + (long long)(unit % per_s) * n;
  const int first = dec_div(a, each), last = dec_div(a + n - 1, each);
  if (first == last) return;                           // (written by that CTA)
  const auto slot = [&](int i) { return parts + (size_t)(2 * i + (i == first ? 1 : 0)) * ROWS * (D + 3); };
  float mx = -INFINITY, sum = 0.f, sumx = 0.f, acc[PER];
#pragma unroll
  for (int e = 0; e < PER; ++e) acc[e] = 0.f;
  for (int i0 = first + warp; i0 <= last; i0 += kJoinWarps * kJoinAtOnce) {
    float m[kJoinAtOnce], l[kJoinAtOnce], lx[kJoinAtOnce], v[kJoinAtOnce][PER];
#pragma unroll
    for (int j = 0; j < kJoinAtOnce; ++j) {
      const float* p = slot(min(i0 + j * kJoinWarps, last));
      m[j] = __ldcg(p + ROWS * D + row);
      l[j] = __ldcg(p + ROWS * (D + 1) + row);
      lx[j] = __ldcg(p + ROWS * (D + 2) + row);
      load_vec<float, PER, true>(p + row * D + lane * PER, v[j]);
    }
#pragma unroll
    for (int j = 0; j < kJoinAtOnce; ++j)
      if (i0 + j * kJoinWarps <= last) {
        const float top = fmaxf(mx, m[j]), w0 = dec_weight(mx, top), w1 = dec_weight(m[j], top);
        mx = top;
        sum = fmaf(w1, l[j], sum * w0);
        sumx = fmaf(w1, lx[j], sumx * w0);
#pragma unroll
        for (int e = 0; e < PER; ++e) acc[e] = fmaf(w1, v[j][e], acc[e] * w0);
      }
  }
  if (lane == 0) { sm[warp][0] = mx; sm[warp][1] = sum; sm[warp][2] = sumx; }
#pragma unroll
  for (int e = 0; e < PER; ++e) so[warp][lane * PER + e] = acc[e];
  __syncthreads();
  const int h = unit % per_s / work.groups * P.group + r % P.group, pos = r / P.group;
  for (int col = threadIdx.x; col < D; col += 32 * kJoinWarps) {
    float top = sm[0][0], total = 0.f, totalx = 0.f, o = 0.f;
#pragma unroll
    for (int w = 1; w < kJoinWarps; ++w) top = fmaxf(top, sm[w][0]);
#pragma unroll
    for (int w = 0; w < kJoinWarps; ++w) {
      const float wt = dec_weight(sm[w][0], top);
      total = fmaf(wt, sm[w][1], total);
      totalx = fmaf(wt, sm[w][2], totalx);
      o = fmaf(wt, so[w][col], o);
    }
    out[(long long)s * P.o_sb + (long long)h * P.o_sh + (long long)pos * P.o_st + col] = __float2bfloat16_rn(o / total);
    if (lse && col == 0) lse[((long long)s * P.n_q + h) * P.chunk + pos] = (top + log2f(totalx)) * 0.6931471805599453f;
  }
}

// ---------------------------------------------------------------------------------------------- host
// Tiles of 8 query rows that a warp takes at once: what its registers hold of O (16 or 32 a tile); at head_dim 64 up to 40 rows, so that
// the cache is read once.
static int dec_tiles(int rows, int d) {
  const int tiles = (rows + 7) / 8;
  if (d == 128) return tiles == 1 ? 1 : 2;
  return tiles <= 3 ? tiles : 5;
}

// Query rows that these kernels take: more of them are faster in a 128-row tile of the tensor-core kernel, though it walks 128 keys for every
// 1.0 to 1.4 us and cuts them into 8 parts at most.  These / those, us: d 128, 20 to 32 rows over 32768 keys 46 / 83, over 4003 18.4 / 22.6, over 8 sequences of
// 8192 80 / 78; d 64, 40 rows over 3 sequences of 20011 42 / 45, 64 rows 64 / 44.  One sequence of 20011, d 64, MXFP8, 4 KV heads: 16 / 24 / 32 / 40 rows 26.7 / 28.9 /
// 36.6 / 37.0 here (32 rows as the five tiles of 40), 48 rows in the tensor-core kernel 49.
bool decode_mx_applies(const quoka_params* p) {
  const long long rows = (long long)p->chunk_len * (p->n_q_heads / p->n_kv_heads);
  return p->chunk_len == 1 || rows <= (p->head_dim == 64 ? 40 : 32);
}

// Parts of the shared units: two slots a CTA, one CTA per SM.
size_t decode_mx_scratch_bytes(const quoka_params* p) {
  const int sms = device_sm_count() > 0 ? device_sm_count() : 148;
  return (size_t)sms * 2 * (p->head_dim == 64 ? 40 : 16) * (p->head_dim + 3) * sizeof(float);
}

constexpr int kDecWhole = 24;                          // granules that a CTA takes alone
// The largest cluster of up to 16 CTAs of which `units` are resident at once (1: none): a property of the device and the kernel, asked for once.
template <int FMT, int D, int NT>
static int largest_cluster(long long units, size_t smem) {
  constexpr int kMost = 16, kDevices = 64;
  static std::atomic<int> resident[kDevices][kMost + 1];       // + 1
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kDevices) return 1;
  for (int cl = (int)std::min<long long>(kMost, device_sm_count() / units); cl > 1; --cl) {
    int n = resident[dev][cl].load(std::memory_order_relaxed);
    if (n == 0) {
      const auto kernel = decode_mx_kernel<FMT, D, NT>;
      cudaLaunchConfig_t cfg = {};
      cfg.gridDim = dim3((unsigned)cl);
      cfg.blockDim = dim3(32 * kDecWarps<NT>);
      cfg.dynamicSmemBytes = smem;
      cudaLaunchAttribute attr;
      attr.id = cudaLaunchAttributeClusterDimension;
      attr.val.clusterDim.x = (unsigned)cl;
      attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
      cfg.attrs = &attr;
      cfg.numAttrs = 1;
      if (cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess || cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess) {
        cudaGetLastError();
        n = 0;
      }
      resident[dev][cl].store(++n, std::memory_order_relaxed);
    }
    if (n > units) return cl;
  }
  return 1;
}

template <int FMT, int D, int NT>
static cudaError_t launch_decode_mx_t(const DevParams& P, const void* q, const void* k, const void* v, const int32_t* k_idx, const int32_t* k_cnt, void* out,
                                      float* lse, float* parts, cudaStream_t st, bool chained) {
  constexpr int WARPS = kDecWarps<NT>, ROWS = 8 * NT;
  DecWork work;
  work.groups = (P.chunk * P.group + ROWS - 1) / ROWS;
  work.own = P.chunk;
  work.k_cnt = k_idx ? k_cnt : nullptr;
  const int sms = device_sm_count();
  if (sms <= 0) return cudaErrorInvalidDevice;
  const long long units = (long long)P.batch * P.n_kv * work.groups;
  const long long most = ((k_idx ? (long long)P.budget_cap : (long long)P.max_ctx) + P.chunk + kDecGranule - 1) / kDecGranule;      // granules of a unit
  const size_t smem = 1024 + (size_t)WARPS * kDecStages * (DecBytes<FMT, D>::kStage + 8) + (size_t)kDecLast<NT> * ROWS * (D + 4 + 3) * sizeof(float);
  cudaError_t e = cudaFuncSetAttribute(decode_mx_kernel<FMT, D, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  // How units are shared, us of one sequence, 8 KV heads, d 128, one position of 4 heads, MXFP8, over 300 / 700 / 1000 / 1500 / 2000 / 4003 / 8192 / 16384 / 32768 rows:
  //   a CTA per unit       9.0 / 12.3 / 12.8 / 16.4 / 18.5
  //   a cluster per unit   1000 rows on: 12.3 / 12.3 / 12.3 / 14.4 / 16.4 / 20.5 / 28.7 (of 10 CTAs: on a B200 seven clusters of 11 to 16 are resident, 11 of 10)
  //   one list             16.4 to 4003 rows / 20.5 / 22.9 / 28.7: joining parts costs a launch and a round trip through L2, some 3 rounds of the warps
  // so a CTA to 24 granules (four positions over 700 rows: 14.4 alone, 16.4 in clusters), then clusters where they take 3 rounds more than the list at
  // most, which takes what its longest sequence needs or more: sequences of a batch may differ, and their clusters do not help each other.  (8
  // sequences of 1500 rows: 14.4, as a list 20.5; two of 9393 rows 20.5 / 23.7, of 9393 and 100 20.5 / 22.6.)
  // No clusters: a CTA to 4 rounds (the same 8 sequences 16.4), or where units are many.
  int per_unit = most <= kDecWhole || units >= 64ll * sms ? 1 : 0;
  if (per_unit == 0) {
    const int cl = largest_cluster<FMT, D, NT>(units, smem);
    const auto rounds = [&](long long granules, long long over) { return (granules + over * WARPS - 1) / (over * WARPS); };
    if (cl > 1 && rounds(most, cl) <= 3 + rounds(units / P.batch * most, sms)) per_unit = cl;
    else if (most <= 4 * WARPS) per_unit = 1;
  }
  const long long ctas = per_unit > 0 ? units * per_unit : std::min<long long>(sms, (units * most + WARPS - 1) / WARPS);
  if (ctas > 0x7FFFFFFFll) return cudaErrorInvalidConfiguration;
  CUtensorMap tm_k, tm_v;
  if (!encode_mx_tile_map(&tm_k, P, FMT, k, kDecGranule) || !encode_mx_tile_map(&tm_v, P, FMT, v, kDecGranule)) return cudaErrorInvalidValue;
  e = launch_kernel("decode_mx", decode_mx_kernel<FMT, D, NT>, dim3((unsigned)ctas), dim3(32 * WARPS), smem, st, std::max(per_unit, 1), chained, P, work, (const __nv_bfloat16*)q,
                    (const uint8_t*)k, (const uint8_t*)v, k_idx, (__nv_bfloat16*)out, lse, parts, per_unit, tm_k, tm_v);
  if (e != cudaSuccess) return e;
  count_launch();
  if (per_unit == 0) {
    e = launch_kernel("decode_mx_join", decode_mx_join_kernel<D, NT>, dim3((unsigned)units, ROWS), dim3(32 * kJoinWarps), 0, st, 1, true, P, work, (const float*)parts, (int)ctas,
                      (__nv_bfloat16*)out, lse);
    if (e != cudaSuccess) return e;
    count_launch();
  }
  return cudaGetLastError();
}

cudaError_t launch_decode_mx(const DevParams& P, int fmt, const void* q, const void* k, const void* v, const int32_t* k_idx, const int32_t* k_cnt, void* out,
                             float* lse, float* parts, cudaStream_t st, bool chained) {
  const int tiles = dec_tiles(P.chunk * P.group, P.d);
  return mx_dispatch(QUOKA_BF16, fmt, P.d, [&](auto, auto f, auto d) {
    constexpr int FMT = decltype(f)::value, D = decltype(d)::value;
    if (tiles == 1) return launch_decode_mx_t<FMT, D, 1>(P, q, k, v, k_idx, k_cnt, out, lse, parts, st, chained);
    if (tiles == 2) return launch_decode_mx_t<FMT, D, 2>(P, q, k, v, k_idx, k_cnt, out, lse, parts, st, chained);
    if constexpr (D == 64) {
      if (tiles == 3) return launch_decode_mx_t<FMT, D, 3>(P, q, k, v, k_idx, k_cnt, out, lse, parts, st, chained);
      return launch_decode_mx_t<FMT, D, 5>(P, q, k, v, k_idx, k_cnt, out, lse, parts, st, chained);
    }
    return cudaErrorInvalidValue;
  });
}

}  // namespace quoka
