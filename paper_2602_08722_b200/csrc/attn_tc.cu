// The plan and the launches of the tensor-core attention kernels (attn_tc.cuh, attn_tc_pair.cuh).
#include <algorithm>
#include <cmath>

#include "attn_tc.cuh"

namespace quoka {

// How an attention call is laid out on the GPU: the form of its row blocks, and parts of their key tiles.
//
// Forms: two Q tiles per CTA or one; at head_dim 128 a row block is that of a pair of CTAs or of one.  A pair's step (a key tile)
// is the faster one per row, one CTA's row blocks are smaller: chunks of a few positions, or few heads per KV head, leave
// a pair with CTAs or tiles without rows.
// Parts: a grid of fewer CTAs than SMs (short chunks, few heads) leaves part of the GPU idle while every CTA walks its whole
// key sequence; cutting each row block's tiles into parts, one CTA (pair) each, fills it.  Parts merge through memory, or,
// a pair's, in a cluster of 2 * parts CTAs where all of a grid's clusters are resident at once: the device holds 33, 22 or 15
// of 4, 6 or 8 CTAs of this shared memory, the limits leave some free (a second wave costs more than any split gives).
//
// The model, in microseconds: start and end of a CTA, its steps, and what parts cost on top; the parts of a sparse call start
// only when the selection has ended, whole row blocks walk the chunk's own tiles under it (half of these count).  Measured with
// one thing varied at a time, a step with one / two Q tiles: a pair 1.09 / 1.39 us (listed rows 1.25 / 1.45), one CTA at head_dim
// 128 1.02 / 1.91 (1.41 / 1.93: it gathers whole rows of its own), at head_dim 64 1.02 / 1.38 (1.13 / 1.42); parts through memory
// 9 us for two and 20 for eight, at head_dim 64 8 and 12; in a cluster 3 to 6.  Then moved, most by less than a tenth, to fit
// whole calls: 284 of them, 1 to 8 sequences, 5 to 32 heads, chunks of 16 to 3238, 2 to 516 tiles, each with every form
// and number of parts (5000 times).  The plan's choice takes 0.8 % more time than the best form in the geometric mean; pairs
// only and the same cost of parts for both head dims took 2 % (25 % at most).  For instance, this choice / the one
// before, us: dense, 8 heads of 8 KV heads, 1100 queries over 8192 rows 56 (one CTA, one tile, 2 parts) / 60 (pairs); 32 heads of 8,
// 128 over 8192 38 / 45; 32 heads of 32, 64 over 32768 96 / 176; sparse, 8 heads of 8, 1100 queries, 983 of 8192 rows 48 (pairs,
// one tile, whole) / 55 (two tiles, clusters of two parts).
//
// A grid of q full waves and a rest has its lightest row blocks, as many as the rest, cut instead: the whole ones then
// end after about q waves and the parts level the end.  The model is the total work over the SMs plus a third of a part
// for the uneven end, against q + 1 waves of average jobs.  48 calls without / with parts, in turns over the same buffers: what
// the model puts below 0.92 of the whole row blocks (sparse) and 0.94 (dense) gains 1 to 11 %,
// around the line some gain 5 % and some lose 7, above it nearly all lose 4 to 10.  32 heads, us, and the model: sparse, 3700 queries
// over 8192 of 65536 rows 621 / 561 (0.82), 1550 over 3932 of 32768 165 / 154 (0.86), 2900 over 8192 415 / 404 (0.91), 4096 over
// 15729 of 131072 1132 / 1086 (0.91), 1700 over 3932 168 / 182 (0.925), 3072 over 16384 828 / 784 (0.93), 1850 over 8192 270 / 287 (0.95), 2000
// over 8192 276 / 297 (1.01); head_dim 64 3800 over 3932 304 / 284 (0.85), 1850 over 8192 243 / 228 (0.91), 2000 over 8192 246 / 260 (0.99);
// dense, 1850 over 16384 411 / 392 (0.91), 3000 over 32768 1444 / 1331 (0.91), 2048 over 32768 967 / 914 (0.94), 1850 over 8192 217 / 241
// (0.95), 2150 over 32768 945 / 1002 (1.00); head_dim 64 2000 over 32768 746 / 682 (0.92), 3050 over 8192 331 / 344 (0.95).  Sparse
// calls of a batch stay whole (their budgets differ).
// Partial results above 128 MiB are not written where a call has as many blocks of 256 positions of a head as there are SMs
// (most such have waves enough; of those whose heads packed into tiles make fewer CTAs, eight parts of 127 CTAs and more,
// which only dense calls over 94,000 rows and more would take, for a promised tenth).

// How the query rows of a call are laid out: see QRows.
struct AttnShape {
  int span, block;                 // chunk positions of a Q tile and of a row block
  long long blocks, per_rb, jobs;  // row blocks of a head group; CTAs of one row block of every head; CTAs
};
static AttnShape attn_shape(const quoka_params* p, const AttnPlan& plan) {
  AttnShape a;
  a.span = kQTile / plan.pack;
  a.block = plan.q_tiles * plan.ctas * a.span;
  a.blocks = (p->chunk_len + a.block - 1) / a.block;
  a.per_rb = (long long)(p->n_q_heads / plan.pack) * plan.ctas * p->batch;
  a.jobs = a.per_rb * a.blocks;
  return a;
}
// Whole row blocks of two Q tiles per CTA (head_dim 128: of a pair of CTAs), `pack` heads to a tile.
static AttnPlan attn_whole(const quoka_params* p, int pack) {
  AttnPlan plan;
  plan.ctas = p->head_dim == 128 ? 2 : 1;
  plan.pack = pack;
  return plan;
}
// Heads that may share a Q tile: divisors of the group whose row blocks the grid's second dimension holds (32 heads to a tile
// at head_dim 64: chunks of 524280 positions; one head: of 16.7 million).
static bool attn_pack_fits(const quoka_params* p, int pack) {
  return p->n_q_heads / p->n_kv_heads % pack == 0 && (pack == 1 || attn_shape(p, attn_whole(p, pack)).blocks <= 65535);
}
static int attn_largest_pack(const quoka_params* p) {
  int pack = std::min(p->n_q_heads / p->n_kv_heads, 32);
  while (pack > 1 && !attn_pack_fits(p, pack)) --pack;
  return pack;
}
static double attn_step_us(const quoka_params* p, int q_tiles, int ctas, bool sparse) {
  static constexpr double us[3][2][2] = {{{1.02, 1.13}, {1.38, 1.42}},     // head_dim 64: one Q tile, two; dense, listed
                                         {{0.95, 1.35}, {2.00, 2.05}},     // head_dim 128, one CTA
                                         {{1.09, 1.25}, {1.35, 1.30}}};    // and a pair
  return us[p->head_dim == 64 ? 0 : ctas][q_tiles - 1][sparse ? 1 : 0];
}
// The plan for `pack` heads to a tile over `tiles` key tiles besides the chunk's own, with no more scratch than `room`;
// *model_us: what the model says.
static AttnPlan attn_plan_of(const quoka_params* p, int pack, int tiles, bool sparse, size_t room, long long sms, double* model_us) {
  constexpr double kStart[3] = {6.0, 9.0, 9.5}, kStartTwoOfPair = 11.5;                // head_dim 64, 128, a pair
  constexpr double kParts128 = 5.2, kPart128 = 1.6, kParts64 = 5.5, kPart64 = 1.0, kCluster = 3.8, kSparseParts = 3.0, kOwn = 0.5;
  const bool wide = p->head_dim == 128;
  AttnPlan plan = attn_whole(p, pack);
  const AttnShape two = attn_shape(p, plan);
  const auto own = [](long long positions) { return (double)((positions + kKeyTile - 1) / kKeyTile); };
  // at least as many blocks of 256 positions of a head as SMs
  const bool bounded = (long long)p->n_q_heads * p->batch * ((p->chunk_len + 255) / 256) >= sms;
  double best = 1e30;
  for (int ctas = wide ? 2 : 1; ctas >= 1; --ctas) {
    for (int q_tiles = 2; q_tiles >= 1; --q_tiles) {
      AttnPlan form = attn_whole(p, pack);
      form.q_tiles = q_tiles; form.ctas = ctas;
      const AttnShape a = attn_shape(p, form);
      // the last row block, which may have no second tiles, and the one before it
      const double step = attn_step_us(p, q_tiles, ctas, sparse);
      const long long before = (a.blocks - 1) * a.block;
      const double step_last = p->chunk_len - before <= ctas * a.span ? attn_step_us(p, 1, ctas, sparse) : step;
      const auto walk = [&](double w) {
        return std::max(step_last * (tiles + w * own(p->chunk_len)), before > 0 ? step * (tiles + w * own(before)) : 0.0);
      };
      const double start = ctas == 2 && q_tiles == 2 ? kStartTwoOfPair : kStart[wide ? ctas : 0];
      const double w = sparse ? kOwn : 1.0, x = (double)a.jobs / (double)sms;
      // (CTAs of a grid of waves do not start in step: between the number of waves and the mean)
      const double mean = step * (tiles + 0.5 * w * (own(p->chunk_len) + (double)a.block / kKeyTile));
      const double whole = a.jobs <= sms ? start + walk(w) : 0.5 * (x + std::ceil(x)) * (start + mean);
      // what lies further from the calls that the model was fitted to has to promise some percent: one CTA in the place of a pair,
      // parts through memory, more than a wave; in grids of a wave and more every other form
      const double sure = (wide && ctas == 1 ? 1.04 : 1.0) * (a.jobs > sms ? 1.02 : 1.0);
      const auto consider = [&](double us, int parts, bool in_cluster) {
        AttnPlan next = form;
        next.parts = parts; next.in_cluster = in_cluster;
        next.split_rb = parts > 1 ? (int)a.blocks : 0;
        us *= parts > 1 && !in_cluster ? 1.02 * sure : sure;
        if (best < 1e30 && (us >= (two.jobs >= sms ? 0.97 : 1.0) * best || a.blocks * parts > 65535)) return;
        if (attn_plan_scratch_bytes(p, next) > room || (bounded && attn_split_partial_bytes(p, next) > kMostAttnPartials)) return;
        best = us;
        plan = next;
      };
      consider(whole, 1, false);
      if (a.jobs > sms) continue;
      const double rest = start + (sparse ? kSparseParts : 0.0), t = walk(1.0);
      for (int parts = 2; parts <= 8 && 2 * parts <= tiles + 1; ++parts) {
        const double waves = (double)(((int)a.jobs * parts - 1) / (int)sms + 1);
        consider(rest + waves * (t / parts + (wide ? kParts128 + kPart128 * parts : kParts64 + kPart64 * parts)), parts, false);
        if (ctas == 2 && parts <= 4 && a.jobs / 2 <= (parts == 2 ? 28 : parts == 3 ? 20 : 14))
          consider(rest + t / parts + kCluster, parts, true);
      }
    }
  }
  *model_us = best;
  const long long n_rb = two.blocks, per_rb = two.per_rb, jobs = two.jobs;
  const long long q = jobs / sms, rest = jobs % sms;
  if (jobs < sms || rest == 0 || (sparse && p->batch > 1) || plan.q_tiles != 2 || plan.ctas != (wide ? 2 : 1)) return plan;
  constexpr double kPartCost = 6.0;
  const double own_step = (double)two.block / kKeyTile;                      // the chunk's own tiles grow by this per row block
  const long long split = (rest + per_rb - 1) / per_rb;                      // row blocks to cut; block r has about (r + 1) * own_step of its own tiles
  const double t_all = tiles + 3 + 0.5 * own_step * n_rb, t_whole = tiles + 3 + 0.5 * own_step * (split + n_rb), t_split = tiles + 3 + 0.5 * own_step * split;
  double least = (sparse ? 0.92 : 0.94) * (double)(q + 1) * t_all;
  for (int parts = 2; parts <= 8 && parts <= (tiles + 1) / 6; ++parts) {
    const double t_part = t_split / parts + kPartCost;
    const double cost = ((double)(jobs - split * per_rb) * t_whole + (double)(split * per_rb * parts) * t_part) / (double)sms + 0.3 * t_part;
    AttnPlan cand = attn_whole(p, pack);
    cand.split_rb = (int)split; cand.parts = parts;
    if (cost < least && attn_split_partial_bytes(p, cand) <= kMostAttnPartials && attn_plan_scratch_bytes(p, cand) <= room) {
      least = cost;
      plan = cand;
      *model_us = std::min(*model_us, kStartTwoOfPair + attn_step_us(p, 2, plan.ctas, sparse) * cost / 0.9);
    }
  }
  return plan;
}
// How many heads share a tile: the whole group where its heads fill tiles (1, 2, 4, 8, 16 or 32 of them), else the largest
// divisor that the model puts within 2 % of the best one.  More heads make fewer CTAs of a short chunk, and leave rows over in
// those of a long one.  Two KV heads over 16384 rows, every divisor of 15 groups of 9 to 40 heads, 64, 600 and 2048 queries, both head
// dims, sparse and dense: the choice takes 1.0 % more time than the best one in the geometric mean (18 % at most), the largest
// divisor up to 32 6 % (45 %).  Dense, 26 heads to a KV head, 1 / 2 / 13 / 26 of them to a tile: 64 queries, head_dim 128, 154 /
// 94 / 57 / 57 us; 2048 queries, head_dim 64, 597 / 586 / 630 / 791.
static AttnPlan attn_plan(const quoka_params* p, int tiles, bool sparse, size_t room) {
  const int largest = attn_largest_pack(p);
  const long long sms = device_sm_count();
  if (p->dtype != QUOKA_BF16 || p->impl == QUOKA_IMPL_SIMT || p->chunk_len <= 1 || sms <= 0) return attn_whole(p, largest);
  double best, us;
  AttnPlan plan = attn_plan_of(p, largest, tiles, sparse, room, sms, &best);
  if (kQTile % largest == 0) return plan;
  for (int pack = largest - 1; pack >= 1; --pack) {
    if (!attn_pack_fits(p, pack)) continue;
    const AttnPlan other = attn_plan_of(p, pack, tiles, sparse, room, sms, &us);
    if (us < 0.98 * best) { plan = other; best = us; }
  }
  return plan;
}
AttnPlan attn_plan_sparse(const quoka_params* p, int budget_cap, size_t room) { return attn_plan(p, (budget_cap + kKeyTile - 1) / kKeyTile, true, room); }
AttnPlan attn_plan_dense(const quoka_params* p, size_t room) { return attn_plan(p, (p->max_ctx_len + kKeyTile - 1) / kKeyTile, false, room); }
static size_t attn_split_jobs(const quoka_params* p, const AttnPlan& plan) { return (size_t)attn_shape(p, plan).per_rb * plan.split_rb; }
size_t attn_split_partial_bytes(const quoka_params* p, const AttnPlan& plan) {
  return plan.in_cluster ? 0 : attn_split_jobs(p, plan) * plan.parts * 2 * kSplitTileFloats * sizeof(float);
}
size_t attn_split_counter_bytes(const quoka_params* p, const AttnPlan& plan) { return plan.in_cluster ? 0 : attn_split_jobs(p, plan) * 8 * sizeof(int32_t); }
size_t attn_plan_scratch_bytes(const quoka_params* p, const AttnPlan& plan) {
  return (attn_split_counter_bytes(p, plan) + 255) / 256 * 256 + (attn_split_partial_bytes(p, plan) + 255) / 256 * 256;
}

// The launches of an attention call: the whole row blocks, then the ones in parts.
//
// Programmatic stream serialisation, (1) inside the fused call: the first launch may start while the kernel before it on
// the stream (the key selection, which signals early and writes none of this kernel's other inputs) still runs; it touches
// the selection's outputs only after its own griddepcontrol.wait.  A stand-alone call keeps the ordinary stream order:
// whatever ran before it may have written q, k or v.  (2) The parts always: their CTAs take the SMs that the whole row
// blocks' last wave leaves idle.  The whole row blocks let them start once every CTA has begun (dense) or has learnt the
// list length (sparse: the selection is complete by then, so the parts need not wait for it), and the parts' last CTA
// waits for the whole row blocks before it ends.
quoka_status launch_attn_plan(const quoka_params* p, const DevParams& P, const AttnPlan& plan, AttnKernel (*pick)(bool, bool, bool),
                              const char* name, int cluster, int threads, size_t smem, const CUtensorMap& tm_q, const CUtensorMap& tm_k,
                              const CUtensorMap& tm_v, const void* k, const void* v, const int32_t* k_idx, const int32_t* k_cnt,
                              void* out, float* lse, cudaStream_t st, bool after_selection) {
  const bool sparse = k_idx != nullptr, split = plan.split_rb > 0 && (P.attn_partials || plan.in_cluster);
  DevParams PP = P;
  const AttnShape shape = attn_shape(p, plan);
  PP.attn_row_blocks = (int)shape.blocks;
  PP.attn_split_rb = split ? plan.split_rb : 0;
  PP.attn_parts = split ? plan.parts : 1;
  const int whole = PP.attn_row_blocks - PP.attn_split_rb;
  PP.attn_after_whole = whole > 0 ? 1 : 0;
  if (split && !plan.in_cluster && !after_selection &&          // (the fused call clears the counters in an earlier kernel)
      cudaMemsetAsync(P.attn_counters, 0, attn_split_counter_bytes(p, plan), st) != cudaSuccess)
    return QUOKA_ERR_CUDA;
  for (int parts = whole > 0 ? 0 : 1; parts <= (split ? 1 : 0); ++parts) {
    AttnKernel kernel = pick(sparse, parts != 0, plan.in_cluster);
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) return QUOKA_ERR_CUDA;
    const bool early = parts && whole > 0 ? true : sparse && after_selection;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(shape.per_rb / P.batch), parts ? PP.attn_split_rb * PP.attn_parts : whole, P.batch);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    cfg.attrs = attr;
    if (early) {
      attr[cfg.numAttrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
      attr[cfg.numAttrs++].val.programmaticStreamSerializationAllowed = 1;
    }
    if (parts && plan.in_cluster) {           // (the other kernels' clusters are part of the kernel)
      attr[cfg.numAttrs].id = cudaLaunchAttributeClusterDimension;
      attr[cfg.numAttrs].val.clusterDim.x = (unsigned)cluster;
      attr[cfg.numAttrs].val.clusterDim.y = (unsigned)PP.attn_parts;
      attr[cfg.numAttrs++].val.clusterDim.z = 1;
    }
    log_launch(name, cfg.gridDim, cfg.blockDim, smem, parts && plan.in_cluster ? cluster * PP.attn_parts : cluster, early);
    if (cudaLaunchKernelEx(&cfg, kernel, PP, tm_q, tm_k, tm_v, (const __nv_bfloat16*)k, (const __nv_bfloat16*)v, k_idx, k_cnt,
                           (__nv_bfloat16*)out, lse) != cudaSuccess)
      return QUOKA_ERR_CUDA;
    count_launch();
  }
  return cudaGetLastError() == cudaSuccess ? QUOKA_OK : QUOKA_ERR_CUDA;
}

static AttnShape attn_usual_shape(const quoka_params* p) { return attn_shape(p, attn_whole(p, attn_largest_pack(p))); }
bool attn_below_a_wave(const quoka_params* p) { return attn_usual_shape(p).jobs < device_sm_count(); }
// (above a wave the cost of a plan with parts is more than q waves of average jobs, its line at most 0.94 (q + 1): none from q = 16 on)
bool attn_may_have_parts(const quoka_params* p) { return attn_usual_shape(p).jobs < 17ll * device_sm_count(); }
int attn_same_plan_up_to(const quoka_params* p, int chunk) {
  int last = (chunk + kKeyTile - 1) / kKeyTile * kKeyTile;
  for (int pack = attn_largest_pack(p); pack >= 1; --pack) {
    const int span = kQTile / pack;
    if (attn_pack_fits(p, pack)) last = std::min(last, (chunk + span - 1) / span * span);
  }
  return last;
}

bool attn_tc_supported(const quoka_params* p) {
  if (p->dtype != QUOKA_BF16) return false;
  return kv_places_fit(p, 8);                         // the loaders address cache rows in 32-bit units of 16 bytes
}
bool kv_places_fit(const quoka_params* p, int unit) {
  typedef __int128 Wide;                              // (nothing bounds the strides that a caller may give)
  const Wide pages = p->page_size ? p->kv_rows : p->batch, rows = p->page_size ? kPage : p->kv_rows;
  const Wide elements = (pages - 1) * p->kv_stride_b + (Wide)(p->n_kv_heads - 1) * p->kv_stride_h + (rows - 1) * p->kv_stride_t + p->head_dim;
  return elements / unit < (Wide)0xFFFFFFFFll;
}

bool encode_q_tensor_map(CUtensorMap* out, const DevParams& P, const void* q) {
  const uint64_t dims[5] = {(uint64_t)P.d, (uint64_t)P.attn_pack, (uint64_t)P.chunk, (uint64_t)(P.n_q / P.attn_pack), (uint64_t)P.batch};
  const uint64_t strides[4] = {(uint64_t)P.q_sh * 2, (uint64_t)P.q_st * 2, (uint64_t)P.q_sh * 2 * P.attn_pack, (uint64_t)P.q_sb * 2};
  const uint32_t box[5] = {64, (uint32_t)P.attn_pack, (uint32_t)P.attn_span, 1, 1};
  return encode_tensor_map_bf16(out, q, 5, dims, strides, box);
}

DevParams attn_of_plan(const DevParams& P0, const AttnPlan& plan) {
  DevParams P = P0;
  P.attn_pack = plan.pack;
  P.attn_span = kQTile / plan.pack;
  P.attn_qtiles = plan.q_tiles;
  return P;
}

quoka_status launch_attn_tc(const quoka_params* p, const DevParams& P0, const void* q, const void* k, const void* v,
                            const int32_t* k_idx, const int32_t* k_cnt, void* out, float* lse, cudaStream_t st,
                            bool after_selection, const AttnPlan& plan) {
  DevParams P = attn_of_plan(P0, plan);
  P.list_of_selection = after_selection ? 1 : 0;
  if (plan.ctas == 2) return launch_attn_tc_pair(p, P, q, k, v, k_idx, k_cnt, out, lse, st, after_selection, plan);
  CUtensorMap tm_q, tm_k, tm_v;
  if (!encode_q_tensor_map(&tm_q, P, q)) return QUOKA_ERR_CUDA;
  if (!encode_kv_tensor_map(&tm_k, p, k, 64) || !encode_kv_tensor_map(&tm_v, p, v, 64)) return QUOKA_ERR_CUDA;
  const bool wide = P.d == 128;
  return launch_attn_plan(p, P, plan, wide ? pick_attn_tc<128, 0> : pick_attn_tc<64, 0>, "attn_tc", /*cluster=*/1, kAttnThreads,
                          wide ? attn_tc_smem<128>() : attn_tc_smem<64>(), tm_q, tm_k, tm_v, k, v, k_idx, k_cnt, out, lse, st, after_selection);
}

}  // namespace quoka
