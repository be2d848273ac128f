// bf16 MFMA GEMM for the stage's four projections (paper Sec. 3.4: linear layers dominate the
// execution time of a decode step, and only the batch size sets their cost).
//
//   out[M, N] = epilogue( A[M, K] * W^T ),   A bf16 M x K,  W bf16 Npad x Kpad  (both K-contiguous in
//   32-column blocks; W and the stage's own activations are pair-interleaved, see OperandLayout)
//
// Both operands are K-contiguous, so an MFMA fragment is one 16-byte load.  The product is formed
// transposed, D[n][m] = sum_k W[n][k] A[m][k], with the weights as the MFMA "A" operand: a lane
// then holds four consecutive output columns n of one row m, which makes the epilogue's stores
// 8 bytes wide and lets the SwiGLU epilogue find gate and up of one column in the same lane.
//
// Tiles go from global memory straight into LDS (direct-to-LDS loads, a ring of 32-wide k-stages,
// one barrier per stage) with an XOR swizzle of the 16-byte chunks applied on the global side, so
// that the fragment reads are free of bank conflicts.  For small M (decode) the K range is split
// across workgroups; the fp32 partials are summed by the kernel that consumes the projection, or
// by a reduce kernel that applies the epilogue.
#include <math.h>
#include <stdio.h>
#include <stdlib.h>

#include <initializer_list>
#include <mutex>
#include <unordered_map>

#include "gemm_kernel.h"

namespace tdp {

// Sum the split-K partials and apply the epilogue.  One thread per 4 output columns.
__global__ __launch_bounds__(256) void gemm_reduce_kernel(const GemmParams p, int out_cols) {
  const int64_t idx = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  const int groups = out_cols / 4;
  if (idx >= (int64_t)p.M * groups) return;
  const int m = (int)(idx / groups);
  const int j = (int)(idx % groups) * 4;
  auto sum_at = [&](int n) {
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
    for (int z = 0; z < p.splits; ++z)
      s += *reinterpret_cast<const f32x4*>(p.ws + ((int64_t)z * p.M + m) * p.Npad + n);
    return s;
  };
  if (p.epilogue == EPI_SWIGLU) {
    const int ng = (j / 32) * 64 + (j % 32);
    f32x4 g = sum_at(ng), u = sum_at(ng + 32);
    bf16x4 o;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = (bf16)(silu_f(g[e]) * u[e]);
    *reinterpret_cast<bf16x4*>(p.out + operand_offset(p.u_lay, m, j)) = o;
  } else {
    const f32x4 t = sum_at(j);
    float v[4] = {t[0], t[1], t[2], t[3]};
    store_row4(p, m, j, v);
  }
}

// The same for a product of integers: the sums are exact, then the scales.  (Gated results in rows of ldo, plain and gated in bf16 or fp32.)
__global__ __launch_bounds__(256) void gemm_reduce_int_kernel(const GemmIntParams p, int out_cols) {
  const int64_t idx = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  const int groups = out_cols / 4;
  if (idx >= (int64_t)p.M * groups) return;
  const int m = (int)(idx / groups);
  const int j = (int)(idx % groups) * 4;
  const float as = p.a_scale[m];
  auto sum_at = [&](int n) {
    i32x4 s = {0, 0, 0, 0};
    for (int z = 0; z < p.splits; ++z)
      s += *reinterpret_cast<const i32x4*>(p.ws + ((int64_t)z * p.M + m) * p.Npad + n);
    return scaled(__builtin_bit_cast(f32x4, s), *reinterpret_cast<const f32x4*>(p.w_scale + n), as);
  };
  float v[4];
  if (p.epilogue == EPI_SWIGLU) {
    const int ng = (j / 32) * 64 + (j % 32);
    const f32x4 g = sum_at(ng), u = sum_at(ng + 32);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = silu_f(g[e]) * u[e];
    store_values4(p, m, j, v);
  } else {
    const f32x4 t = sum_at(j);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = t[e];
    store_row4(p, m, j, v);
  }
}

// Kernel variants; 1 .. kGemmTileMax can be selected by callers (GemmArgs::force_tile), the planner chooses among
// all.  A tile has as many rows as the batch needs, in steps of 32: rows past M cost as much as real ones
// (matrix pipe, LDS reads, power), and with tiles of 128 and 256 rows alone a batch of 307 paid for 512 (gate/up 57344 x
// 8192: 366 us, with 2 x 160 rows 278; M = 384: 371 -> 308; M = 200: 202 -> 180).  128 weight rows per
// tile instead of 256 where the weights are what counts (M up to 128: twice the workgroups, half the split-K
// factor where the order of the sums is free; M = 48, 22016 x 4096: 45 -> 39 us) and
// between 160 and 256 rows on narrow projections.  The ring takes what LDS there is; two or three workgroups
// per CU where a tile is small enough (their fill and epilogue then overlap the neighbour's stages).
enum GemmKind { kOrdinary, kRotating, kMaximum, kStatistics, kIntegers, kIntStatistics, kKinds };
struct TileInfo {
  int at, wt, ns, wg_per_cu;
  bool chunked;           // can sum K in chunks
  double stage_us;        // a 32-wide stage of one tile on a CU, the matrix pipe's part (see plan_cost)
  int bm() const { return at * 32; }
  int bn() const { return wt * 32; }
  int ring_rows() const { return (at * 2 + 3) / 4 * 64 + bn(); }  // rows of a ring stage (see IPA)
  int lds_bytes() const { return ns * ring_rows() * 64; }
};
#define TDP_TILE(AT, WT, NS, PER_CU, US) {AT, WT, NS, PER_CU, kChunked<AT, WT, NS>, US},
static const TileInfo kTiles[] = {{0, 0, 0, 0, false, 0.0}, TDP_GEMM_TILES(TDP_TILE)};
#undef TDP_TILE
constexpr int kTileCount = sizeof(kTiles) / sizeof(kTiles[0]);
#define TDP_ORDINARY(AT, WT, NS, ...) TDP_KERNELS(AT, WT, NS, GemmParams),
#define TDP_ROTATING(AT, WT, NS, ...) TDP_KERNELS(AT, WT, NS, GemmRotateParams),
#define TDP_MAXIMUM(AT, WT, NS, ...) TDP_KERNELS(AT, WT, NS, GemmMaxParams),
static const GemmKernels kOrdinaryKernels[] = {TDP_GEMM_TILES(TDP_ORDINARY)}, kRotatingKernels[] = {TDP_GEMM_TILES(TDP_ROTATING)},
                         kMaximumKernels[] = {TDP_GEMM_TILES(TDP_MAXIMUM)};
#undef TDP_ORDINARY
#undef TDP_ROTATING
#undef TDP_MAXIMUM
// null: no such kernel (see gemm_can_rotate, kChunksOnlyTile)
static const void* gemm_kernel(int tile, GemmKind kind, bool nt) {
  const GemmKernels* const kinds[kKinds] = {kOrdinaryKernels,          kRotatingKernels,   kMaximumKernels,
                                            gemm_statistics_kernels(), gemm_int_kernels(), gemm_int_statistics_kernels()};
  return kinds[kind][tile - 1].of[nt ? 1 : 0];
}
// The 128 x 128 tile that has room for chunked sums is used for those only: otherwise two workgroups per CU (tile 3) are 7 to 15 %
// faster at the same split-K factor (1367 pairs of launches, M from 1 to 16384).
constexpr int kChunksOnlyTile = 11;

static bool g_print_plan = false;  // tuning aid, read from the environment once (gemm_setup)

hipError_t gemm_setup() {
  static std::once_flag once;
  static hipError_t result = hipSuccess;
  std::call_once(once, [] {
    g_print_plan = getenv("TDP_GEMM_PLAN") != nullptr;
    hipError_t e;
    e = hipSuccess;
    for (int i = 1; i < kTileCount; ++i)
      for (int kind = 0; kind < kKinds; ++kind)
        for (bool nt : {false, true}) {
          const void* const kernel = gemm_kernel(i, (GemmKind)kind, nt);
          if (kernel && e == hipSuccess)
            e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, kTiles[i].lds_bytes());
        }
    result = e;
  });
  return result;
}

// Estimated time in us of a launch with this tile and split-K factor (per = 64-wide k-tiles of a split).  An XCD
// makes its eighth of the tiles in rounds of 32 CUs x wg_per_cu; a 32-wide stage of a round costs the matrix
// pipe, the LDS fill of a CU, the XCD's reads through its fabric port, the chip's reads of the weights and the
// latency the ring has to cover - none of which hides behind another entirely, hence the power sum;
// a round ends with its epilogue; split-K adds the fp32 partials' round trip and, where no later kernel sums them,
// a reduce launch.  The constants are a least-squares fit to 10,000 launches timed on cold weights (19 projection
// shapes, M from 4 to 19346, 1 to 16 splits): the tile and factor that this picks are on average 1.3 % slower
// than the fastest measured, against 32 % for the rule it replaces (M <= 128, narrow, else; rounds of k-tiles).  Up to 128
// rows the choice is narrower, see sum_order_splits.
// `rotated`: the QKV projection of a stage where its sums are free.  It stores fp32 whether it is split or not, so each
// store costs alike (0.6 us per million elements), and each split more costs the rotation 0.5 us and 0.33 per million
// elements (128 to 512 rows, seven shapes).  Charged for the store of a split alone, like the other projections, 13B at 512 rows took
// 256 x 128 tiles unsplit where 256 x 256 in two splits are faster (with the rotation 79.2 + 51.2 us against 70.5 + 51.9); Qwen at
// 512 rows 56.0 + 16.9 against 45.3 + 17.8, 70B at 384 rows 87.1 + 15.8 against 67.5 + 18.4.  Over 264 cases with M from 129 to
// 16384 the choice was 2.5 % slower than the fastest, now 0.2 %.
// (These costs are of the projection with a rotation kernel behind it.  An unsplit tile of 256 weight rows of a 16-bit prefill stores no
// fp32 and has none, see gemm_can_rotate; the plan, which decode and 8-bit caches share, does not count that in, so it can keep a split
// or a tile of 128 weight rows where rotating in the epilogue would be a little ahead.)
static double plan_cost(const TileInfo& ti, int64_t M, int64_t Npad, int per, int splits, int epilogue, bool defer,
                        bool rotated, bool integers) {
  const double tm = (double)((M + ti.bm() - 1) / ti.bm()), tn = (double)(Npad / ti.bn());
  const double tiles = tm * tn * splits;
  const int64_t per_xcd = ((int64_t)tiles + 7) / 8, slots = 32 * ti.wg_per_cu;
  const int64_t full = (per_xcd - 1) / slots, last = per_xcd - full * slots;  // full rounds, tiles of the last one
  const double band = tm / (double)(((int64_t)tm + 3) / 4);                   // rows of tiles in a band
  const double mfma = ti.at * ti.wt;
  const double a_rows = ti.ring_rows() - ti.bn(), bn = ti.bn();
  auto stage = [&](int64_t n) {  // n tiles of the XCD at once
    const double per_cu = (double)((n + 31) / 32);
    const double cols = ceil((double)n / band);
    const double on_chip = (double)(8 * n) < tiles ? (double)(8 * n) : tiles;
    const double terms[5] = {per_cu * ti.stage_us,
                             per_cu * ti.ring_rows() * (0.064 / 117.6),
                             ((band < n ? band : (double)n) * a_rows + cols * bn) * (512e-6 / 11.1),
                             on_chip / tm * bn * (64e-6 / 18.3),
                             0.21 / (ti.ns - 1)};
    double sum = 0;
    for (double t : terms) sum += t * sqrt(t);  // power 1.5
    return cbrt(sum * sum);
  };
  auto epi = [&](int64_t n) { return 0.94 + 0.12 * mfma * (double)((n + 31) / 32); };
  double us = 1.9 + full * (2 * per * stage(slots) + epi(slots)) + 2 * per * stage(last) + epi(last);
  const double elems = M * (double)Npad;
  if (rotated) {
    us += 0.6e-6 * splits * elems + (splits - 1) * (0.5 + 0.33e-6 * elems);
  } else if (splits > 1) {
    us += 0.81e-6 * splits * elems + 0.15 * splits;
    // (Of integers, whose factor is free for small batches too: over 97 cases of 1 to 8191 rows, nine shapes, the choice is 2.3 % slower than
    // the fastest tile and factor with 5.4 us, at most 31 % - 48 rows of 4096 x 12288 unsplit, 22.4 us, instead of in two, 18.7 - and
    // with 2 us 1.3 and 14 %.)
    if (!defer) us += integers ? 2.0 : 5.4;
    else if (epilogue == EPI_STORE) us += 0.4e-6 * (splits - 1) * elems;  // read by the rotation
  }
  return us * (1.0 + 0.004 * tm);  // ties: fewer rows of tiles, the weights are read fewer times
}

// The order in which a projection of up to 128 rows sums over K, as a split-K factor.  fp32 sums in another order differ in
// their last bits, which the bf16 roundings behind them carry through every layer: about 0.5 % of a
// hidden state after a few layers, as much as bf16 itself costs, and enough to turn a greedy token between near-equal
// logits (measured once in four runs: 2 of 48 over four layers and a vocabulary of 32000).  The distance to the 64-bit result is the
// same in either order.  What the rule below is for is nothing but this: decode batches of up to 128 rows give the bits that they
// gave when every such launch was made of 128 x 256 tiles, one per CU (in super-blocks dealt to the XCDs, 1.8 us per round
// of k-tiles plus the partials' round trip - the cost that it minimises), whatever tile makes the sum now: as that many split-K
// workgroups or, where the tile has registers for it, chunk by chunk in one.  The factor depends on M, N, K and the
// workspace, so a request's bits may change with the batch around it (4096 x 4096 is 16 splits up to 64 rows, 11 at 128), and above
// 128 rows the plan is free.  Keeping it costs what a freer factor would gain: 13B decode, 128 rows, two layers 1206 against 1172
// us; 7B token step, 48 rows, 796 against 738.
// Short sums (K <= 1024) are free: there another order moves a hidden state by 3e-5 at most, and a freer factor takes a
// two-layer stage of hidden size 256 from 66 to 59 us.
constexpr int kSumOrderRows = 128, kSumOrderKTiles = 16;
static int sum_order_splits(int64_t M, int64_t Npad, int k_tiles, int64_t workspace_elems) {
  const int tn = (int)(Npad / 256);
  int most = k_tiles / 4 < 16 ? (k_tiles / 4 > 0 ? k_tiles / 4 : 1) : 16;
  if (most > k_tiles) most = k_tiles;
  int best = 1;
  double best_cost = 1e300;
  for (int sp = 1; sp <= most; ++sp) {
    if (sp > 1 && sp * M * Npad > workspace_elems) break;
    const int per = (k_tiles + sp - 1) / sp;
    if ((k_tiles + per - 1) / per != sp) continue;
    for (int lg = 5; lg >= 0; --lg) {
      const int size = 1 << lg, n_sb = (tn + size - 1) / size;
      int load[8] = {0, 0, 0, 0, 0, 0, 0, 0}, longest = 0;
      for (int g = 0; g < n_sb * sp; ++g) {
        const int sb = g % n_sb;
        load[g & 7] += (sb + 1) * size <= tn ? size : tn - sb * size;
      }
      for (int x : load) longest = x > longest ? x : longest;
      double cost = (double)((longest + 31) / 32) * (per + 6.0);
      if (sp > 1) cost += 1.1e-6 * sp * M * (double)Npad + 2.0;
      cost *= 1.0 + 0.02 * (5 - lg);
      if (cost < best_cost) {
        best_cost = cost;
        best = sp;
      }
    }
  }
  return best;
}

static GemmPlan search_plan(const GemmPlanKey& a) {
  GemmPlan plan{0, 1, 0};
  const int k_tiles_total = (int)(a.Kpad / 64);
  const bool forced = a.force_tile >= 1 && a.force_tile <= kGemmTileMax;
  double best_cost = 1e300;
  // up to kSumOrderRows rows the order of the sums is given, and only how it is made is chosen
  const int order = a.force_splits <= 0 && !forced && !a.integers && a.M <= kSumOrderRows && k_tiles_total > kSumOrderKTiles
                        ? sum_order_splits(a.M, a.Npad, k_tiles_total, a.workspace_elems) : 0;
  const bool rotated = a.defer && a.epilogue == EPI_STORE && order == 0;
  for (int t = forced ? a.force_tile : 1; t <= (forced ? a.force_tile : kTileCount - 1); ++t) {
    const int64_t tiles1 = (int64_t)((a.M + kTiles[t].bm() - 1) / kTiles[t].bm()) * ((a.Npad + kTiles[t].bn() - 1) / kTiles[t].bn());
    const int k_splits_max = k_tiles_total / 2 < 16 ? (k_tiles_total / 2 > 0 ? k_tiles_total / 2 : 1) : 16;
    int sp = a.force_splits > 0 ? a.force_splits : 1, sp_max = a.force_splits > 0 ? a.force_splits : k_splits_max;
    if (order > 0) sp_max = order;
    if (sp > k_tiles_total) sp = sp_max = k_tiles_total;
    for (; sp <= sp_max; ++sp) {
      const int per = (k_tiles_total + sp - 1) / sp;
      const int real_sp = (k_tiles_total + per - 1) / per;
      const bool chunks = order > 1 && real_sp == 1;
      if (real_sp != sp && a.force_splits <= 0) continue;  // same schedule as a smaller factor
      if (order > 1 && sp != order && (sp > 1 || !kTiles[t].chunked)) continue;
      if (t == kChunksOnlyTile && !chunks && !forced) continue;
      if (real_sp > 1 && (int64_t)real_sp * a.M * a.Npad > a.workspace_elems) break;
      // (four rounds of tiles: nothing is left for a split to gain)
      if (real_sp > 1 && a.force_splits <= 0 && order == 0 && tiles1 * real_sp > 1024 * kTiles[t].wg_per_cu) break;
      double cost = plan_cost(kTiles[t], a.M, a.Npad, per, real_sp, a.epilogue, a.defer, rotated, a.integers);
      // (chunks: the sums between them stop the matrix pipe, and a workgroup's waves do it together; 128 x 15360 x 5120 in
      // two rows of 64 x 128: 48.6 us where the estimate is 40, against 39.4 as four splits)
      if (chunks) cost *= 1.1;
      if (cost < best_cost) {
        best_cost = cost;
        plan = GemmPlan{t, real_sp, chunks ? (k_tiles_total + order - 1) / order : 0};
      }
    }
  }
  if (plan.tile == 0) plan = GemmPlan{forced ? a.force_tile : 1, 1, 0};  // the workspace holds no such split
  return plan;
}

// The search costs tens of microseconds on the host and its answer depends only on the problem's shape, so it
// is remembered (a serving loop asks for the same few shapes every step).
GemmPlan gemm_plan(const GemmPlanKey& key) {
  struct Hash {
    size_t operator()(const GemmPlanKey& k) const {
      uint64_t h = 0x9e3779b97f4a7c15ull;
      for (uint64_t v : {(uint64_t)k.M, (uint64_t)k.force_tile, (uint64_t)k.force_splits, (uint64_t)(k.epilogue * 4 + k.integers * 2 + k.defer),
                         (uint64_t)k.Npad, (uint64_t)k.Kpad, (uint64_t)k.workspace_elems})
        h = (h ^ v) * 0xff51afd7ed558ccdull + (h >> 29);
      return (size_t)h;
    }
  };
  static std::mutex mutex;
  static std::unordered_map<GemmPlanKey, GemmPlan, Hash> cache;
  {
    std::lock_guard<std::mutex> lock(mutex);
    const auto it = cache.find(key);
    if (it != cache.end()) return it->second;
  }
  const GemmPlan plan = search_plan(key);
  std::lock_guard<std::mutex> lock(mutex);
  if (cache.size() < 65536) cache[key] = plan;
  return plan;
}

bool gemm_form_fits(const GemmPlan& f, int M, int64_t Npad, int64_t Kpad, int64_t workspace_elems) {
  const int k_tiles = (int)(Kpad / 64);
  if (f.tile < 1 || f.tile >= kTileCount || f.splits < 1 || f.splits > k_tiles || f.chunk < 0) return false;
  const int per = (k_tiles + f.splits - 1) / f.splits;
  if ((k_tiles + per - 1) / per != f.splits) return false;  // the last splits would have nothing to sum
  if (f.chunk > 0 && (f.splits > 1 || !kTiles[f.tile].chunked)) return false;
  return f.splits == 1 || f.splits * (int64_t)M * Npad <= workspace_elems;
}

bool gemm_form_fits_integers(const GemmPlan& f, int M, int64_t Npad, int64_t Kpad, int64_t workspace_elems) {
  return f.tile != kChunksOnlyTile && f.chunk == 0 && gemm_form_fits(f, M, Npad, Kpad, workspace_elems);
}

void gemm_tile_size(int tile, int* rows, int* weight_rows) {
  *rows = kTiles[tile].bm();
  *weight_rows = kTiles[tile].bn();
}

static GemmPlan plan_of(const GemmArgs& a) {
  // (a vocabulary projection is planned alike whether its logits are wanted or their statistics: the same bits)
  const bool defer = a.splits_used != nullptr && a.epilogue != EPI_SWIGLU && !a.stats;
  return a.form.tile ? a.form
                     : gemm_plan({a.M, a.force_tile, a.force_splits, a.epilogue, defer, a.w_scale != nullptr, a.Npad, a.Kpad, a.workspace_elems});
}

// (A wave of a tile of 256 weight rows has 128 columns, whole heads.  Not for 8-bit pools: with the conversion in it the epilogue is too
// long to be unrolled, and accumulators that are indexed at run time live in memory: 20 times the time.)
bool gemm_can_rotate(const GemmArgs& a) {
  const GemmPlan plan = plan_of(a);
  return a.epilogue == EPI_STORE && plan.splits == 1 && gemm_kernel(plan.tile, kRotating, false);
}

hipError_t launch_gemm(const GemmArgs& a, hipStream_t s) {
  if (a.M <= 0) return hipSuccess;
  GemmParams p;
  p.A = (const bf16*)a.A;
  p.W = (const bf16*)a.W;
  p.out = (bf16*)a.out;
  p.residual = a.residual;
  p.bias = a.epilogue == EPI_SWIGLU ? nullptr : a.bias;
  p.out_f32 = a.epilogue == EPI_SWIGLU && !a.w_scale ? 0 : a.out_f32;
  p.res_f32 = a.residual_f32;
  p.ws = a.workspace;
  p.a_lay = a.a_layout;
  p.w_lay = layout_weights(a.Kpad);
  p.u_lay = a.u_layout;
  p.Kpad = a.Kpad;
  p.Npad = a.Npad;
  p.ldo = a.ldo;
  p.ldr = a.ldr;
  p.M = a.M;
  p.N_store = a.N_store;
  p.epilogue = a.epilogue;
  p.k_tiles_total = (int)(a.Kpad / 64);
  const bool defer = a.splits_used != nullptr && a.epilogue != EPI_SWIGLU;
  const GemmPlan plan = plan_of(a);
  const TileInfo& ti = kTiles[plan.tile];
  const int splits = plan.splits;
  p.tiles_m = (a.M + ti.bm() - 1) / ti.bm();
  p.tiles_n = (int)(a.Npad / ti.bn());
  p.k_tiles_per_split = (p.k_tiles_total + splits - 1) / splits;
  p.splits = splits;
  p.k_tiles_per_chunk = plan.chunk;
  const bool maximum = a.row_max && splits == 1 && a.epilogue == EPI_STORE && a.out_f32 && !a.bias;
  const bool statistics = a.stats && splits == 1 && a.epilogue == EPI_STORE && a.out_f32 && !a.bias;
  if (a.row_max_width) *a.row_max_width = maximum || statistics ? ti.bn() / 2 : 0;
  const int bands = (p.tiles_m + 3) / 4;
  p.band_h = p.tiles_m / bands;
  p.n_tall = p.tiles_m % bands;
  const int tiles = p.tiles_m * p.tiles_n * splits;
  p.chunk_shift = 5 + (ti.wg_per_cu > 2 ? 2 : ti.wg_per_cu - 1);  // (an XCD's slots, or the next power of two)
  p.chunks = tiles >> (3 + p.chunk_shift);
  p.rest = tiles - (p.chunks << (3 + p.chunk_shift));
  auto inverse = [&](int64_t d) { return d > 1 && d * tiles < (1ll << 32) ? (unsigned)(((1ll << 32) + d - 1) / d) : 0u; };
  p.per_split_inv = inverse((int64_t)p.tiles_m * p.tiles_n);
  p.tall_inv = inverse((int64_t)(p.band_h + 1) * p.tiles_n);
  p.low_inv = inverse((int64_t)p.band_h * p.tiles_n);
  p.h_tall_inv = inverse(p.band_h + 1);
  p.h_low_inv = inverse(p.band_h);
  if (g_print_plan)
    fprintf(stderr, "gemm plan: M=%d N=%lld K=%lld tile=%d tiles=%dx%d splits=%d (k-tiles %d each)\n",
            a.M, (long long)a.Npad, (long long)a.Kpad, plan.tile, p.tiles_m, p.tiles_n, splits, p.k_tiles_per_split);
  dim3 grid((tiles + 7) / 8 * 8);
  // a single row of tiles reads every weight byte once: request them as non-temporal (also two rows of a
  // wide projection, see the kernel's comment)
  const bool wnt = p.tiles_m == 1 || (p.tiles_m == 2 && a.Npad >= 32768 && splits == 1);
  auto launch = [&](GemmKind kind, auto params) {
    void* args[] = {&params};
    return hipLaunchKernel(gemm_kernel(plan.tile, kind, wnt), grid, dim3(256), args, ti.lds_bytes(), s);
  };
  const GemmIntParams pi{p, a.a_scale, a.w_scale};
  hipError_t e = a.w_scale   ? (statistics ? launch(kIntStatistics, GemmIntStatsParams{pi, *a.stats}) : launch(kIntegers, pi))
                 : a.rotation ? launch(kRotating, GemmRotateParams{p, *a.rotation})
                 : statistics ? launch(kStatistics, GemmStatsParams{p, *a.stats})
                 : maximum    ? launch(kMaximum, GemmMaxParams{p, a.row_max})
                              : launch(kOrdinary, p);
  if (e != hipSuccess) return e;
  if (a.splits_used) *a.splits_used = defer ? splits : 1;
  if (splits > 1 && !defer) {
    const int out_cols = a.N_store;  // (gated epilogue: columns of the result, half the weight rows)
    const int64_t n_thr = (int64_t)a.M * (out_cols / 4);
    const unsigned blocks = (unsigned)((n_thr + 255) / 256);
    if (a.w_scale) gemm_reduce_int_kernel<<<blocks, 256, 0, s>>>(pi, out_cols);
    else gemm_reduce_kernel<<<blocks, 256, 0, s>>>(p, out_cols);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace tdp
