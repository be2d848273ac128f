// The n_out best continuations of every group of beams, from rows of logits: score of the beam + ln softmax of its row.
//
// Two launches.  The first reads the logits once: a workgroup has a piece of a row (a whole row where there are many), notes its largest logit,
// the sum of exponentials relative to that, and its n_out largest logits in order.  Within a row, candidates are in the order of
// the logits, so nothing else of the row can be chosen.  The second has a workgroup to a group: it joins the sums of every row and ranks the
// candidates of all beams.
//
// Scores of different beams are often close, and which token goes on depends on their order, so what is compared is in 64 bits.  Only the
// exponentials are formed in fp32: relative to the largest logit m of the piece, t = z - m and e^t = 2^(t log2 e) with log2 e in two parts.  The
// largest logit's own term is 1 and nothing else (a row held to one token costs exactly nothing), and rows that differ by a constant have
// the same t, the same sums and the same costs to the bit.  Of any other term t and the exponent are rounded by 2^-24 of themselves, each |t| 2^-24 of
// the term, and the instruction's error is 1 ulp: (1 + |t|) 2^-23 in all.  Terms are added in 64 bits, so ln sum is off by at most
//   2^-23 sum_{z < m} p (1 + m - z),     p the tokens' probabilities:
// nothing of what the likeliest token carries but the additions' 2^-53 each.  (Errors of many different logits largely cancel; those of equal
// logits are equal.)  Measured on 65536 rows of two tokens, up to 86 apart: half of that at most.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>
#include <stdio.h>

#include <algorithm>
#include <new>
#include <type_traits>

#include "../../include/tdp.h"
#include "logit_rows.h"
#include "tdp_device.h"
#include "tdp_kernels.h"

namespace tdp {

int probe_fail(int code, const char* msg);  // sets the thread's error message (stage.hip)

namespace {

typedef unsigned long long u64;
constexpr int kInFlight = 8;    // vectors of a thread
constexpr int kListsMost = 1024;  // of a group
constexpr int kPiecesMost = 64, kPiecesOfMany = 8;
constexpr int kIndexBits = 27;  // of a token, beside 5 of a beam and 32 of a logit's order
static_assert(TDP_MAX_BEAMS <= 32 && TDP_MAX_BEAMS * kPiecesOfMany <= kListsMost && TDP_MAX_TOP <= kTopMost, "what the second kernel holds");

struct BeamArgs {
  int beams, n, width, pieces, k;  // width: columns of a piece
  const int32_t* finished;
  int end_token;
  const float* scores;
  // per (row, piece)
  float* max;
  double* sum;  // relative to it
  u64* keys;  // [k], in order, 0 behind the last
  int32_t *parent, *token;
  float* score;
  int32_t* finished_out;
};

constexpr float kLog2High = 1.44269502f, kLog2Low = 1.92596299e-8f;  // log2 e
// e^(z - m), 1 where they are equal
__device__ __forceinline__ float exp_below(float z, float m) {
  const float t = z - m;
  return __builtin_amdgcn_exp2f(__builtin_fmaf(t, kLog2High, t * kLog2Low));
}

// A piece of a row in vectors from its first element on, wherever that lies in memory: which terms a thread adds up, and with them
// the bits of the sum, do not depend on it, so that beams that are alike are equal.  What is left behind the last whole vector is the first
// threads', an element each.
typedef u32x4 __attribute__((aligned(4))) u32x4_of_float;
typedef u32x4 __attribute__((aligned(2))) u32x4_of_bf16;
template <typename T>
struct BeamRow {
  static constexpr int kPer = 16 / sizeof(T);
  typedef typename std::conditional<sizeof(T) == 4, u32x4_of_float, u32x4_of_bf16>::type Anywhere;
  const T* first;
  int n, body;
  __device__ __forceinline__ BeamRow(const T* row, int n_) : first(row), n(n_), body(n_ / kPer) {}
  __device__ __forceinline__ int index(int v, int e) const { return v * kPer + e; }
  __device__ __forceinline__ u32x4 load(int v) const { return *reinterpret_cast<const Anywhere*>(first + (int64_t)v * kPer); }
  __device__ __forceinline__ float at(int i) const { return (float)first[i]; }
  __device__ __forceinline__ int edge(int tid) const { return body * kPer + tid < n ? body * kPer + tid : -1; }
};

__device__ __forceinline__ double wave_sum_double(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// KEEP: a thread has eight vectors at most and keeps them in registers; else the piece is read twice, and the tokens of threads whose
// largest logit is among the wanted a third time.  Bound: reading, 512 rows of 32000 fp32 logits 18.3 us (65.5 MB, 3.6 TB/s with the beginning and
// the end of two workgroups a CU), 528 of 152067 in bf16, a quarter of them finished, 38 to 39 us (120 MB, 3.1 TB/s): beside it a maximum, an exponential, an
// addition in 64 bits and a comparison to a logit.  (Terms added in fp32 per thread 17.9 and 36 us, in pairs 18.2 and 38; a sum so formed
// is off by 2^-24 of what the likeliest token carries.)
template <typename T, bool KEEP>
__global__ __launch_bounds__(1024, 8) void beams_piece_kernel(const T* __restrict__ logits, int64_t ld, int shift, const BeamArgs a) {
  __shared__ RowShared rs;
  __shared__ TopShared ts;
  __shared__ double wave_total[16];
  extern __shared__ __attribute__((aligned(16))) unsigned char staged_raw[];  // (KEEP) StagedUnits of every wave
  StagedUnits& staged = reinterpret_cast<StagedUnits*>(staged_raw)[threadIdx.x >> 6];
  const int tid = threadIdx.x, threads = blockDim.x, wave = tid >> 6, lane = tid & 63, waves = threads >> 6;
  const int slot = blockIdx.x, m = slot / a.pieces, piece = slot - m * a.pieces;
  u64* const keys = a.keys + (int64_t)slot * a.k;
  if (a.finished && a.finished[m]) {  // the end token alone, at no cost
    for (int i = tid; i < a.k; i += threads) keys[i] = piece == 0 && i == 0 ? key_of(0.f, a.end_token) : 0;
    if (tid == 0) {
      a.max[slot] = piece == 0 ? 0.f : -INFINITY;
      a.sum[slot] = piece == 0 ? 1.0 : 0.0;
    }
    return;
  }
  typedef LogitRow<T> Values;
  typedef BeamRow<T> Row;
  constexpr int kPer = Row::kPer;
  const int first = piece * a.width;
  const Row row(logits + (int64_t)m * ld + first, min(a.width, a.n - first));
  u32x4 z[kInFlight];
  auto fetch = [&](int v0) {
#pragma unroll
    for (int u = 0; u < kInFlight; ++u) z[u] = v0 + u * threads < row.body ? row.load(v0 + u * threads) : Values::nothing();
  };
  float own_max = -INFINITY;
  auto take_max = [&] {
#pragma unroll
    for (int u = 0; u < kInFlight; ++u)
#pragma unroll
      for (int e = 0; e < kPer; ++e) own_max = fmaxf(own_max, Values::value(z[u], e));
  };
  const int edge_at = row.edge(tid);
  if constexpr (KEEP) fetch(tid);
  const float edge = edge_at >= 0 ? row.at(edge_at) : -INFINITY;
  if constexpr (KEEP) {
    take_max();
  } else {
#pragma unroll 1
    for (int v0 = tid; v0 < row.body; v0 += threads * kInFlight) {
      fetch(v0);
      take_max();
    }
  }
  // the maximum of all, and on the way those of 64 groups of lanes
  float v = fmaxf(own_max, edge);
  auto group = [&](int size) {
    if (waves == size && (lane & (size - 1)) == size - 1) rs.group_max[wave * (64 / size) + lane / size] = v;
  };
  group(1);
  v = fmaxf(v, from_front<kDppShift1, 0xf>(v, v));
  group(2);
  v = fmaxf(v, from_front<kDppShift2, 0xf>(v, v));
  group(4);
  v = fmaxf(v, from_front<kDppShift4, 0xf>(v, v));
  group(8);
  v = fmaxf(v, from_front<kDppShift8, 0xf>(v, v));
  group(16);
  v = fmaxf(v, from_front<kDppLast15, 0xa>(v, v));
  v = fmaxf(v, from_front<kDppLast31, 0xc>(v, v));
  if (lane == 63) rs.wave_max[wave] = v;
  if (tid == 0) ts.listed = 0;
  __syncthreads();
  float max = rs.wave_max[0];
  for (int w = 1; w < waves; ++w) max = fmaxf(max, rs.wave_max[w]);
  // Sums relative to it (to 0 where nothing is above minus infinity).
  const float r = max == -INFINITY ? 0.f : max;
  double total = edge_at >= 0 ? (double)exp_below(edge, r) : 0.0;
  auto add = [&](int v0) {
#pragma unroll
    for (int u = 0; u < kInFlight; ++u) {
      if (u > 0 && v0 - tid + u * threads >= row.body) break;  // (the same for all threads)
      asm volatile("" : "+v"(z[u]));  // (bf16: converted here again, the values of two passes would not fit)
#pragma unroll
      for (int e = 0; e < kPer; ++e) total += (double)exp_below(Values::value(z[u], e), r);
    }
  };
  if constexpr (KEEP) {
    add(tid);
  } else {
#pragma unroll 1
    for (int v0 = tid; v0 < row.body; v0 += threads * kInFlight) {
      fetch(v0);
      add(v0);
    }
  }
  total = wave_sum_double(total);
  if (lane == 0) wave_total[wave] = total;
  __syncthreads();
  if (tid == 0) {
    for (int w = 1; w < waves; ++w) total += wave_total[w];
    a.max[slot] = max;
    a.sum[slot] = total;
  }
  const int found = select_top(
      rs, ts, row, max, min(a.k, row.n), edge, edge_at, 1, shift, [&](int) { return own_max; },
      [&](int, int at) {
        ts.units[wave][at] = tid;
        if constexpr (KEEP) {
#pragma unroll
          for (int u = 0; u < kInFlight; ++u) staged[at][u] = z[u];
        }
      },
      [&](int at_slot, int j, int& at) {
        const int vec = ts.units[wave][at_slot] + j / kPer * threads;
        if (vec >= row.body) return 0.f;
        at = row.index(vec, j % kPer);
        if constexpr (KEEP) {
          const unsigned* const p = reinterpret_cast<const unsigned*>(staged[at_slot]);
          if constexpr (sizeof(T) == 4) return __uint_as_float(p[j]);
          else return __uint_as_float(j & 1 ? p[j / 2] & 0xffff0000u : p[j / 2] << 16);
        } else {
          return row.at(at);
        }
      },
      [&](int place, int index, float value) { keys[place] = key_of(value, first + index); });
  for (int i = found + tid; i < a.k; i += threads) keys[i] = 0;
}

// A candidate's place among all of its group as two whole numbers, the larger the better: its score, 0 for none, and what decides
// between equal ones.
struct Candidate {
  u64 score, rest;
};
__device__ __forceinline__ bool better(const Candidate& x, const Candidate& y) {
  return x.score > y.score || (x.score == y.score && x.rest > y.rest);
}
__device__ __forceinline__ double score_of(u64 order) {
  return __longlong_as_double((long long)(order ^ (order >> 63 ? 1ull << 63 : ~0ull)));
}

// One workgroup per group, of 256 threads (64 candidates at most) or 1024.  `lists` = beams * pieces lists of k candidates, each in order.  Up to
// kAllRanked of them are all ranked at once.  Otherwise the first `heads` of every list, n_out in all or more, give a bound, the n_out-th best
// of them: a list goes on behind its heads only if all of them reach it, so at most n_out / heads lists do, and n_out * k / heads <= 1024
// candidates reach it, a few dozen as a rule.
// Bound: look-ups that wait for each other (three) and barriers: 16 candidates 4 us, 64 groups of 128 5 us, 33 of 1280 8 us.
constexpr int kAllRanked = 256;
template <int THREADS>
__global__ __launch_bounds__(THREADS) void beams_group_kernel(const BeamArgs a) {
  __shared__ double largest[TDP_MAX_BEAMS], log_total[TDP_MAX_BEAMS];  // of a row's logits; of its sum relative to that
  __shared__ Candidate pool[kListsMost];
  __shared__ Candidate bound;
  __shared__ int count, places[kListsMost];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, g = blockIdx.x;
  const int64_t slot0 = (int64_t)g * a.beams * a.pieces;
  const int lists = a.beams * a.pieces, all = lists * a.k, n_out = a.k;
  const u64 own_key = tid < all ? a.keys[slot0 * a.k + tid] : 0;  // (asked for with the sums)
  const float own_score = tid < all ? a.scores[(int64_t)g * a.beams + tid / (a.pieces * a.k)] : 0.f;
  for (int b = wave; b < a.beams; b += THREADS / 64) {
    const bool in = lane < a.pieces;
    const int64_t slot = slot0 + b * a.pieces + lane;
    const float own = in ? a.max[slot] : -INFINITY;
    const double sum = in ? a.sum[slot] : 0.0;
    float max = own;
    for (int o = 1; o < 64; o *= 2) max = fmaxf(max, __shfl_xor(max, o, 64));
    // (of a piece with nothing but minus infinity and NaN the sum alone counts: 0, or NaN)
    const double total = wave_sum_double(own == -INFINITY ? sum : sum * exp((double)own - (double)max));
    if (lane == 0) {
      largest[b] = (double)max;
      log_total[b] = max == -INFINITY ? NAN : log(total);
    }
  }
  if (tid == 0) {
    bound = Candidate{0, 0};
    count = 0;
  }
  for (int i = tid; i < kListsMost; i += THREADS) places[i] = 0;
  __syncthreads();
  auto candidate = [&](u64 key, float score, int beam) {
    if (!key) return Candidate{0, 0};
    const unsigned order = (unsigned)(key >> 32);
    const double c = (double)score + (((double)logit_of(order) - largest[beam]) - log_total[beam]);
    if (!(c > -INFINITY)) return Candidate{0, 0};
    const long long bits = __double_as_longlong(c + 0.0);
    return Candidate{(u64)bits ^ (bits < 0 ? ~0ull : 1ull << 63),
                     (u64)(31 - beam) << 59 | (u64)order << kIndexBits | ((unsigned)key & ((1u << kIndexBits) - 1))};
  };
  auto candidate_at = [&](int i) { return candidate(a.keys[slot0 * a.k + i], a.scores[(int64_t)g * a.beams + i / (a.pieces * a.k)], i / (a.pieces * a.k)); };
  // places[i] = how many of the pool's n are better than its i-th: all pairs, shared out over the threads; behind a barrier on both sides
  auto rank_all = [&](int n) {
    int shift = 6;
    while ((1 << shift) < n) ++shift;
    const int i = tid & ((1 << shift) - 1), parts = THREADS >> shift;
    if (i < n) {
      const Candidate c = pool[i];
      int r = 0;
#pragma unroll 4
      for (int j = tid >> shift; j < n; j += parts) r += better(pool[j], c);
      if (r) atomicAdd(&places[i], r);
    }
    __syncthreads();
  };
  const Candidate own = candidate(own_key, own_score, tid / (a.pieces * a.k));
  int n = all, found;  // candidates in the pool, and those among them that are some
  if (all <= kAllRanked) {
    if (tid < all) pool[tid] = own;
    found = __syncthreads_count(own.score != 0);
  } else {
    const int heads = (a.k + lists - 1) / lists, some = lists * heads;
    for (int i = tid; i < some; i += THREADS) pool[i] = candidate_at(i / heads * a.k + i % heads);
    __syncthreads();
    rank_all(some);
    for (int i = tid; i < some; i += THREADS) {
      if (pool[i].score && places[i] == a.k - 1) bound = pool[i];  // (no two are equal)
      places[i] = 0;
    }
    __syncthreads();
    const Candidate least = bound;
    for (int i = tid; i < all; i += THREADS) {
      const Candidate c = i == tid ? own : candidate_at(i);
      if (c.score && !better(least, c)) pool[atomicAdd(&count, 1)] = c;
    }
    __syncthreads();
    n = found = count;
  }
  rank_all(n);
  for (int i = tid; i < n; i += THREADS) {
    const Candidate c = pool[i];
    const int place = places[i];
    if (!c.score || place >= n_out) continue;
    const int64_t at = (int64_t)g * n_out + place;
    const int token = (int)(~c.rest & ((1u << kIndexBits) - 1));
    a.parent[at] = g * a.beams + 31 - (int)(c.rest >> 59);
    a.token[at] = token;
    a.score[at] = (float)score_of(c.score);
    if (a.finished_out) a.finished_out[at] = token == a.end_token;
  }
  for (int i = found + tid; i < n_out; i += THREADS) {
    const int64_t at = (int64_t)g * n_out + i;
    a.parent[at] = a.token[at] = -1;
    a.score[at] = -INFINITY;
    if (a.finished_out) a.finished_out[at] = 0;
  }
}

int fail_hip(hipError_t e, const char* what) {
  char buf[200];
  snprintf(buf, sizeof buf, "%s: %s", what, hipGetErrorString(e));
  return probe_fail(e == hipErrorOutOfMemory ? TDP_ENOMEM : TDP_EHIP, buf);
}

// How a row is cut.  A few rows into enough pieces that they keep the chip busy, of some thousand logits at least (the second kernel ranks
// candidates of every piece: 2 groups of 5 beams, 128256 logits, 31 / 25 pieces 19.1 / 17.3 us, the caches emptied in front).  Many into
// pieces that the registers of a workgroup of 1024 threads hold, as long as they are not too many; bf16, twice as many logits to a thread, of
// 512 (528 rows of 152067, the pass of two inputs in turn: 3 pieces 48 us, 5 of half the threads 39; fp32, 5 pieces 58 us, 8 smaller ones 70).
struct Cut {
  int pieces, threads;
};
Cut cut_of(int rows, int n, int per) {
  const int most = per == 4 ? 1024 : 512;
  const int full = (n + per * kInFlight * most - 1) / (per * kInFlight * most);
  const int wanted = std::min({kPiecesMost, kListsMost / 4 / rows, n / (per * 1024)});
  const int pieces = std::max(1, std::max(std::min(full, kPiecesOfMany), wanted));
  const int vectors = ((n + pieces - 1) / pieces + per - 1) / per;
  int threads = 64;  // four vectors to a thread, eight at most if 1024 are enough for that
  while (threads < 1024 && threads * (threads < most ? 4 : kInFlight) < vectors) threads *= 2;
  return {pieces, threads};
}

size_t slots_of(int max_rows) { return std::max<size_t>(kListsMost, (size_t)kPiecesOfMany * max_rows); }

}  // namespace
}  // namespace tdp

using namespace tdp;

struct tdp_beams {
  tdp_beams_config cfg;
  int device = 0;
  float* max = nullptr;
  double* sum = nullptr;
  u64* keys = nullptr;
};

extern "C" {

int tdp_beams_create(const tdp_beams_config* cfg, tdp_beams** out) {
  if (!cfg || !out) return probe_fail(TDP_EINVAL, "null pointer");
  if (cfg->max_rows < 1 || cfg->max_rows > (1 << 16)) return probe_fail(TDP_EINVAL, "max_rows must be 1 .. 2^16");
  if (cfg->max_out < 1 || cfg->max_out > TDP_MAX_TOP) return probe_fail(TDP_EINVAL, "max_out must be 1 .. TDP_MAX_TOP");
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess) return probe_fail(TDP_EHIP, "no HIP device");
  tdp_beams* h = new (std::nothrow) tdp_beams();
  if (!h) return probe_fail(TDP_ENOMEM, "host allocation failed");
  h->cfg = *cfg;
  h->device = dev;
  const size_t slots = slots_of(cfg->max_rows);
  hipError_t e = hipMalloc((void**)&h->max, slots * sizeof(float));
  if (e == hipSuccess) e = hipMalloc((void**)&h->sum, slots * sizeof(double));
  if (e == hipSuccess) e = hipMalloc((void**)&h->keys, slots * cfg->max_out * sizeof(u64));
  if (e != hipSuccess) {
    const int code = fail_hip(e, "tdp_beams_create");
    tdp_beams_destroy(h);
    return code;
  }
  *out = h;
  return TDP_OK;
}

void tdp_beams_destroy(tdp_beams* h) {
  if (!h) return;
  (void)hipDeviceSynchronize();
  void* ptrs[] = {h->max, h->sum, h->keys};
  for (void* p : ptrs)
    if (p) (void)hipFree(p);
  delete h;
}

int tdp_beams_select(tdp_beams* h, const void* logits, int32_t dtype, int32_t n_groups, int32_t beams, int32_t n, int64_t ld,
                     const float* scores, const int32_t* finished, int32_t end_token, int32_t n_out, int32_t* parent, int32_t* token,
                     float* score, int32_t* finished_out, void* stream) {
  if (!h) return probe_fail(TDP_EINVAL, "null beams object");
  if (dtype != TDP_F32 && dtype != TDP_BF16) return probe_fail(TDP_EINVAL, "dtype must be TDP_F32 or TDP_BF16");
  if (n_groups < 0 || n < 1 || n > (1 << kIndexBits) || ld < n) return probe_fail(TDP_EINVAL, "bad shape");
  if (beams < 1 || beams > TDP_MAX_BEAMS) return probe_fail(TDP_EINVAL, "beams must be 1 .. TDP_MAX_BEAMS");
  if (n_out < 1 || n_out > h->cfg.max_out || n_out > (int64_t)beams * n) return probe_fail(TDP_EINVAL, "n_out must be 1 .. max_out and at most beams * n");
  if ((int64_t)n_groups * beams > h->cfg.max_rows) return probe_fail(TDP_EINVAL, "rows exceed max_rows");
  if (end_token >= n || end_token < (finished ? 0 : -1)) return probe_fail(TDP_EINVAL, "end_token must be a token, or -1 where no beam can be finished");
  if (n_groups == 0) return TDP_OK;
  if (!logits || !scores || !parent || !token || !score) return probe_fail(TDP_EINVAL, "null pointer");
  if ((uintptr_t)logits & (dtype == TDP_F32 ? 3 : 1)) return probe_fail(TDP_EINVAL, "logits must be aligned to their type");
  // (scores are read while results of other groups are written; everything else is read in front of them)
  const int64_t results = 4ll * n_groups * n_out;
  const Range in[] = {{scores, 4ll * n_groups * beams}}, out[] = {{parent, results}, {token, results}, {score, results}, {finished_out, results}};
  if (any_meet(in, out)) return probe_fail(TDP_EINVAL, "outputs must not overlap the scores or one another");
  int dev = -1;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return fail_hip(e, "hipGetDevice");
  if (dev != h->device) return probe_fail(TDP_EINVAL, "the object was created on another device than the current one");
  hipStream_t s = (hipStream_t)stream;
  const int rows = n_groups * beams, per = dtype == TDP_F32 ? 4 : 8;
  const Cut cut = cut_of(rows, n, per);
  const int width = ((n + cut.pieces - 1) / cut.pieces + 7) / 8 * 8, used = (n + width - 1) / width;
  const int vectors = (std::min(width, n) + per - 1) / per, threads = cut.threads;
  const bool keep = vectors <= threads * kInFlight;
  int shift = 0;  // of the elements that a thread has read
  while ((1 << shift) < (vectors + threads - 1) / threads * per) ++shift;
  const BeamArgs a{beams, n, width, used, n_out, finished, end_token, scores, h->max, h->sum, h->keys, parent, token, score, finished_out};
  const unsigned grid = (unsigned)rows * used;
  const size_t lds = keep ? threads / 64 * sizeof(StagedUnits) : 0;
#define TDP_PIECES(T, KEEP) beams_piece_kernel<T, KEEP><<<grid, threads, lds, s>>>((const T*)logits, ld, shift, a)
  if (dtype == TDP_F32) {
    if (keep) TDP_PIECES(float, true); else TDP_PIECES(float, false);
  } else {
    if (keep) TDP_PIECES(bf16, true); else TDP_PIECES(bf16, false);
  }
#undef TDP_PIECES
  if (beams * used * n_out <= 64) beams_group_kernel<256><<<n_groups, 256, 0, s>>>(a);
  else beams_group_kernel<1024><<<n_groups, 1024, 0, s>>>(a);
  e = hipGetLastError();
  return e == hipSuccess ? TDP_OK : fail_hip(e, "tdp_beams_select");
}

}  // extern "C"
