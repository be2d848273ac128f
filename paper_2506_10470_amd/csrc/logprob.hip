// Log-probabilities of rows of logits: of a given token of every row, the entropy of its distribution and its likeliest tokens, from
// logits in memory (logprob_rows_kernel) or from what the vocabulary projection's epilogue has noted of them (logprob_pieces_kernel).
//
// With m the largest logit of a row, s = sum e^(z - m) and t = sum (z - m) e^(z - m) (LogSum):
//   ln p_j = (z_j - m) - ln s,      entropy = - sum p ln p = ln s - t / s.
// One pass makes all three, relative to a running maximum; everything is fp32, relative to the maximum, so that no large numbers cancel.
#include <math.h>

#include "tdp_device.h"
#include "tdp_kernels.h"

namespace tdp {

typedef __attribute__((__vector_size__(4 * sizeof(unsigned)))) unsigned u32x4;

// A row of logits, in 16-byte vectors of aligned addresses: its first element may stand in the middle of one (`lead` elements of
// another row, or none at all, in front of it), and so may its last.  Vectors that the row does not fill are read element by element.
template <typename T>
struct LogitRow {
  static constexpr int kPer = 16 / sizeof(T);
  const T* base;  // aligned; element j of the row is base[lead + j]
  int lead, n;
  __device__ __forceinline__ LogitRow(const T* row, int n_) : n(n_) {
    lead = (int)(((uintptr_t)row & 15) / sizeof(T));
    base = row - lead;
  }
  __device__ __forceinline__ int vectors() const { return (lead + n + kPer - 1) / kPer; }
  __device__ __forceinline__ int index(int v, int e) const { return v * kPer + e - lead; }
  __device__ __forceinline__ void load(int v, float (&z)[kPer]) const {
    if (v * kPer >= lead && v * kPer + kPer <= lead + n) {
      const u32x4 raw = *reinterpret_cast<const u32x4*>(base + (int64_t)v * kPer);
      if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < 4; ++e) z[e] = __uint_as_float(raw[e]);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          z[2 * e] = __uint_as_float(raw[e] << 16);
          z[2 * e + 1] = __uint_as_float(raw[e] & 0xffff0000u);
        }
      }
    } else {
#pragma unroll
      for (int e = 0; e < kPer; ++e) {
        const int j = index(v, e);
        z[e] = j >= 0 && j < n ? (float)base[lead + j] : -INFINITY;
      }
    }
  }
};

// ---- the likeliest tokens ----------------------------------------------------------------------------------------------------------
// The k largest logits of a row (k <= 32), of equal ones those of lower index, in that order; a NaN is none of them.
//
// The row is in units (what a thread has read, or a piece of the projection) whose largest logits are known.  The maxima of 64 groups of
// units give a bound: the k-th largest of them, tau, has at least k logits of the row at or above it.  Only units that reach tau are
// looked at again, a few dozen of a thousand; what is above tau goes into a list, what equals it into another, and an entry's
// place in the answer is the number of entries before it.  (A list per lane that every logit is compared with, as the pass runs, costs
// several times the pass: a wave inserts some hundred times.)
// More than kAbove logits above tau (rows whose large logits are all in a few units): the k-th largest of those in the list is a higher bound,
// and the look is repeated.  More than kEqual equal to tau (a masked row with fewer than k tokens left; ties everywhere): the row is
// gone through in order for as many as are wanted.
constexpr int kTopMost = 32, kAbove = 1024, kEqual = 256, kUnits = 1024;
static_assert(kTopMost <= 64, "the bound is one of 64 maxima");

struct TopShared {
  float value[kAbove + kEqual];
  int index[kAbove + kEqual];
  int equal[kEqual];
  int units[kUnits];
  int above, equals, n_units;
  float tau;
  int found, wave_count[16];
};

// One wave: the k-th largest of its lanes' values (1 <= k <= 64).
__device__ __forceinline__ float kth_of_wave(float v, int k) {
  int before = 0;
  const int lane = threadIdx.x & 63;
#pragma unroll 8
  for (int j = 0; j < 64; ++j) {
    const float o = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), j));
    before += o > v || (o == v && j < lane) ? 1 : 0;
  }
  const unsigned long long at = __ballot(before == k - 1);
  return __shfl(v, __builtin_ctzll(at), 64);
}

// The place of entry i among the first c of the lists.
__device__ __forceinline__ int place_of(const TopShared& sh, int i, int c) {
  const float v = sh.value[i];
  const int at = sh.index[i];
  int place = 0;
  for (int j = 0; j < c; ++j) {
    const float o = sh.value[j];
    place += o > v || (o == v && sh.index[j] < at) ? 1 : 0;
  }
  return place;
}

// All threads of the workgroup (whole waves); sh.tau is set.  push(tau): puts the units that reach tau into sh.units (sh.n_units counts them, also
// past kUnits).  Unit u's vectors are u * unit_stride + j * vector_stride, j < per_unit, of n_units_all units.
// write(place, index, value) is called once for every place found; returns how many there are.
template <typename Row, typename Push, typename Write>
__device__ __forceinline__ int select_top(TopShared& sh, const Row& row, int k, int n_units_all, int per_unit, int unit_stride,
                                          int vector_stride, Push push, Write write) {
  const int tid = threadIdx.x, threads = blockDim.x, vectors = row.vectors();
  for (;;) {
    const float tau = sh.tau;
    if (tid == 0) sh.above = sh.equals = sh.n_units = 0;
    __syncthreads();
    push(tau);
    __syncthreads();
    const bool all = sh.n_units > kUnits;
    const int n_units = all ? n_units_all : sh.n_units;
    for (int64_t q = tid; q < (int64_t)n_units * per_unit; q += threads) {
      const int i = (int)(q / per_unit), j = (int)(q - (int64_t)i * per_unit);
      const int64_t v = (int64_t)(all ? i : sh.units[i]) * unit_stride + (int64_t)j * vector_stride;
      if (v >= vectors) continue;
      float z[Row::kPer];
      row.load((int)v, z);
#pragma unroll
      for (int e = 0; e < Row::kPer; ++e) {
        const int at = row.index((int)v, e);
        if (!(z[e] >= tau) || at < 0 || at >= row.n) continue;
        if (z[e] > tau) {
          const int p = atomicAdd(&sh.above, 1);
          if (p < kAbove) {
            sh.value[p] = z[e];
            sh.index[p] = at;
          }
        } else {
          const int p = atomicAdd(&sh.equals, 1);
          if (p < kEqual) sh.equal[p] = at;
        }
      }
    }
    __syncthreads();
    if (sh.above <= kAbove) break;
    for (int i = tid; i < kAbove; i += threads)
      if (place_of(sh, i, kAbove) == k - 1) sh.tau = sh.value[i];  // (one entry)
    __syncthreads();
  }
  const float tau = sh.tau;
  const int above = sh.above, equals = sh.equals;
  int c = above;
  if (above < k && equals <= kEqual) {
    for (int i = tid; i < equals; i += threads) {
      sh.value[above + i] = tau;
      sh.index[above + i] = sh.equal[i];
    }
    c = above + equals;
  } else if (above < k) {
    // in the order of the row, a logit per thread and turn
    const int wanted = k - above, wave = tid >> 6, lane = tid & 63;
    int found = 0;
    for (int64_t first = 0; first < row.n && found < wanted; first += threads) {
      const int64_t at = first + tid;
      const bool hit = at < row.n && (float)row.base[row.lead + at] == tau;
      const unsigned long long hits = __ballot(hit);
      if (lane == 0) sh.wave_count[wave] = __popcll(hits);
      __syncthreads();
      int p = found + __popcll(hits & ((1ull << lane) - 1));
      int total = 0;
      for (int w = 0; w < threads / 64; ++w) {
        if (w < wave) p += sh.wave_count[w];
        total += sh.wave_count[w];
      }
      if (hit && p < wanted) {
        sh.value[above + p] = tau;
        sh.index[above + p] = (int)at;
      }
      found += total;
      __syncthreads();
    }
    c = above + min(found, wanted);
  }
  __syncthreads();
  for (int i = tid; i < c; i += threads) {
    const int place = place_of(sh, i, c);
    if (place < k) write(place, sh.index[i], sh.value[i]);
  }
  return min(c, k);
}

// ---- a row's answer ----------------------------------------------------------------------------------------------------------------
// The threads' sums joined (every thread gets the row's); group_max: the largest logit of every lane's group, in the first wave.
// Sums of lanes, then of waves, in a fixed order: the result does not depend on the schedule.
struct JoinShared {
  LogSum wave[16], row;
  float lane_max[16][64];
};
__device__ __forceinline__ LogSum join_block(JoinShared& sh, LogSum l, float own_max, bool groups, float& group_max) {
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, waves = blockDim.x >> 6;
#pragma unroll
  for (int o = 1; o < 64; o *= 2) join(l, of_lane(l, o));
  if (waves == 1) {
    group_max = own_max;
    return l;
  }
  if (lane == 0) sh.wave[wave] = l;
  if (groups) sh.lane_max[wave][lane] = own_max;
  __syncthreads();
  if (wave == 0) {
    LogSum w = lane < waves ? sh.wave[lane] : no_logits();
#pragma unroll
    for (int o = 1; o < 16; o *= 2) join(w, of_lane(w, o));
    if (lane == 0) sh.row = w;
    if (groups)
      for (int i = 0; i < waves; ++i) group_max = i == 0 ? sh.lane_max[0][lane] : fmaxf(group_max, sh.lane_max[i][lane]);
  }
  __syncthreads();
  return sh.row;
}

// The sums, and the tokens if any are wanted (TOP: only then has the workgroup the memory for them); shared by both kernels.
template <bool TOP, typename Row, typename Push>
__device__ __forceinline__ void answer_row(const LogprobArgs& a, JoinShared& js, TopShared* ts, const Row& row, const LogSum& own, float own_max,
                                           float target_logit, bool has_target, int n_units_all, int per_unit, int unit_stride,
                                           int vector_stride, Push push) {
  const int m = blockIdx.x, tid = threadIdx.x;
  float group_max = -INFINITY;
  const LogSum l = join_block(js, own, own_max, TOP, group_max);
  const float log_sum = logf(l.sum);
  if (tid == 0) {
    if (a.logprob) a.logprob[m] = !a.targets ? -log_sum + 0.f * l.max : has_target ? (target_logit - l.max) - log_sum : -INFINITY;
    if (a.entropy) a.entropy[m] = log_sum - l.weighted / l.sum;
  }
  if constexpr (!TOP) return;
  const int k = max(a.n_top, a.next_token ? 1 : 0);
  if (tid < 64) {
    const float tau = kth_of_wave(group_max, k);
    if (tid == 0) ts->tau = tau;
  }
  __syncthreads();
  const int found = select_top(*ts, row, k, n_units_all, per_unit, unit_stride, vector_stride, push, [&](int place, int index, float value) {
    if (place == 0 && a.next_token) a.next_token[m] = index;
    if (place < a.n_top) {
      a.top_index[(int64_t)m * a.n_top + place] = index;
      a.top_logprob[(int64_t)m * a.n_top + place] = (value - l.max) - log_sum;
    }
  });
  for (int place = found + tid; place < a.n_top; place += blockDim.x) {  // (a row with fewer logits that are numbers)
    a.top_index[(int64_t)m * a.n_top + place] = -1;
    a.top_logprob[(int64_t)m * a.n_top + place] = NAN;
  }
  if (found == 0 && tid == 0 && a.next_token) a.next_token[m] = 0;
}

// One workgroup per row, every logit read once, kInFlight vectors of a thread at a time.
constexpr int kInFlight = 4;
template <typename T, bool TOP>
__global__ __launch_bounds__(1024) void logprob_rows_kernel(const T* __restrict__ logits, int64_t ld, int n, const LogprobArgs a) {
  __shared__ JoinShared js;
  TopShared* ts = nullptr;
  if constexpr (TOP) {
    __shared__ TopShared top;
    ts = &top;
  }
  const int m = blockIdx.x, tid = threadIdx.x, threads = blockDim.x;
  typedef LogitRow<T> Row;
  const Row row(logits + (int64_t)m * ld, n);
  const int vectors = row.vectors();
  LogSum l = no_logits();
  for (int64_t v0 = tid; v0 < vectors; v0 += (int64_t)threads * kInFlight) {
    float z[kInFlight][Row::kPer];
#pragma unroll
    for (int u = 0; u < kInFlight; ++u) {
      const int64_t v = v0 + (int64_t)u * threads;
      if (v < vectors) {
        row.load((int)v, z[u]);
      } else {
#pragma unroll
        for (int e = 0; e < Row::kPer; ++e) z[u][e] = -INFINITY;
      }
    }
    float max = l.max;
#pragma unroll
    for (int u = 0; u < kInFlight; ++u)
#pragma unroll
      for (int e = 0; e < Row::kPer; ++e) max = fmaxf(max, z[u][e]);
    if (max > l.max) raise(l, max);
#pragma unroll
    for (int u = 0; u < kInFlight; ++u)
#pragma unroll
      for (int e = 0; e < Row::kPer; ++e) add_logit(l, z[u][e]);
  }
  const int target = a.targets ? a.targets[m] : -1;
  const bool has_target = target >= 0 && target < n;
  const float own_max = l.max;
  answer_row<TOP>(a, js, ts, row, l, own_max, has_target ? (float)logits[(int64_t)m * ld + target] : 0.f, has_target, threads,
             (vectors + threads - 1) / threads, 1, threads, [&](float tau) {
               if (own_max >= tau) ts->units[atomicAdd(&ts->n_units, 1)] = tid;  // (at most 1024)
             });
}

// One workgroup per row: the pieces' sums are joined; logits are read again for tokens alone.
template <bool TOP>
__global__ __launch_bounds__(256) void logprob_pieces_kernel(const RowStatistics st, int count, int width, const float* __restrict__ logits,
                                                             int64_t ld, int n, const LogprobArgs a) {
  __shared__ JoinShared js;
  TopShared* ts = nullptr;
  if constexpr (TOP) {
    __shared__ TopShared top;
    ts = &top;
  }
  const int m = blockIdx.x, tid = threadIdx.x, threads = blockDim.x;
  const int64_t first = (int64_t)m * count;
  LogSum l = no_logits();
  for (int i = tid; i < count; i += threads) join(l, LogSum{st.max[first + i], st.sum[first + i], st.weighted[first + i]});
  const LogitRow<float> row(logits + (int64_t)m * ld, n);
  const int target = a.targets ? a.targets[m] : -1;
  const bool has_target = target >= 0 && target < n;
  answer_row<TOP>(a, js, ts, row, l, l.max, has_target ? st.target_logit[m] : 0.f, has_target, count, width / 4, width / 4, 1, [&](float tau) {
    for (int i = tid; i < count; i += threads)
      if (st.max[first + i] >= tau) {
        const int p = atomicAdd(&ts->n_units, 1);
        if (p < kUnits) ts->units[p] = i;
      }
  });
}

hipError_t launch_logprob_rows(const void* logits, int logits_are_bf16, int64_t ld, int M, int n, const LogprobArgs& a, hipStream_t s) {
  if (M <= 0) return hipSuccess;
  const int64_t vectors = ((int64_t)n * (logits_are_bf16 ? 2 : 4) + 15) / 16;
  const int threads = vectors >= 4096 ? 1024 : vectors >= 1024 ? 512 : vectors >= 256 ? 256 : 64;
  const bool top = a.n_top > 0 || a.next_token;
#define TDP_ROWS(T, TOP) logprob_rows_kernel<T, TOP><<<M, threads, 0, s>>>((const T*)logits, ld, n, a)
  if (logits_are_bf16) {
    if (top) TDP_ROWS(bf16, true);
    else TDP_ROWS(bf16, false);
  } else {
    if (top) TDP_ROWS(float, true);
    else TDP_ROWS(float, false);
  }
#undef TDP_ROWS
  return hipGetLastError();
}

hipError_t launch_logprob_pieces(const RowStatistics& st, int count, int width, const float* logits, int64_t ld, int M, int n,
                                 const LogprobArgs& a, hipStream_t s) {
  if (M <= 0) return hipSuccess;
  if (a.n_top > 0 || a.next_token) logprob_pieces_kernel<true><<<M, 256, 0, s>>>(st, count, width, logits, ld, n, a);
  else logprob_pieces_kernel<false><<<M, 256, 0, s>>>(st, count, width, logits, ld, n, a);
  return hipGetLastError();
}

}  // namespace tdp
