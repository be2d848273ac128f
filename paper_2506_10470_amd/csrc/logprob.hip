// Log-probabilities of rows of logits: of a given token of every row, the entropy of its distribution and its likeliest tokens, from
// logits in memory (logprob_rows_kernel) or from what the vocabulary projection's epilogue has noted of them (logprob_pieces_kernel).
// The numbers that both make of a row, and what they mean: LogSum (tdp_device.h).
#include <math.h>

#include "logit_rows.h"
#include "tdp_device.h"
#include "tdp_kernels.h"

namespace tdp {

// ---- a row's answer ----------------------------------------------------------------------------------------------------------------
// The threads' sums joined, and the tokens if any are wanted (TOP: only then has the workgroup the memory for them); shared by both kernels.
// The order of the sums is fixed: a result does not depend on the schedule.
template <bool TOP, typename Row, typename Largest, typename Stage, typename Element>
__device__ __forceinline__ void answer_row(const LogprobArgs& a, RowShared& rs, TopShared* ts, const Row& row, LogSum l, float target_logit,
                                           bool has_target, float edge, int edge_at, int turns, int shift, Largest largest_of, Stage stage,
                                           Element element) {
  const int m = blockIdx.x, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, waves = blockDim.x >> 6;
  // the wave's maximum, and on the way those of groups of as many lanes as there are waves: 64 of them in all
  float v = l.max;
  auto group = [&](int size) {
    if (TOP && waves == size && (lane & (size - 1)) == size - 1) rs.group_max[wave * (64 / size) + lane / size] = v;
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
  raise(l, of_last(v, 63));
  l.sum = whole_sum(l.sum);
  l.weighted = whole_sum(l.weighted);
  if (TOP && tid == 0) ts->listed = 0;
  if (waves > 1) {
    if (lane == 0) {
      rs.wave_max[wave] = l.max;
      rs.wave_sum[wave] = l.sum;
      rs.wave_weighted[wave] = l.weighted;
    }
    __syncthreads();
    // every wave joins the waves' sums: one to a lane, in rows of 16
    const int w = lane & 15;
    l = w < waves ? LogSum{rs.wave_max[w], rs.wave_sum[w], rs.wave_weighted[w]} : no_logits();
    v = l.max;
    v = fmaxf(v, from_front<kDppShift1, 0xf>(v, v));
    v = fmaxf(v, from_front<kDppShift2, 0xf>(v, v));
    v = fmaxf(v, from_front<kDppShift4, 0xf>(v, v));
    v = fmaxf(v, from_front<kDppShift8, 0xf>(v, v));
    raise(l, of_last(v, 15));
    l.sum = of_last(row_sum(l.sum), 15);
    l.weighted = of_last(row_sum(l.weighted), 15);
  } else if (TOP) {
    __syncthreads();
  }
  const float log_sum = logf(l.sum);
  auto logprob = [&](float z) { return (z - l.max) - log_sum; };
  if (tid == 0) {
    if (a.logprob) a.logprob[m] = a.targets && !has_target ? -INFINITY : logprob(a.targets ? target_logit : l.max);
    if (a.entropy) a.entropy[m] = log_sum - l.weighted / l.sum;
  }
  if constexpr (TOP) {
    const int k = max(a.n_top, a.next_token ? 1 : 0);
    auto write = [&](int place, int index, float value) {
      if (place == 0 && a.next_token) a.next_token[m] = index;
      if (place < a.n_top) {
        a.top_index[(int64_t)m * a.n_top + place] = index;
        a.top_logprob[(int64_t)m * a.n_top + place] = logprob(value);
      }
    };
    const int found = select_top(rs, *ts, row, l.max, k, edge, edge_at, turns, shift, largest_of, stage, element, write);
    for (int place = found + tid; place < a.n_top; place += blockDim.x) {  // (a row with fewer logits that are numbers)
      a.top_index[(int64_t)m * a.n_top + place] = -1;
      a.top_logprob[(int64_t)m * a.n_top + place] = NAN;
    }
    if (found == 0 && tid == 0 && a.next_token) a.next_token[m] = 0;
  }
}

// One workgroup per row, every logit read once.  A thread owns every `threads`-th vector.  KEEP: it has at most eight, and keeps them in
// registers for the tokens; else any number, eight at a time, and those of threads whose largest logit is wanted are read again.  What
// each turn of eight adds is then a sum of its own, and the sum of those is kept in two numbers: in one, like terms are rounded
// alike time after time, and a row of 2^24 was off by 2e-4 where a chain of 64 is by 4e-6 at most.
constexpr int kInFlight = 8;
// NT: the loads are marked non-temporal, from 240 MiB on, what the memory-side cache cannot hold beside anything else (1 GB of bf16: 180
// -> 172 us, 263 MB of fp32: 46 -> 41); below that logits that a projection has just written may still be there.
template <typename T, bool TOP, bool KEEP, bool NT, bool PARTS>
__global__ __launch_bounds__(1024, 8) void logprob_rows_kernel(const T* __restrict__ logits, int64_t ld, int n, int parts, int64_t stride,
                                                               int shift, const LogprobArgs a) {
  __shared__ RowShared rs;
  TopShared* ts = nullptr;
  if constexpr (TOP) {
    __shared__ TopShared top;
    ts = &top;
  }
  extern __shared__ __attribute__((aligned(16))) unsigned char staged_raw[];  // (TOP and KEEP) StagedUnits of every wave
  StagedUnits& staged = reinterpret_cast<StagedUnits*>(staged_raw)[threadIdx.x >> 6];
  const int m = blockIdx.x, tid = threadIdx.x, threads = blockDim.x;
  typedef LogitRow<T, PARTS> Row;
  constexpr int kPer = Row::kPer;
  Row row(logits + (int64_t)m * ld, n);
  if constexpr (PARTS) {
    row.parts = parts;
    row.stride = stride;
  }
  LogSum l = no_logits();
  float lost_sum = 0.f, lost_weighted = 0.f;
  u32x4 z[kInFlight];
  auto fetch = [&](int v0) {
#pragma unroll
    for (int u = 0; u < kInFlight; ++u) z[u] = v0 + u * threads < row.body ? row.template load<NT>(v0 + u * threads) : Row::nothing();
  };
  auto add = [&](int v0) {
    float max = l.max;
#pragma unroll
    for (int u = 0; u < kInFlight; ++u)
#pragma unroll
      for (int e = 0; e < kPer; ++e) max = fmaxf(max, Row::value(z[u], e));
    if (max > l.max) {
      if constexpr (!KEEP) take_in(l, lost_sum, lost_weighted);
      raise(l, max);
    }
    const float r = reference_of(max);
    LogSum turn{max, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < kInFlight; ++u) {
      if (u > 0 && v0 - tid + u * threads >= row.body) break;  // (the same for all threads)
      asm volatile("" : "+v"(z[u]));  // (bf16: converted here again, the values of two passes would not fit)
#pragma unroll
      for (int e = 0; e < kPer; ++e) add_distance(turn, Row::value(z[u], e) - r);
    }
    if constexpr (KEEP) {
      l = turn;
    } else {
      add_in_two(l.sum, lost_sum, turn.sum);
      add_in_two(l.weighted, lost_weighted, turn.weighted);
    }
  };
  const int target = a.targets ? a.targets[m] : -1, edge_at = PARTS ? -1 : row.edge(tid);  // (PARTS: rows of whole vectors)
  if constexpr (KEEP) fetch(tid);
  const bool has_target = target >= 0 && target < n;
  const float target_logit = has_target ? row.at(target) : 0.f, edge = edge_at >= 0 ? row.at(edge_at) : -INFINITY;
  if constexpr (KEEP) {
    add(tid);
  } else {
#pragma unroll 1
    for (int v0 = tid; v0 < row.body; v0 += threads * kInFlight) {
      fetch(v0);
      add(v0);
    }
    take_in(l, lost_sum, lost_weighted);
  }
  const float own_max = l.max;
  if (edge_at >= 0) {
    LogSum one{edge, 0.f, 0.f};
    add_distance(one, edge - reference_of(edge));
    join(l, one);
  }
  answer_row<TOP>(
      a, rs, ts, row, l, target_logit, has_target, edge, edge_at, 1, shift, [&](int) { return own_max; },
      [&](int, int slot) {
        ts->units[tid >> 6][slot] = tid;
        if constexpr (KEEP) {
#pragma unroll
          for (int u = 0; u < kInFlight; ++u) staged[slot][u] = z[u];
        }
      },
      [&](int slot, int j, int& at) {
        const int v = ts->units[tid >> 6][slot] + j / kPer * threads;
        if (v >= row.body) return 0.f;
        at = row.index(v, j % kPer);
        if constexpr (KEEP) {
          const unsigned* const p = reinterpret_cast<const unsigned*>(staged[slot]);
          if constexpr (sizeof(T) == 4) return __uint_as_float(p[j]);
          else return __uint_as_float(j & 1 ? p[j / 2] & 0xffff0000u : p[j / 2] << 16);
        } else {
          return row.at(at);
        }
      });
}

// One workgroup per row: the pieces' sums are joined; logits (rows of whole vectors) are read again for tokens alone.
template <bool TOP>
__global__ __launch_bounds__(256) void logprob_pieces_kernel(const RowStatistics st, int count, int shift, const float* __restrict__ logits,
                                                             int64_t ld, int n, const LogprobArgs a) {
  __shared__ RowShared rs;
  TopShared* ts = nullptr;
  if constexpr (TOP) {
    __shared__ TopShared top;
    ts = &top;
  }
  const int m = blockIdx.x, tid = threadIdx.x, threads = blockDim.x;
  const int64_t first = (int64_t)m * count;
  const int target = a.targets ? a.targets[m] : -1;
  const bool has_target = target >= 0 && target < n;
  const float target_logit = has_target ? st.target_logit[m] : 0.f;
  LogSum l = no_logits();
  for (int i = tid; i < count; i += threads) join(l, LogSum{st.max[first + i], st.sum[first + i], st.weighted[first + i]});
  const LogitRow<float> row(logits + (int64_t)m * ld, n);
  answer_row<TOP>(
      a, rs, ts, row, l, target_logit, has_target, -INFINITY, -1, (count + threads - 1) / threads, shift,
      [&](int turn) { return tid + turn * threads < count ? st.max[first + tid + turn * threads] : -INFINITY; },
      [&](int turn, int slot) { ts->units[tid >> 6][slot] = tid + turn * threads; },
      [&](int slot, int j, int& at) {
        const int i = (ts->units[tid >> 6][slot] << shift) + j;
        if (i >= n) return 0.f;
        at = i;
        return row.at(i);
      });
}

hipError_t launch_logprob_rows(const void* logits, int logits_are_bf16, int64_t ld, int M, int n, int parts, int64_t stride, const LogprobArgs& a,
                               hipStream_t s) {
  if (M <= 0) return hipSuccess;
  const int per = logits_are_bf16 ? 8 : 4, vectors = n / per;
  const bool top = a.n_top > 0 || a.next_token;
  int threads = 64;  // two vectors to a thread, if 1024 are enough for that (with tokens or without: one order of the sums)
  while (threads < 1024 && threads * 2 < vectors) threads *= 2;
  const bool keep = vectors <= threads * kInFlight;
  int shift = 0;  // of the elements that a thread has read
  while ((1 << shift) < (vectors + threads - 1) / threads * per) ++shift;
  const bool nt = !top && (int64_t)M * n * (16 / per) >= (240ll << 20);
  const size_t lds = top && keep ? threads / 64 * sizeof(StagedUnits) : 0;
#define TDP_ROWS(T, TOP, KEEP, NT, PARTS)                                                                                               \
  logprob_rows_kernel<T, TOP, KEEP, NT, PARTS><<<rows, threads, lds, s>>>((const T*)logits + first * ld, ld, n, parts, stride, shift, \
                                                                          a.from_row(first))
#define TDP_ROWS_OF(T, PARTS)                                     \
  do {                                                            \
    if (top && keep) TDP_ROWS(T, true, true, false, PARTS);       \
    else if (top) TDP_ROWS(T, true, false, false, PARTS);         \
    else if (keep && nt) TDP_ROWS(T, false, true, !PARTS, PARTS); \
    else if (keep) TDP_ROWS(T, false, true, false, PARTS);        \
    else if (nt) TDP_ROWS(T, false, false, !PARTS, PARTS);        \
    else TDP_ROWS(T, false, false, false, PARTS);                 \
  } while (0)
  const int64_t most = (1ll << 31) / threads;  // rows of a launch: its threads are counted in 32 bits
  for (int64_t first = 0; first < M; first += most) {
    const unsigned rows = (unsigned)(M - first < most ? M - first : most);
    if (parts > 1) TDP_ROWS_OF(float, true);
    else if (logits_are_bf16) TDP_ROWS_OF(bf16, false);
    else TDP_ROWS_OF(float, false);
  }
#undef TDP_ROWS_OF
#undef TDP_ROWS
  return hipGetLastError();
}

hipError_t launch_logprob_pieces(const RowStatistics& st, int count, int width, const float* logits, int64_t ld, int M, int n,
                                 const LogprobArgs& a, hipStream_t s) {
  if (M <= 0) return hipSuccess;
  int shift = 0;
  while ((1 << shift) < width) ++shift;  // (64 or 128)
  if (a.n_top > 0 || a.next_token) logprob_pieces_kernel<true><<<M, 256, 0, s>>>(st, count, shift, logits, ld, n, a);
  else logprob_pieces_kernel<false><<<M, 256, 0, s>>>(st, count, shift, logits, ld, n, a);
  return hipGetLastError();
}

}  // namespace tdp
