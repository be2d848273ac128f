// Rows of logits and the largest of them: what the kernels for log-probabilities and for beams share.
#pragma once
#include <math.h>

#include "tdp_device.h"

namespace tdp {

typedef __attribute__((__vector_size__(4 * sizeof(unsigned)))) unsigned u32x4;

// A row of logits, which may begin and end anywhere in a 16-byte vector of memory: its whole vectors, the `body`, and up to seven elements on
// either side, the edges, which the first threads hold one each.  PARTS: the fp32 partials of a split projection, whose sums (in the
// order of the splits) are the logits.
template <typename T, bool PARTS = false>
struct LogitRow {
  static constexpr int kPer = 16 / sizeof(T);
  const T* first;
  int n, off, body;  // elements; in front of the body; whole vectors
  int parts = 1;
  int64_t stride = 0;  // elements from a part to the next
  __device__ __forceinline__ LogitRow(const T* row, int n_) : first(row), n(n_) {
    const int lead = (int)(((uintptr_t)row & 15) / sizeof(T));
    off = lead ? kPer - lead : 0;
    body = max(0, (n - off) / kPer);
    if (n < off) body = 0;
  }
  __device__ __forceinline__ int index(int v, int e) const { return off + v * kPer + e; }
  template <bool NT>
  __device__ __forceinline__ u32x4 load(int v) const {
    const T* const p = first + off + (int64_t)v * kPer;
    if constexpr (PARTS) {
      f32x4 sum = *reinterpret_cast<const f32x4*>(p);
      for (int i = 1; i < parts; ++i) sum += *reinterpret_cast<const f32x4*>(p + i * stride);
      return __builtin_bit_cast(u32x4, sum);
    } else if constexpr (NT) {
      return __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
    } else {
      return *reinterpret_cast<const u32x4*>(p);
    }
  }
  __device__ __forceinline__ float at(int i) const {
    float z = (float)first[i];
    if constexpr (PARTS)
      for (int j = 1; j < parts; ++j) z += first[i + j * stride];
    return z;
  }
  // the element on an edge that thread tid holds, or -1
  __device__ __forceinline__ int edge(int tid) const {
    const int i = tid < kPer ? tid : off + body * kPer + tid - kPer;
    return tid < kPer ? (i < off && i < n ? i : -1) : tid < 2 * kPer && i < n ? i : -1;
  }
  static __device__ __forceinline__ u32x4 nothing() {
    const unsigned x = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;  // minus infinity
    return u32x4{x, x, x, x};
  }
  static __device__ __forceinline__ float value(u32x4 raw, int e) {
    if constexpr (sizeof(T) == 4) return __uint_as_float(raw[e]);
    else return __uint_as_float(e & 1 ? raw[e / 2] & 0xffff0000u : raw[e / 2] << 16);
  }
};

// A sum of many terms in two numbers: `lost` takes what an addition to `sum` rounds off, exactly where |v| <= |sum|.  (Terms of one sign,
// 64 at most: elsewhere the sum at least doubles, so that what such additions round off is in all twice the last one's, u of the sum.)
__device__ __forceinline__ void add_in_two(float& sum, float& lost, float v) {
  const float s = sum + v;
  lost += v - (s - sum);
  sum = s;
}
__device__ __forceinline__ void take_in(LogSum& l, float& lost_sum, float& lost_weighted) {
  l.sum += lost_sum;
  l.weighted += lost_weighted;
  lost_sum = lost_weighted = 0.f;
}

// ---- sums over lanes -------------------------------------------------------------------------------------------------------------
// A lane's value joined with those of the lanes in front of it, by DPP: behind step i lane l holds what lanes l - 2^i + 1 .. l of its row of 16
// have, then rows 1 and 3, 2 and 3 take what stands in front of them.  Lane 63 holds all.
constexpr int kDppShift1 = 0x111, kDppShift2 = 0x112, kDppShift4 = 0x114, kDppShift8 = 0x118, kDppLast15 = 0x142, kDppLast31 = 0x143;
template <int STEP, int ROWS>
__device__ __forceinline__ float from_front(float v, float otherwise) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(__float_as_uint(otherwise), __float_as_uint(v), STEP, ROWS, 0xf, false));
}
__device__ __forceinline__ float row_sum(float v) {
  v += from_front<kDppShift1, 0xf>(v, 0.f);
  v += from_front<kDppShift2, 0xf>(v, 0.f);
  v += from_front<kDppShift4, 0xf>(v, 0.f);
  return v + from_front<kDppShift8, 0xf>(v, 0.f);
}
__device__ __forceinline__ float of_last(float v, int lane) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), lane)); }
__device__ __forceinline__ float whole_sum(float v) {
  v = row_sum(v);
  v += from_front<kDppLast15, 0xa>(v, 0.f);
  return of_last(v + from_front<kDppLast31, 0xc>(v, 0.f), 63);
}

// ---- the likeliest tokens ----------------------------------------------------------------------------------------------------------
// The k largest logits of a row (k <= 32), of equal ones those of lower index, in that order; a NaN is none of them.
//
// The row is in units, what a thread has read or a piece of the projection, whose largest logits threads know.  The maxima of 64 groups of
// threads give a bound: just below the k-th largest of them, tau has at least k logits of the row at or above it.  Only units whose
// largest reaches tau are looked at again, a few dozen of a thousand, a wave its own, and what reaches it there goes into a list, about
// twice k long; an entry's place in the answer is the number of entries before it.  (A list per lane that every logit is compared with, as
// the pass runs, costs several times the pass: a wave inserts some hundred times.)
// Where many groups share the k-th maximum (a masked row with fewer tokens left than wanted: minus infinity, or whatever number stands for
// it), only logits above it are listed; what is missing equals it, and is found by going through the row in order.  Where the
// list overflows all the same (ties everywhere; large logits all in a few groups) logits above tau are listed from the whole
// row, and tau is raised to the k-th largest listed if that overflows.  One such raise is enough for logits in no order; ones that ascend within a
// few groups can gain a list's length at a time, so after kRaises of them tau becomes the k-th largest of the row, found by counting in 16 passes.
// The code is kept short (loops, one place that lists): a workgroup has one row or two, and fetching instructions for the first
// time is a good part of what a few hundred of them take.
constexpr int kTopMost = 32, kListed = 512, kTied = 16, kStaged = 8, kRaises = 3;
static_assert(kTopMost <= 64, "the bound is one of 64 maxima");

struct RowShared {
  float wave_max[16], wave_sum[16], wave_weighted[16];
  float group_max[64];
};
struct TopShared {
  unsigned long long list[kListed + kTopMost + 8];
  int units[16][kStaged];
  int listed;
  float tau;
  int wave_count[16];
};
// Units that threads hold in registers, eight vectors each, those of one wave.
typedef u32x4 StagedUnits[kStaged][8];

// Logits in an order of whole numbers.  (Both zeros are one value.)
__device__ __forceinline__ unsigned order_of(float z) {
  const unsigned bits = __float_as_uint(z + 0.f);
  return bits ^ ((unsigned)((int)bits >> 31) | 0x80000000u);
}
__device__ __forceinline__ float logit_of(unsigned order) { return __uint_as_float(order ^ (order >> 31 ? 0x80000000u : 0xffffffffu)); }
// A logit and its index as one number: larger logits first, then lower indices.
__device__ __forceinline__ unsigned long long key_of(float z, int at) { return (unsigned long long)order_of(z) << 32 | (unsigned)~at; }

// A number that at least k of the lanes' values reach, and of those that end in 14 zero bits the largest: 2^-9 of itself below the k-th
// largest value at most.  (1 <= k <= 64; two bits of it at a time, from counts of lanes: nine steps that wait for each other, 0.4 us,
// where 64 comparisons with values read from lanes take 1.3.)
__device__ __forceinline__ float bound_of_wave(float v, int k) {
  const unsigned order = order_of(v);
  unsigned bound = 0;
#pragma unroll 3
  for (int bit = 30; bit >= 14; bit -= 2) {
    const unsigned one = bound | 1u << bit, two = bound | 2u << bit, three = bound | 3u << bit;
    const int n1 = __popcll(__ballot(order >= one)), n2 = __popcll(__ballot(order >= two)), n3 = __popcll(__ballot(order >= three));
    bound = n3 >= k ? three : n2 >= k ? two : n1 >= k ? one : bound;
  }
  return bound > order_of(-INFINITY) ? logit_of(bound) : -INFINITY;
}

// The place of a key among the first c of the list.
__device__ __forceinline__ int place_of(const TopShared& sh, unsigned long long key, int c) {
  int place = 0;
  for (int j = 0; j < c; j += 8) {  // (the list has room for eight more than it can hold)
    unsigned long long other[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) other[i] = sh.list[j + i];
#pragma unroll
    for (int i = 0; i < 8; ++i) place += (int)(other[i] > key) & (int)(j + i < c);
  }
  return place;
}

// All threads of the workgroup (a power of two of whole waves).  group_max and listed = 0 are in LDS, behind a barrier.
// In turn i < turns a lane has a unit whose largest logit is largest_of(i); stage(i, slot) puts it where element(slot, j, &at) finds its logit j of
// 2^shift, and its index (-1: none).  edge: the thread's element outside all units, edge_at its index or -1.  write(place, index, value) is
// called once for every place found; returns how many there are.
template <typename Row, typename Largest, typename Stage, typename Element, typename Write>
__device__ __forceinline__ int select_top(const RowShared& rs, TopShared& sh, const Row& row, float largest, int k, float edge, int edge_at,
                                          int turns, int shift, Largest largest_of, Stage stage, Element element, Write write) {
  const int tid = threadIdx.x, threads = blockDim.x, wave = tid >> 6, lane = tid & 63, waves = threads >> 6;
  float tau = largest;  // (k = 1)
  bool above = tau == -INFINITY;
  if (k > 1) {
    const float v = rs.group_max[lane];
    tau = bound_of_wave(v, k);
    above = __popcll(__ballot(v >= tau)) >= k + kTied || tau == -INFINITY;
    if (above) {  // the least of them: the k-th largest, unless that is one of many different ones just below each other
      float least = v >= tau ? v : INFINITY;
      for (int o = 1; o < 64; o *= 2) least = fminf(least, __shfl_xor(least, o, 64));
      tau = least;
    }
  }
  auto reaches = [&](float z) { return above ? z > tau : z >= tau; };
  auto list = [&](float z, int at) {
    if (at < 0 || !reaches(z)) return;
    const int p = atomicAdd(&sh.listed, 1);
    if (p < kListed) sh.list[p] = key_of(z, at);
  };
#pragma unroll 1
  for (int turn = 0; turn < turns; ++turn) {
    bool flag = reaches(largest_of(turn));
    unsigned long long flags = __ballot(flag);
#pragma unroll 1
    while (flags) {
      const int slot = __popcll(flags & ((1ull << lane) - 1));
      const bool now = flag && slot < kStaged;
      if (now) stage(turn, slot);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      const int total = min((int)__popcll(flags), kStaged) << shift;  // (2^3 units of 2^20 logits at most)
#pragma unroll 1
      for (int q0 = lane; q0 < total; q0 += 128) {
        int at0 = -1, at1 = -1;
        const float z0 = element(q0 >> shift, q0 & ((1 << shift) - 1), at0);
        const int q1 = q0 + 64;
        float z1 = 0.f;
        if (q1 < total) z1 = element(q1 >> shift, q1 & ((1 << shift) - 1), at1);
        list(z0, at0);
        list(z1, at1);
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      flag = flag && !now;
      flags = __ballot(flag);
    }
  }
  list(edge, edge_at);
  __syncthreads();
  int c = sh.listed;
  if (c > kListed) {
    above = true;
    for (int raises = 0;; ++raises) {
      __syncthreads();
      if (tid == 0) sh.listed = 0;
      __syncthreads();
#pragma unroll 1
      for (int64_t i = tid; i < row.n; i += threads) list(row.at((int)i), (int)i);
      __syncthreads();
      c = sh.listed;
      if (c <= kListed) break;
      if (raises < kRaises) {
        for (int i = tid; i < kListed; i += threads)
          if (place_of(sh, sh.list[i], kListed) == k - 1) sh.tau = logit_of((unsigned)(sh.list[i] >> 32));  // (one entry)
        __syncthreads();
        tau = sh.tau;
      } else {
        unsigned bound = 0;  // two bits of it at a time
#pragma unroll 1
        for (int bit = 30; bit >= 0; bit -= 2) {
          int reached[3] = {0, 0, 0};
          if (tid < 3) sh.wave_count[tid] = 0;
#pragma unroll 1
          for (int64_t i = tid; i < row.n; i += threads) {
            const float z = row.at((int)i);
            const unsigned order = z == z ? order_of(z) : 0u;
#pragma unroll
            for (int q = 0; q < 3; ++q) reached[q] += order >= (bound | (q + 1u) << bit);
          }
          __syncthreads();
#pragma unroll
          for (int q = 0; q < 3; ++q) atomicAdd(&sh.wave_count[q], reached[q]);
          __syncthreads();
          unsigned next = bound;
#pragma unroll
          for (int q = 0; q < 3; ++q) next = sh.wave_count[q] >= k ? bound | (q + 1u) << bit : next;
          bound = next;
          __syncthreads();
        }
        tau = logit_of(bound);
      }
    }
  }
  if (c < k) {
    // those that equal tau, in the order of the row, a logit per thread and turn
    const int wanted = k - c;
    int found = 0;
    for (int64_t first = 0; first < row.n && found < wanted; first += threads) {
      const int64_t at = first + tid;
      const bool hit = at < row.n && row.at((int)at) == tau;
      const unsigned long long hits = __ballot(hit);
      if (lane == 0) sh.wave_count[wave] = __popcll(hits);
      __syncthreads();
      int p = found + __popcll(hits & ((1ull << lane) - 1));
      int total = 0;
#pragma unroll 1
      for (int w = 0; w < waves; ++w) {
        if (w < wave) p += sh.wave_count[w];
        total += sh.wave_count[w];
      }
      if (hit && p < wanted) sh.list[c + p] = key_of(tau, (int)at);
      found += total;
      __syncthreads();
    }
    c += min(found, wanted);
  }
  for (int i = tid; i < c; i += threads) {
    const unsigned long long key = sh.list[i];
    const int place = place_of(sh, key, c);
    if (place < k) write(place, (int)~(unsigned)key, logit_of((unsigned)(key >> 32)));
  }
  return min(c, k);
}

}  // namespace tdp
