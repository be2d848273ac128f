// Decode attention of rows that share a prefix (beams of a prompt, requests behind one system prompt): the keys and values of the pages on
// which the block tables of a group agree are read once for all (query head, row) pairs of the group, its columns.
//
// What is shared is found in the tables, not told: a group is rows that may share something, and its prefix is the leading pages that are the
// same in all of them, whole pages in front of every row's last token.  So the answer is that of ordinary decode attention whatever
// the groups are.  Three launches: the plan (once per step), the prefixes, the rows.  The prefix kernel leaves partials (reference m, sum
// l, unnormalised output o, per span of the prefix) in the first slots of every row and head; a row's own kernel attends to what the row has
// behind its prefix and combines all.
//
// Times of whole calls in the comments here are of calls alone, each behind a write that has emptied the caches.
#include <algorithm>

#include "tdp_device.h"
#include "tdp_kernels.h"

namespace tdp {
namespace {

constexpr int kMinSpanPages = kDecodeSpanMin / 16;
// Partials that one wave of four joins by itself, one after another; of more each has a quarter, four on their way at a time.  Whole calls, 8
// K/V heads, never / from 8 / from 24 on: a row of 4000 tokens 30 / 27 / 30 us, 4 rows of up to 8000 46 / 50 / 46 and of up to 16000 95 / 83 / 83, a row
// of up to 32000 70 / 54, of up to 131000 164 / 124; two rows behind a prefix of 131000, 2 heads, 174 / 112.
constexpr int kJoinedAlone = 8;
constexpr int kResident = 3 * 256;  // workgroups of the sixteen-column kernel that the chip holds at once (two to three per CU)

// How a batch is attended to: a pure function of sizes that the host knows.
//
// columns: of a tile of the prefix kernel, by the average group's (a large group among many small ones gets the small ones' tiles and is read once
// for each).  Prefixes of 1200 to 2000 tokens, 8 K/V heads of 128 channels, 8 query heads to each, the whole call, tiles of 16 / 64 / 128
// columns: 64 groups of 32 columns 136 / 171 / 180 us, of 48 201 / 185 / 195, of 128 380 / 226 / 225, 16 groups of 96 87 / 93 / 90, of 128 107 / 97 /
// 96, 24 of 256 216 / 148 / 141.  Of few groups the tiles count less: four with a prefix of 2400 to 4000 tokens, of 24 columns 39 / 48 / 49, 32
// 44 / 52 / 52, 48 47 / 51 / 52, 64 53 / 55 / 55, 96 57 / 67 / 62, 128 59 / 66 / 62, 256 85 / 99 / 90, 512 137 / 112 / 105; 8-bit pools 24
// 41 / 41 / 42, 32 44 / 44 / 44, 48 48 / 45 / 47, 64 51 / 48 / 49, 96 53 / 58 / 55, 128 56 / 62 / 58, 256 79 / 93 / 88, 512 107 / 97 / 93 (so with 64 to
// 256 columns four groups would have up to 15 % from tiles of 16).
// wanted: spans of the prefixes per K/V head (spans of a group times its tiles), as many as make the workgroups that the chip holds at once,
// twice that for 64 columns.  16 columns, 512 / 768 / 1536 / 2048 workgroups: 8 groups of 8000 tokens, 32 heads 148 / 147 / 148 / 156 us, 32 of 1500
// 135 / 135 / 141 / 142; 64 columns, 4 groups of 8 x 8, 512 / 768 / 1024 / 1536: 55 / 53 / 53 / 53; 128 columns, 512 rows behind one prompt of 2100,
// 256 / 512 / 768 / 1536: 155 / 140 / 152 / 166.
struct Form {
  int columns, wanted;
};
Form form_of(int batch, int n_groups, int n_q_heads, int n_kv_heads) {
  const int G = n_q_heads / n_kv_heads;
  const int64_t average = n_groups > 0 ? ((int64_t)batch * G + n_groups - 1) / n_groups : 0;
  Form f;
  f.columns = average <= 32 ? 16 : average <= 64 ? 64 : 128;
  const int units = f.columns == 16 ? kResident : f.columns == 64 ? 1024 : 512;
  f.wanted = (units + n_kv_heads - 1) / n_kv_heads;
  return f;
}
// Whether the waves of a workgroup share a row's span out, or have one each.  Own tokens of up to 100 / 400 / 1000 (whole calls, 8 K/V heads,
// shared out against one each): 32 rows 32 / 33 us and 28 / 42, 64 rows 35 / 36 and 33 / 43, 128 rows 41 / 38 and 46 / 47, 256 rows 56 / 47, 70 / 67
// and 118 / 129, 512 rows 89 / 73, 120 / 115 and 221 / 222; 8-bit pools, up to 200, 96 rows 41 / 40, 256 rows 59 / 48.
bool rows_split(int batch, int n_kv_heads) { return (int64_t)batch * n_kv_heads < 1024; }
int items_of(const SharedBatch& b, const Form& f) {
  return (int)((int64_t)b.batch * (b.n_q_heads / b.n_kv_heads) / f.columns) + b.n_groups + f.wanted;
}

// ---- plan ------------------------------------------------------------------------------------------------------------------------

struct PlanArgs {
  SharedBatch b;
  int columns, wanted, max_prefix_items;
  int32_t* row_pages;  // [batch]: pages that a row has in common with the first of its group
  int32_t* group;      // [4][n_groups], where they are too many for LDS
  unsigned* done;
  int32_t* counts;
  int4 *prefix_items, *row_items;
};
constexpr int kPlanThreads = 256, kPlanRows = 16;  // rows that a workgroup compares, as long as there are not too many workgroups
constexpr int kPlanHeld = 1024;                    // rows, and groups, that the last workgroup holds in LDS
constexpr int kClasses = 17;                       // of row spans by their length
typedef i32x4 __attribute__((aligned(4))) i32x4_of_int;
// (The length is brought into the row's range before `add` joins it, as a decode step brings its position: 2^31 - 1 + 1 would be no length.)
__device__ __forceinline__ int row_tokens(const SharedBatch& b, int r) {
  return min(max(b.lens[r], 0), b.max_pages_per_seq * 16 - b.add) + b.add;
}

// A thread's value plus those of all threads of the workgroup in front of it, and the sum of all.
__device__ __forceinline__ int plan_scan(int v, int* part, int* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    const int up = __shfl_up(v, o, 64);
    if (lane >= o) v += up;
  }
  __syncthreads();  // (part may still be read)
  if (lane == 63) part[wave] = v;
  __syncthreads();
  int all = 0;
#pragma unroll
  for (int w = 0; w < kPlanThreads / 64; ++w) {
    v += w < wave ? part[w] : 0;
    all += part[w];
  }
  *total = all;
  return v;
}
// The last i in [0, n) with at[i] <= v (at ascending; 0 if there is none).
__device__ __forceinline__ int last_not_above(const int32_t* at, int n, int v) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (at[mid] <= v) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// Workgroups compare tables, each those of a range of rows; the one that finishes last makes both work lists (prefix items: two records
//   (first row of the group, first column, columns of the group, span), (first page, pages, row whose table names them, 0);
// row items: (row, pages of the prefix, tokens behind it, span | spans of the prefix << 16)).  Results of other workgroups, which run on
// other XCDs, are stored and read past the caches, and counted when they have arrived.
// Rows of length zero attend to nothing: what their tables hold is not looked at.
// Bound: a chain of look-ups and barriers (a workgroup alone: 5 us), and the tables, which one CU reads at some 30 GB/s.  4 rows 7 us; 162 rows in
// 24 groups, 250 pages 13 us (loads 3, comparison 3, groups' sums 3, prefix items 2, row items 2); 512 rows in one group 15 us.  A workgroup per
// 8 / 16 / 32 / 64 rows, the whole call: 512 rows behind one prompt 141 / 140 / 140 / 144 us, 24 groups of 8 155 / 154 / 154 / 158, 256 rows 56 / 56 / 57 / 62.
__global__ __launch_bounds__(kPlanThreads) void shared_plan_kernel(const PlanArgs a) {
  constexpr int T = kPlanThreads;
  __shared__ int32_t s_starts[kPlanHeld + 1], s_tokens[kPlanHeld], s_group[4 * kPlanHeld], s_pages[T], s_first[T];
  __shared__ int is_last, longest_limit, part[T / 64], class_at[kClasses];
  __shared__ unsigned long long work;
  const SharedBatch& b = a.b;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, P = b.max_pages_per_seq, n_groups = b.n_groups;
  const bool few = n_groups <= kPlanHeld, held = b.batch <= kPlanHeld;
  if (few && n_groups > 0)
    for (int g = tid; g <= n_groups; g += T) s_starts[g] = b.group_starts[g];
  if (held)
    for (int r = tid; r < b.batch; r += T) s_tokens[r] = row_tokens(b, r);
  auto tokens_of = [&](int r) { return held ? s_tokens[r] : row_tokens(b, r); };
  const int32_t* const starts = few ? s_starts : b.group_starts;
  // the group of a row, or -1: [begin, end) of a group, in bounds whatever the starts are
  auto begin_of = [&](int g) { return min(max(starts[g], 0), b.batch); };
  auto end_of = [&](int g) { return min(max(starts[g + 1], begin_of(g)), b.batch); };
  auto group_of = [&](int r) {
    if (n_groups == 0) return -1;
    const int g = last_not_above(starts, n_groups, r);
    return r >= begin_of(g) && r < end_of(g) ? g : -1;
  };
  if (n_groups > 0) {
    const int each = (b.batch + gridDim.x - 1) / gridDim.x, own_begin = min((int)blockIdx.x * each, b.batch), own_end = min(own_begin + each, b.batch);
    for (int t0 = own_begin; t0 < own_end; t0 += T) {
      const int rows = min(own_end - t0, T);
      if (tid == 0) longest_limit = 0;
      __syncthreads();  // (starts are there; the tile before is done with)
      if (tid < rows) {
        // as many pages as a row has in front of its last token, and the first row of its group that has some; -1: no tokens, or no group
        const int r = t0 + tid, g = group_of(r), own_tokens = tokens_of(r);
        int first = r, limit = -1;
        if (g >= 0 && own_tokens > 0) {
          limit = (own_tokens - 1) >> 4;
          int tokens = 0;
          for (first = begin_of(g); first < r && (tokens = tokens_of(first)) <= 0;) ++first;
          if (first < r && P < 4) {
            limit = 0;  // (tables of three entries have nothing worth sharing, nor four entries to look at at once)
          } else if (first < r) {
            limit = min(limit, (tokens - 1) >> 4);
            atomicMax(&longest_limit, limit);
          }
        }
        s_pages[tid] = limit;
        s_first[tid] = first;
      }
      __syncthreads();
      // the first difference from that row: a wave compares eight rows' 256 entries at a time, four side by side to a lane, low pages first
      constexpr int ROWS = 8, SIDE = 4;
      const int chunks = P >= SIDE ? (longest_limit + 64 * SIDE - 1) / (64 * SIDE) : 0, eights = (rows + ROWS - 1) / ROWS;
      for (int i = wave; i < eights * chunks; i += T / 64) {
        const int c = i / eights, row0 = (i - c * eights) * ROWS;
        int limit[ROWS], at[ROWS];
        i32x4 want[ROWS], got[ROWS];
#pragma unroll
        for (int j = 0; j < ROWS; ++j) {
          const int row = min(row0 + j, rows - 1), of = s_first[row];
          limit[j] = of == t0 + row ? 0 : *(volatile int*)&s_pages[row];
          at[j] = min((c * 64 + lane) * SIDE, max(limit[j], SIDE) - SIDE);  // (in the row, and not used where there is nothing to compare)
          want[j] = *reinterpret_cast<const i32x4_of_int*>(b.block_tables + (int64_t)of * P + at[j]);
          got[j] = *reinterpret_cast<const i32x4_of_int*>(b.block_tables + (int64_t)(t0 + row) * P + at[j]);
        }
#pragma unroll
        for (int j = 0; j < ROWS; ++j) {
          int differs = 0x7fffffff;
#pragma unroll
          for (int u = SIDE - 1; u >= 0; --u)
            if (got[j][u] != want[j][u]) differs = at[j] + u;
          if (differs < limit[j]) atomicMin(&s_pages[min(row0 + j, rows - 1)], differs);
        }
      }
      __syncthreads();
      if (tid < rows) store_agent(a.row_pages + t0 + tid, s_pages[tid]);
    }
    if (gridDim.x > 1) {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
      if (tid == 0) {
        const unsigned before = __hip_atomic_fetch_add(a.done, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        is_last = before + 1 == gridDim.x;
        if (is_last) __hip_atomic_store(a.done, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      }
      __syncthreads();
      if (!is_last) return;
    }
  }
  const bool in_lds = gridDim.x == 1 && b.batch <= T;  // what has been found out of the rows
  auto pages_of = [&](int r) { return in_lds ? s_pages[r] : load_agent(a.row_pages + r); };
  if (!in_lds) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (alone, with several tiles: its own stores)
  // What the groups share, and how much there is to do for it: [n_groups] each of pages, longest row, first and last row with tokens.
  int32_t* const common = few ? s_group : a.group;
  const int pitch = few ? kPlanHeld : n_groups;
  int32_t *const longest = common + pitch, *const first = longest + pitch, *const last = first + pitch;
  int32_t* const spans = longest;  // (then) spans of the prefix
  if (tid == 0) work = 0;
  if (tid < kClasses) class_at[tid] = 0;
  for (int g = tid; g < n_groups; g += T) {
    common[g] = first[g] = 0x7fffffff;
    longest[g] = 0;
    last[g] = -1;
  }
  __syncthreads();
  for (int r = tid; n_groups > 0 && r < b.batch; r += T) {
    const int g = group_of(r), pages = g >= 0 ? pages_of(r) : -1;
    if (pages >= 0) {
      atomicMin(common + g, pages);
      atomicMax(longest + g, tokens_of(r));
      atomicMin(first + g, r);
      atomicMax(last + g, r);
    }
  }
  __syncthreads();
  auto tiles_of = [&](int g) { return ((end_of(g) - begin_of(g)) * (b.n_q_heads / b.n_kv_heads) + a.columns - 1) / a.columns; };
  for (int g = tid; g < n_groups; g += T) {
    int pages = common[g];
    // A short prefix is left to the rows where one of them has more than the shortest span behind it: a row has as many slots for partials as
    // spans of that length, so that prefix and spans together could need one more than there are.
    if (last[g] <= first[g] || (pages < kMinSpanPages && longest[g] - pages * 16 > kDecodeSpanMin)) pages = 0;
    common[g] = pages;
    if (pages) atomicAdd(&work, (unsigned long long)tiles_of(g) * (unsigned long long)pages);
  }
  __syncthreads();
  // prefixes in spans as long as the number wanted allows, all of a group equally long; their items, a thread each
  const unsigned long long all_pages = work + a.wanted - 1;  // (a division of 32 bits where that is enough: a fifth of the time)
  const int span = max(kMinSpanPages, (int)(all_pages >> 32 ? all_pages / (unsigned)a.wanted : (unsigned)all_pages / (unsigned)a.wanted));
  auto spans_of = [&](int pages) { return pages > 0 ? max(1, min((pages + span - 1) / span, pages / kMinSpanPages)) : 0; };
  int base = 0;
  for (int g0 = 0; g0 < n_groups; g0 += T) {
    const int g = g0 + tid, pages = g < n_groups ? common[g] : 0;
    const int own_spans = spans_of(pages), n = own_spans ? own_spans * tiles_of(g) : 0;
    int total;
    const int behind = plan_scan(n, part, &total);
    s_first[tid] = behind - n;
    if (g < n_groups) spans[g] = own_spans;
    __syncthreads();
    for (int i = tid; i < total && base + i < a.max_prefix_items; i += T) {
      const int at = last_not_above(s_first, min(n_groups - g0, T), i), of = g0 + at;  // (the last that begins there is the one that has some)
      const int row = begin_of(of), tiles = tiles_of(of), own = i - s_first[at];
      const unsigned s = own / tiles, from = s * (unsigned)common[of] / spans[of], to = (s + 1) * (unsigned)common[of] / spans[of];
      a.prefix_items[2 * (base + i)] = make_int4(row, (own - s * tiles) * a.columns, (end_of(of) - row) * (b.n_q_heads / b.n_kv_heads), s);
      a.prefix_items[2 * (base + i) + 1] = make_int4(from, to - from, first[of], 0);
    }
    base += total;
    __syncthreads();
  }
  if (tid == 0) a.counts[0] = min(base, a.max_prefix_items);
  // The rows' spans, longest first by sixteenths of span_len, so that the launch ends on short ones: counted per class, then placed.  (In no
  // fixed order within a class; a row's result does not depend on its place.)
  struct Row {
    int pages, tokens, spans, in_front;
  };
  auto row_of = [&](int r) {
    Row x{0, tokens_of(r), 0, 0};
    const int g = x.tokens > 0 ? group_of(r) : -1;
    if (g >= 0) {
      x.pages = common[g];
      x.in_front = x.pages ? spans[g] : 0;
    }
    x.tokens -= x.pages * 16;
    x.spans = max(1, (x.tokens + b.span_len - 1) / b.span_len);
    return x;
  };
  auto class_of = [&](const Row& x) {  // of the last span; 0: whole spans
    const int tokens = x.tokens - (x.spans - 1) * b.span_len;
    return kClasses - 1 - max(0, tokens - 1) / (b.span_len / (kClasses - 1));
  };
  Row own{0, 0, 0, 0};
  for (int r = tid; r < b.batch; r += T) {
    own = row_of(r);
    if (own.spans > 1) atomicAdd(&class_at[0], own.spans - 1);
    atomicAdd(&class_at[class_of(own)], 1);
  }
  __syncthreads();
  if (tid < 64) {
    const int n = tid < kClasses ? class_at[tid] : 0;
    int at = n;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
      const int up = __shfl_up(at, o, 64);
      if (tid >= o) at += up;
    }
    if (tid < kClasses) class_at[tid] = at - n;
    if (tid == kClasses - 1) a.counts[1] = at;
  }
  __syncthreads();
  for (int r = tid; r < b.batch; r += T) {
    if (b.batch > T) own = row_of(r);
    const int at = own.spans > 1 ? atomicAdd(&class_at[0], own.spans - 1) : 0, last_at = atomicAdd(&class_at[class_of(own)], 1);
    for (int k = 0; k < own.spans; ++k)
      a.row_items[k + 1 < own.spans ? at + k : last_at] = make_int4(r, own.pages, own.tokens, k | own.in_front << 16);
  }
}

// ---- sixteen columns -------------------------------------------------------------------------------------------------------------

// Attention of up to sixteen columns to a span of pages, keys and values from memory straight into MFMA operands, as in decode attention: the
// columns are the 16-wide side of 16x16x32 MFMAs, scores are formed transposed, and their rows are assigned to tokens so that a lane's elements
// are the consecutive tokens that it supplies to O^T += V^T P^T.
//
// PREFIX: the columns are (row, head) pairs of a group, the span one of its prefix; the partials go to the columns' slots.  Otherwise they are the
// heads of one row, the span one of what it has behind its prefix; the prefix's partials, and those of the row's other spans if it has some
// (whoever is done last), are combined with them.
// SPLIT: the four waves of a workgroup share the span out; otherwise each has one of its own, with no LDS and no barrier: short spans by
// the thousand are mostly their own beginning and end.  Prefixes are always shared out (a span each: up to 20 % slower, but for some 256 to 512
// short 8-bit prefixes, where it was 7 to 9 % faster).
//
// Bound: reading.  24 prefixes of 2400 to 4000 tokens, 32 heads of 128 8-bit channels 105 us (588 MB, 5.6 TB/s); what 512 rows of 8 heads have behind
// their prefix, 15 to 312 tokens, 69 us (332 MB, and 34 MB of partials, 5.3 TB/s; with 168 registers for three waves to a SIMD instead of what two
// allow 71 us; begun from the prefix's partials instead of ended with them 71 us; ordinary instead of non-temporal loads 85, and 119 for the 105).
template <int DH, bool KV8, bool PREFIX, bool SPLIT>
__global__ __launch_bounds__(256, DH == 128 ? 2 : 3) void attn_columns_kernel(const bf16* __restrict__ q, int64_t ld, int n_q_heads, KvLayout kv,
                                                              const int4* __restrict__ items, const int32_t* __restrict__ count,
                                                              const int32_t* __restrict__ block_tables, int max_pages_per_seq,
                                                              float* __restrict__ part_o, float* __restrict__ part_ml,
                                                              unsigned* __restrict__ spans_done, int max_spans, int span_len,
                                                              bf16* __restrict__ out, OperandLayout out_lay, float scale_log2, float out_scale) {
  constexpr int KS = DH / 32;        // k-steps of the score MFMA
  constexpr int DT = DH / 16;        // 16-channel tiles of the output
  constexpr int BT = KV8 ? 64 : 32;  // tokens per block
  constexpr int NT = BT / 16;        // score tiles per block
  constexpr int NP = BT / 32;        // k-steps of the output MFMA per block
  constexpr int LT = BT / 4;         // consecutive tokens of a block whose scores end up in one lane
  constexpr int kChunk = 256;        // pages whose ids the wave holds at once, four to a lane
  constexpr int PITCH = DT * 4 + 2;
  __shared__ float s_state[SPLIT ? 3 * 64 * PITCH : 1];
  __shared__ int s_last;
  const int Hkv = kv.n_kv_heads, G = n_q_heads / Hkv;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r16 = lane & 15, kg = lane >> 4;
  const bf16* const kpool = (const bf16*)kv.k_pool;
  const bf16* const vpool = (const bf16*)kv.v_pool;
  const uint8_t* const kpool8 = (const uint8_t*)kv.k_pool;
  const uint8_t* const vpool8 = (const uint8_t*)kv.v_pool;
  const int krow0 = (r16 >> 2) * LT + (r16 & 3);  // token (within a block) of this lane's row in score tile t: krow0 + t * 4
  const int units = *count * Hkv, stride = SPLIT ? gridDim.x : gridDim.x * 4;
  for (int unit = SPLIT ? blockIdx.x : blockIdx.x * 4 + wave; unit < units; unit += stride) {
    const int item = unit / Hkv, kvh = unit - item * Hkv;
    // the lane's column of an item
    struct Column {
      int row, head;
      bool real;
    };
    auto column_of = [&](int4 x) {
      if constexpr (PREFIX) {
        const int col = x.y + r16, c = min(col, x.z - 1), r = c / G;
        return Column{x.x + r, kvh * G + c - r * G, col < x.z};
      } else {
        return Column{x.x, kvh * G + min(r16, G - 1), r16 < G};
      }
    };
    int tokens;
    const int32_t* table;
    bf16x8 qf[KS];
    {
      const int4 x = items[PREFIX ? 2 * item : item];
      if constexpr (PREFIX) {
        const int4 y = items[2 * item + 1];
        tokens = y.y * 16;
        table = block_tables + (int64_t)y.z * max_pages_per_seq + y.x;
      } else {
        const int begin = (x.w & 0xffff) * span_len;
        tokens = min(x.z - begin, span_len);
        table = block_tables + (int64_t)x.x * max_pages_per_seq + x.y + begin / 16;
      }
      // Query fragments.  bf16 pools: k-step kk covers channels kk*32 + kg*8 .. +8.  8-bit pools: a lane's 16-byte key load covers channels
      // ld*64 + kg*16 .. +16, whose halves feed k-steps 2 ld and 2 ld + 1, so the query is gathered in that order.
      const Column c = column_of(x);
      const bf16* qp = q + (int64_t)c.row * ld + (int64_t)c.head * DH;
#pragma unroll
      for (int kk = 0; kk < KS; ++kk) qf[kk] = ld_bf16x8(qp + (KV8 ? (kk >> 1) * 64 + kg * 16 + (kk & 1) * 8 : kk * 32 + kg * 8));
    }
    f32x4 o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) o[d] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = kNegBig, lsum = 0.f;

    for (int c0 = 0; c0 < tokens; c0 += kChunk * 16) {
      const int n_total = min(tokens - c0, kChunk * 16), last_entry = (n_total - 1) >> 4;
      int my_pages[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) my_pages[j] = table[(c0 >> 4) + min(lane + 64 * j, last_entry)];
      const int n_blocks = (n_total + BT - 1) / BT;
      const int t_begin = SPLIT ? BT * ((wave * n_blocks) >> 2) : 0;
      const int t_end = SPLIT ? min(BT * (((wave + 1) * n_blocks) >> 2), n_total) : n_total;
      if (t_begin >= t_end) continue;
      auto page_of = [&](int i) -> int64_t {  // i is wave-uniform
        const int r = i >> 6;
        return __builtin_amdgcn_readlane(r == 0 ? my_pages[0] : r == 1 ? my_pages[1] : r == 2 ? my_pages[2] : my_pages[3], i & 63);
      };
      struct KBlock {
        bf16x8 kf[2][KS];  // bf16: [score tile][k-step]; 8 bits: 16 raw bytes per entry, [t / 2][(t % 2) * KS/2 + ld]
      };
      struct VBlock {
        bf16x8 vf[DT];     // bf16: 8 tokens of a channel; 8 bits: 16 raw bytes = 16 tokens of a channel
      };
      auto load_k = [&](int tb, KBlock& blk) {
        int64_t page[BT / 16];
#pragma unroll
        for (int j = 0; j < BT / 16; ++j) page[j] = page_of(min((tb >> 4) + j, last_entry));
        if constexpr (KV8) {
          const int64_t kpage = (r16 >> 2) == 0 ? page[0] : (r16 >> 2) == 1 ? page[1] : (r16 >> 2) == 2 ? page[2] : page[3];
          const uint8_t* kp = kpool8 + (kpage * Hkv + kvh) * (16 * DH) + (r16 & 3) * 64 + kg * 16;
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int l = 0; l < KS / 2; ++l)
              blk.kf[t >> 1][(t & 1) * (KS / 2) + l] = ld_bf16x8_nt(reinterpret_cast<const bf16*>(kp + (t * 4) * 64 + l * 1024));
        } else {
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            const int tok = krow0 + t * 4;
            const bf16* kp = kpool + (page[tok >> 4 & 1] * Hkv + kvh) * (16 * DH) + (tok & 15) * 32 + kg * 8;
#pragma unroll
            for (int kk = 0; kk < KS; ++kk) blk.kf[t][kk] = ld_bf16x8_nt(kp + kk * (16 * 32));
          }
        }
      };
      auto load_v = [&](int tb, VBlock& blk) {
        int64_t page[BT / 16];
#pragma unroll
        for (int j = 0; j < BT / 16; ++j) page[j] = page_of(min((tb >> 4) + j, last_entry));
        if constexpr (KV8) {
          const int64_t vpage = kg == 0 ? page[0] : kg == 1 ? page[1] : kg == 2 ? page[2] : page[3];
          const uint8_t* vp = vpool8 + ((vpage * Hkv + kvh) * DH + r16) * 16;
#pragma unroll
          for (int d = 0; d < DT; ++d) blk.vf[d] = ld_bf16x8_nt(reinterpret_cast<const bf16*>(vp + d * 16 * 16));
        } else {
          const int64_t vpage = kg < 2 ? page[0] : page[1];
          const bf16* vp = vpool + ((vpage * Hkv + kvh) * DH + r16) * 16 + (kg & 1) * 8;
#pragma unroll
          for (int d = 0; d < DT; ++d) blk.vf[d] = ld_bf16x8_nt(vp + d * 16 * 16);
        }
      };
      auto compute_block = [&](int tb, KBlock& blk, VBlock& vblk) {
        f32x4 s[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
          if constexpr (KV8) {
#pragma unroll
            for (int l = 0; l < KS / 2; ++l) {
              bf16x8 k0, k1;
              e4m3x16_to_bf16x8x2(__builtin_bit_cast(uint4, blk.kf[t >> 1][(t & 1) * (KS / 2) + l]), k0, k1);
              s[t] = mfma16(k0, qf[2 * l], s[t]);
              s[t] = mfma16(k1, qf[2 * l + 1], s[t]);
            }
          } else {
#pragma unroll
            for (int kk = 0; kk < KS; ++kk) s[t] = mfma16(blk.kf[t][kk], qf[kk], s[t]);
          }
        }
        // lane holds tokens tb + kg*LT + t*4 + i of column r16
        const int tok_base = tb + kg * LT;
        float mx = kNegBig;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float v = (tok_base + t * 4 + i < n_total) ? s[t][i] * scale_log2 : kNegBig;
            s[t][i] = v;
            mx = fmaxf(mx, v);
          }
        mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
        mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
        const float m_new = fmaxf(m, mx);
        const float alpha = exp2f(m - m_new);
        bf16x8 pb[NP];
        float psum = 0.f;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float pv = exp2f(s[t][i] - m_new);
            psum += pv;
            pb[t >> 1][(t & 1) * 4 + i] = (bf16)pv;  // (rounded for the MFMA alone: the sum is of what it was)
          }
        lsum = lsum * alpha + psum;
        m = m_new;
        const bool tail = tb + BT > n_total;  // slots behind the span may hold anything, even NaN
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          o[d] *= alpha;
          if constexpr (KV8) {
            uint4 raw = __builtin_bit_cast(uint4, vblk.vf[d]);
            if (tail) {  // keep the first n_total - tok_base bytes (tokens tok_base .. tok_base + 15)
              const int keep = min(max(n_total - tok_base, 0), 16);
              auto mask = [&](int w) -> uint32_t {
                const int k4 = min(max(keep - 4 * w, 0), 4);
                return k4 == 4 ? 0xffffffffu : (1u << (8 * k4)) - 1u;
              };
              raw.x &= mask(0);
              raw.y &= mask(1);
              raw.z &= mask(2);
              raw.w &= mask(3);
            }
            bf16x8 v0, v1;
            e4m3x16_to_bf16x8x2(raw, v0, v1);
            o[d] = mfma16(v0, pb[0], o[d]);
            o[d] = mfma16(v1, pb[NP - 1], o[d]);
          } else {
            if (tail) {
#pragma unroll
              for (int j = 0; j < 8; ++j)
                if (tok_base + j >= n_total) vblk.vf[d][j] = (bf16)0.0f;
            }
            o[d] = mfma16(vblk.vf[d], pb[0], o[d]);
          }
        }
      };
      // Keys a block ahead in one of two register sets, values into one set at the start of the block's own turn; every block is loaded once.
      KBlock k0, k1;
      VBlock v;
      int tb = t_begin;
      load_k(tb, k0);
      for (; tb + 2 * BT < t_end; tb += 2 * BT) {
        load_v(tb, v);
        load_k(tb + BT, k1);
        compute_block(tb, k0, v);
        load_v(tb + BT, v);
        load_k(tb + 2 * BT, k0);
        compute_block(tb + BT, k1, v);
      }
      if (tb + BT < t_end) {
        load_v(tb, v);
        load_k(tb + BT, k1);
        compute_block(tb, k0, v);
        load_v(tb + BT, v);
        compute_block(tb + BT, k1, v);
      } else {
        load_v(tb, v);
        compute_block(tb, k0, v);
      }
    }
    lsum += __shfl_xor(lsum, 16, 64);
    lsum += __shfl_xor(lsum, 32, 64);

    // one more state of this lane's column, wherever it comes from
    auto join = [&](float m2, float l2, auto o_of) {
      const float m_new = fmaxf(m, m2), mine = exp2f(m - m_new), its = exp2f(m2 - m_new);
      m = m_new;
      lsum = lsum * mine + l2 * its;
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        const f32x4 x = o_of(d);
        o[d] = o[d] * mine + x * its;
      }
    };
    // the other waves' states, in order, joined by the first wave
    auto gather = [&] {
      __syncthreads();  // (those of before have been read)
      if (wave > 0) {
        float* const at = s_state + ((wave - 1) * 64 + lane) * PITCH;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int i = 0; i < 4; i += 2) *reinterpret_cast<float2*>(at + d * 4 + i) = make_float2(o[d][i], o[d][i + 1]);
        *reinterpret_cast<float2*>(at + DT * 4) = make_float2(m, lsum);
      }
      __syncthreads();
      if (wave > 0) return;
#pragma unroll
      for (int w = 0; w < 3; ++w) {
        const float* const at = s_state + (w * 64 + lane) * PITCH;
        const float2 ml = *reinterpret_cast<const float2*>(at + DT * 4);
        join(ml.x, ml.y, [&](int d) {
          const float2 x = *reinterpret_cast<const float2*>(at + d * 4), y = *reinterpret_cast<const float2*>(at + d * 4 + 2);
          return f32x4{x.x, x.y, y.x, y.y};
        });
      }
    };
    if constexpr (SPLIT) {
      gather();
      if (PREFIX && wave > 0) continue;
    }
    // (the item is read again: what it says would hold registers through all of the above)
    int item_again = item;
    asm volatile("" : "+s"(item_again));
    const int4 it = items[PREFIX ? 2 * item_again : item_again];
    const Column c = column_of(it);
    const int row = c.row, head = c.head;
    const bool real = c.real;
    const int in_front = PREFIX ? 0 : it.w >> 16, slot = PREFIX ? it.w : in_front + (it.w & 0xffff);
    const int own_spans = PREFIX ? 1 : max(1, (it.z + span_len - 1) / span_len);
    const int64_t base = ((int64_t)row * n_q_heads + head) * max_spans;
    float* const o_at = part_o + base * DH + kg * 4;  // channels d * 16 + kg * 4 + i of slot 0
    if constexpr (PREFIX) {
      if (real) {
#pragma unroll
        for (int d = 0; d < DT; ++d) *reinterpret_cast<f32x4*>(o_at + (int64_t)slot * DH + d * 16) = o[d];
        if (kg == 0) *reinterpret_cast<float2*>(part_ml + (base + slot) * 2) = make_float2(m, lsum);
      }
    } else {
      // The waves share the joining out as well where there is much of it.
      const bool together = SPLIT && in_front + own_spans > kJoinedAlone;
      if (SPLIT && wave > 0 && !together) continue;
      if (own_spans > 1) {
        // The spans of a row are made on different XCDs, whose L2s do not see each other: partials are stored and read past them, the wave waits
        // until its stores have arrived, and only then is the span counted.  The last one puts the counter back for the next launch.
        bool last = false;
        if (!SPLIT || wave == 0) {
          if (real) {
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
              for (int i = 0; i < 4; ++i) store_agent(o_at + (int64_t)slot * DH + d * 16 + i, o[d][i]);
            if (kg == 0) {
              store_agent(part_ml + (base + slot) * 2, m);
              store_agent(part_ml + (base + slot) * 2 + 1, lsum);
            }
          }
          asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
          unsigned before = 0;
          unsigned* const done = spans_done + (int64_t)row * Hkv + kvh;
          if (lane == 0) before = __hip_atomic_fetch_add(done, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
          before = __builtin_amdgcn_readfirstlane(before);
          last = before + 1 == (unsigned)own_spans;
          if (last && lane == 0) __hip_atomic_store(done, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        if (together) {
          if (threadIdx.x == 0) s_last = last;  // (that of the unit before was read in front of a barrier)
          __syncthreads();
          last = s_last;
        }
        if (!last) continue;
      }
      if (own_spans > 1 || (SPLIT && wave > 0)) {
        m = kNegBig;
        lsum = 0.f;
#pragma unroll
        for (int d = 0; d < DT; ++d) o[d] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
      // in the order of the spans, whoever is last (a row's only span, in registers, first)
      const int all = in_front + (own_spans > 1 ? own_spans : 0);
      if (together) {
        // a quarter to a wave, four on their way at a time
        const int from_k = (wave * all) >> 2, to_k = ((wave + 1) * all) >> 2;
        for (int k = from_k; k < to_k; k += 4) {
          float2 ml[4];
          float2 x[4][2 * DT];
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const int at = min(k + u, to_k - 1);
            const float* const from = o_at + (int64_t)at * DH;
            ml[u] = load_agent2(part_ml + (base + at) * 2);
#pragma unroll
            for (int d = 0; d < DT; ++d) {
              x[u][2 * d] = load_agent2(from + d * 16);
              x[u][2 * d + 1] = load_agent2(from + d * 16 + 2);
            }
          }
#pragma unroll
          for (int u = 0; u < 4; ++u)
            if (k + u < to_k)
              join(ml[u].x, ml[u].y, [&](int d) { return f32x4{x[u][2 * d].x, x[u][2 * d].y, x[u][2 * d + 1].x, x[u][2 * d + 1].y}; });
        }
        gather();
        if (wave > 0) continue;
      } else {
        for (int k = 0; k < in_front; ++k) {
          const float* const from = o_at + (int64_t)k * DH;
          const float2 ml = *reinterpret_cast<const float2*>(part_ml + (base + k) * 2);
          f32x4 x[DT];
#pragma unroll
          for (int d = 0; d < DT; ++d) x[d] = *reinterpret_cast<const f32x4*>(from + d * 16);
          join(ml.x, ml.y, [&](int d) { return x[d]; });
        }
        for (int k = in_front; k < all; ++k) {
          const float* const from = o_at + (int64_t)k * DH;
          const float2 ml = load_agent2(part_ml + (base + k) * 2);
          f32x4 x[DT];
#pragma unroll
          for (int d = 0; d < DT; ++d) {
            const float2 lo = load_agent2(from + d * 16), hi = load_agent2(from + d * 16 + 2);
            x[d] = f32x4{lo.x, lo.y, hi.x, hi.y};
          }
          join(ml.x, ml.y, [&](int d) { return x[d]; });
        }
      }
      if (real) {
        const float scale = it.z > 0 ? out_scale / lsum : 0.f;  // (a row without tokens gives zeros)
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          bf16x4 v4;
#pragma unroll
          for (int i = 0; i < 4; ++i) v4[i] = (bf16)(o[d][i] * scale);
          *reinterpret_cast<bf16x4*>(out + operand_offset(out_lay, row, head * DH + d * 16 + kg * 4)) = v4;
        }
      }
    }
  }
}

// ---- many columns ------------------------------------------------------------------------------------------------------------

// One workgroup of four waves per (item, K/V head).  NWC waves, two or four, have 32 columns each, and 4 / NWC waves share the tokens of a block
// out for the same columns.  A block of 64 tokens of K and V^T is staged in LDS, double buffered and swizzled,
// and feeds the 32x32x16 MFMAs of all columns; scores are formed transposed, with their rows permuted so that a lane's elements are the
// consecutive tokens that it supplies to O^T += V^T P^T, as in the prefill kernel, whose masks are not needed here: a prefix is whole pages.
// Bound: reading the pages up to about a hundred columns, MFMA beyond (and storing the partials: 512 rows of 64 heads behind 1664 tokens, 27.9
// GFLOP and 34 MB of partials, 48 us).
template <int DH, int NWC, bool KV8>
__global__ __launch_bounds__(256, 2) void attn_prefix_kernel(const bf16* __restrict__ q, int64_t ld, int n_q_heads, KvLayout kv,
                                                                            const int4* __restrict__ items, const int32_t* __restrict__ count,
                                                                            const int32_t* __restrict__ block_tables, int max_pages_per_seq,
                                                                            float* __restrict__ part_o, float* __restrict__ part_ml,
                                                                            int max_spans, float scale_log2) {
  constexpr int NWT = 4 / NWC;               // waves that share the tokens out
  constexpr int NH = 2;                      // 32-token halves of a block
  constexpr int BLK = 32 * NH, NPG = BLK / 16;
  constexpr int KS = DH / 16, DT = DH / 32;  // k-steps of the scores, 32-channel tiles of the output
  constexpr int CR = DH / 8;                 // 16-byte chunks of a key in LDS
  constexpr int RWK = DH == 128 ? 1 : 2;     // keys in a 256-byte bank window
  constexpr int HEAD = 16 * DH;              // elements of a page, one K/V head
  constexpr int HALF = 32 * DH;              // elements of a half
  __shared__ __attribute__((aligned(16))) bf16 lds[2][2][NH][HALF];  // [K, V][buffer]
  bf16* const sK = &lds[0][0][0][0];
  bf16* const sV = &lds[1][0][0][0];

  const int Hkv = kv.n_kv_heads, G = n_q_heads / Hkv;
  const int item = blockIdx.x / Hkv, kvh = blockIdx.x - item * Hkv;
  if (item >= *count) return;
  const int4 it = items[2 * item], it2 = items[2 * item + 1];
  const int first_page = it2.x, n_pages = it2.y, n_tokens = n_pages * 16;
  const int32_t* const table = block_tables + (int64_t)it2.z * max_pages_per_seq + first_page;
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, kg = lane >> 5;
  const int wc = w % NWC, wt = w / NWC;

  // the lane's column; columns behind the last are computed as the last one and never stored
  struct Column {
    int row, head;
    bool real;
  };
  auto column_of = [&](int4 x) {
    const int col = x.y + wc * 32 + l32, c = min(col, x.z - 1), r = c / G;
    return Column{x.x + r, kvh * G + c - r * G, col < x.z};
  };
  const bool idle = it.y + wc * 32 >= it.z;  // (the whole wave)
  bf16x8 qf[KS];
  {
    const Column c = column_of(it);
    const bf16* qp = q + (int64_t)c.row * ld + (int64_t)c.head * DH + kg * 8;
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) qf[kk] = ld_bf16x8(qp + kk * 16);
  }
  f32x16 o[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
  float m = kNegBig, lsum = 0.f;

  // token of this lane's row r = l32 in the score tile: (r/16)*16 + ((r%8)/4)*8 + ((r/8)%2)*4 + r%4
  const int krow = (l32 >> 4) * 16 + ((l32 >> 2) & 1) * 8 + ((l32 >> 3) & 1) * 4 + (l32 & 3);
  const int k_swz = (krow / RWK) % CR;

  // Staging.  Pages of a block are looked up a block before they are requested; entries behind the last page repeat it.  16-bit pools go
  // straight into LDS, 1 KiB to an instruction, each lane fetching what the swizzle wants at its place: wave w takes NPG / 4 pages of
  // keys, and as much of the values, WPH waves to a half.  8-bit pools go through registers and are converted when they have arrived.
  constexpr int NCH = BLK * CR / 256;                      // 8-element chunks of K, and of V, per thread
  constexpr int TPI = 512 / DH, NJ = 16 / TPI;             // keys of an instruction, instructions of a page
  constexpr int WPH = 4 / NH, NV = DH / WPH / 16;          // waves of a half of V, instructions of one
  constexpr int KP = KV8 ? NPG : NPG / 4;
  const int v_row = lane >> 2, v_chunk = (lane & 3) ^ ((v_row >> 2) & 3);
  // the pages that this thread asks for something of: of keys those of its wave, of values its own (8 bits: all of the block, for both)
  int k_page[KP], v_page = 0;
  auto look_up = [&](int b) {
    auto id = [&](int i) { return table[min(b * NPG + i, n_pages - 1)]; };
    if constexpr (KV8) {
#pragma unroll
      for (int p = 0; p < KP; ++p) k_page[p] = __builtin_amdgcn_readfirstlane(id(p));
    } else {
#pragma unroll
      for (int p = 0; p < KP; ++p) k_page[p] = id(w * KP + p);
      v_page = id(w / WPH * 2 + (v_chunk >> 1));
    }
  };
  uint2 kraw[KV8 ? NCH : 1], vraw[KV8 ? NCH : 1];
  const unsigned k_lds = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char*)sK;
  const unsigned v_lds = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char*)sV;
  auto request = [&](unsigned lds_addr, const bf16* from) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds_addr), "v"(from) : "memory");
  };
  auto request_from = [&](unsigned lds_addr, const bf16* base, unsigned bytes) {  // base: the same for the wave
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds_addr), "v"(bytes), "s"(base) : "memory");
  };
  auto load_block = [&](int buf) {
    if constexpr (KV8) {
#pragma unroll
      for (int j = 0; j < NCH; ++j) {
        const int ci = tid + 256 * j;
        // K: consecutive threads walk the pool in address order - the 8 chunks of a 64-byte piece, the 16 tokens of the page, the
        // pieces of the row, the pages of the block
        const int kq = ci % 8, kt16 = (ci / 8) % 16, kpiece = (ci / 128) % (CR / 8);
        const int vr = (ci >> 2) % DH, vc = ci & 3;
        constexpr int PER = 256 / (16 * CR);  // pages of 256 chunks of keys: 1 or 2
        const int kp = PER == 1 ? k_page[j] : w < 2 ? k_page[(PER * j) % KP] : k_page[(PER * j + 1) % KP];
        const int v0 = k_page[256 * j / (DH * 4) * 2], v1 = k_page[256 * j / (DH * 4) * 2 + 1], vp = vc < 2 ? v0 : v1;
        kraw[j] = *reinterpret_cast<const uint2*>((const uint8_t*)kv.k_pool + ((int64_t)kp * Hkv + kvh) * HEAD + ((kpiece * 16 + kt16) * 64 + kq * 8));
        vraw[j] = *reinterpret_cast<const uint2*>((const uint8_t*)kv.v_pool + ((int64_t)vp * Hkv + kvh) * HEAD + (vr * 16 + (vc & 1) * 8));
      }
    } else {
#pragma unroll
      for (int p = 0; p < KP; ++p) {
        const int pg = w * KP + p;  // of the block
        const bf16* kp = (const bf16*)kv.k_pool + ((int64_t)__builtin_amdgcn_readfirstlane(k_page[p]) * Hkv + kvh) * HEAD;
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          const int slot = j * TPI + lane / CR, ktok = (pg & 1) * 16 + slot, kc = (lane % CR) ^ ((ktok / RWK) % CR);
          request_from(k_lds + ((buf * NH + (pg >> 1)) * HALF + ((pg & 1) * 16 + j * TPI) * DH) * 2, kp, ((kc / 4) * 512 + slot * 32 + kc % 4 * 8) * 2);
        }
      }
      const int half = w / WPH, part = w % WPH;
      const bf16* vp = (const bf16*)kv.v_pool + ((int64_t)v_page * Hkv + kvh) * HEAD + (part * (DH / WPH) + v_row) * 16 + (v_chunk & 1) * 8;
#pragma unroll
      for (int j = 0; j < NV; ++j)
        request(v_lds + ((buf * NH + half) * HALF + (part * (DH / WPH) + j * 16) * 32) * 2, vp + j * 256);
    }
  };
  // block b has arrived in buffer buf for all waves
  auto settle = [&](int b, int buf) {
    if constexpr (KV8) {
#pragma unroll
      for (int j = 0; j < NCH; ++j) {
        const int ci = tid + 256 * j;
        const int kq = ci % 8, kt16 = (ci / 8) % 16, kpiece = (ci / 128) % (CR / 8), kpg = ci / (16 * CR);
        const int ksub = kpg >> 1, ktok = (kpg & 1) * 16 + kt16, kc = kpiece * 8 + kq;
        const int vsub = ci / (DH * 4), vr = (ci >> 2) % DH, vc = ci & 3;
        union {
          uint32_t u[4];
          bf16x8 x;
        } k8, v8;
        e4m3x4_to_bf16x4(kraw[j].x, k8.u[0], k8.u[1]);
        e4m3x4_to_bf16x4(kraw[j].y, k8.u[2], k8.u[3]);
        e4m3x4_to_bf16x4(vraw[j].x, v8.u[0], v8.u[1]);
        e4m3x4_to_bf16x4(vraw[j].y, v8.u[2], v8.u[3]);
        st_bf16x8(sK + (buf * NH + ksub) * HALF + ktok * DH + ((kc ^ ((ktok / RWK) % CR)) << 3), k8.x);
        st_bf16x8(sV + (buf * NH + vsub) * HALF + vr * 32 + ((vc ^ ((vr >> 2) & 3)) << 3), v8.x);
      }
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    if ((b + 1) * BLK > n_tokens) {  // what stands behind the span is the last page again: zeros, so that no infinity meets a weight of zero
#pragma unroll
      for (int j = 0; j < NCH; ++j) {
        const int ci = tid + 256 * j, vsub = ci / (DH * 4), vr = (ci >> 2) % DH, vc = ci & 3;
        if (b * BLK + vsub * 32 + vc * 8 >= n_tokens)
          st_bf16x8(sV + (buf * NH + vsub) * HALF + vr * 32 + ((vc ^ ((vr >> 2) & 3)) << 3), zero_bf16x8());
      }
      __syncthreads();
    }
  };

  const int n_blocks = (n_tokens + BLK - 1) / BLK;
  look_up(0);
  load_block(0);
  look_up(1);
  settle(0, 0);
  // The queries are used, and so waited for, in front of the loop: inside it every turn would wait for them again, and so for the
  // requests of the next block, which are behind them in the same counter.
#pragma unroll
  for (int kk = 0; kk < KS; ++kk) asm volatile("" : "+v"(qf[kk]));
  for (int b = 0, buf = 0; b < n_blocks; ++b, buf ^= 1) {
    const bool more = b + 1 < n_blocks;
    if (more) load_block(buf ^ 1);
    look_up(b + 2);
#pragma unroll
    for (int sub = 0; sub < NH / NWT; ++sub) {
      const int half = NWT == 1 ? sub : wt, kb = b * BLK + half * 32;
      if (kb >= n_tokens || idle) continue;
      const bf16* const kh = sK + (buf * NH + half) * HALF + krow * DH;
      const bf16* const vh = sV + (buf * NH + half) * HALF;
      f32x16 sc;
#pragma unroll
      for (int i = 0; i < 16; ++i) sc[i] = 0.f;
      bf16x8 kf[KS];  // all fragments first: one LDS round trip
#pragma unroll
      for (int kk = 0; kk < KS; ++kk) kf[kk] = ld_bf16x8(kh + (((kk * 2 + kg) ^ k_swz) << 3));
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int kk = 0; kk < KS; ++kk) sc = mfma32(kf[kk], qf[kk], sc);
      __builtin_amdgcn_sched_barrier(0);
      // on their way during the softmax (8-bit pools, whose codes wait in registers: a quarter of them)
      constexpr int VD = KV8 && NWC == 4 && DT > 2 ? 1 : DT;
      bf16x8 vf[VD][2];
      auto fragment = [&](int d, int st) {
        const int r = d * 32 + l32;
        return ld_bf16x8(vh + r * 32 + (((st * 2 + kg) ^ ((r >> 2) & 3)) << 3));
      };
#pragma unroll
      for (int d = 0; d < VD; ++d)
#pragma unroll
        for (int st = 0; st < 2; ++st) vf[d][st] = fragment(d, st);
      __builtin_amdgcn_sched_barrier(0);
      // element i of this lane is token kb + (i/8)*16 + kg*8 + i%8 of its column
      if (kb + 32 > n_tokens) {  // (an odd number of pages)
#pragma unroll
        for (int i = 8; i < 16; ++i) sc[i] = kNegBig;
      }
      float mx = sc[0];
#pragma unroll
      for (int i = 1; i < 16; ++i) mx = fmaxf(mx, sc[i]);
      mx = fmaxf(mx, __shfl_xor(mx, 32, 64)) * scale_log2;  // scale > 0: max commutes with it
      if (__any(mx > m + kRescaleSlack)) {
        const float m_new = fmaxf(m, mx);
        const float alpha = __builtin_amdgcn_exp2f(m - m_new);
        lsum *= alpha;
        m = m_new;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[d][i] *= alpha;
      }
      bf16x8 pb[2];
      float psum = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float pv = __builtin_amdgcn_exp2f(fmaf(sc[i], scale_log2, -m));
        psum += pv;
        pb[i >> 3][i & 7] = (bf16)pv;  // (rounded for the MFMA alone: the sum is of what it was)
      }
      lsum += psum;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int st = 0; st < 2; ++st) o[d] = mfma32(d < VD ? vf[d < VD ? d : 0][st] : fragment(d, st), pb[st], o[d]);
    }
    if (more) settle(b + 1, buf ^ 1);
  }
  lsum += __shfl_xor(lsum, 32, 64);

  // waves that had other tokens of the same columns: joined through LDS, in order
  if constexpr (NWT > 1) {
    constexpr int PITCH = DT * 16 + 2;  // floats of a lane: its o, m, l; (an even number that is no multiple of 32 banks)
    static_assert((NWT - 1) * NWC * 64 * PITCH * 4 <= (int)sizeof(lds), "every wave but the first of its columns leaves its state");
    float* const state = reinterpret_cast<float*>(&lds[0][0][0][0]);
    __syncthreads();
    if (wt > 0) {
      float* at = state + (((wt - 1) * NWC + wc) * 64 + lane) * PITCH;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; i += 2) *reinterpret_cast<float2*>(at + d * 16 + i) = make_float2(o[d][i], o[d][i + 1]);
      *reinterpret_cast<float2*>(at + DT * 16) = make_float2(m, lsum);
    }
    __syncthreads();
    if (wt > 0) return;
#pragma unroll
    for (int t = 0; t < NWT - 1; ++t) {
      const float* at = state + ((t * NWC + wc) * 64 + lane) * PITCH;
      const float2 ml = *reinterpret_cast<const float2*>(at + DT * 16);
      const float m_new = fmaxf(m, ml.x), mine = __builtin_amdgcn_exp2f(m - m_new), its = __builtin_amdgcn_exp2f(ml.x - m_new);
      m = m_new;
      lsum = lsum * mine + ml.y * its;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
          const float2 v = *reinterpret_cast<const float2*>(at + d * 16 + i);
          o[d][i] = o[d][i] * mine + v.x * its;
          o[d][i + 1] = o[d][i + 1] * mine + v.y * its;
        }
    }
  }
  // (the item is read again: what it says would hold registers through all of the above)
  int item_again = item;
  asm volatile("" : "+s"(item_again));
  const int4 again = items[2 * item_again];
  const Column c = column_of(again);
  if (!c.real) return;
  const int64_t slot = ((int64_t)c.row * n_q_heads + c.head) * max_spans + again.w;
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *reinterpret_cast<f32x4*>(part_o + slot * DH + d * 32 + g * 8 + kg * 4) =
          f32x4{o[d][g * 4], o[d][g * 4 + 1], o[d][g * 4 + 2], o[d][g * 4 + 3]};
  if (kg == 0) *reinterpret_cast<float2*>(part_ml + slot * 2) = make_float2(m, lsum);
}

}  // namespace

int attn_prefix_items_most(int max_batch, int n_q_heads, int n_kv_heads) {
  return max_batch * (n_q_heads / n_kv_heads) / 16 + max_batch + (1024 + n_kv_heads - 1) / n_kv_heads;
}

// Spans of what rows have behind their prefix: as in decode attention where four waves share one, shorter where each is a wave's (512 / 1024 /
// 2048 tokens, 8 K/V heads: 256 rows of up to 400 tokens 72 / 68 / 68 us, 512 of up to 1000 255 / 221 / 215; two groups of 8 rows of 64 heads, up to 1000, 52 / 63 / 63).
int attn_shared_span(int batch, int n_kv_heads) {
  return rows_split(batch, n_kv_heads) ? attn_decode_span(batch, n_kv_heads) : 1024;
}

hipError_t launch_attn_shared_plan(const SharedBatch& b, const SharedScratch& sc, hipStream_t s) {
  if (b.batch <= 0) return hipSuccess;
  const Form f = form_of(b.batch, b.n_groups, b.n_q_heads, b.n_kv_heads);
  const int workgroups = b.n_groups > 0 ? std::min(64, (b.batch + kPlanRows - 1) / kPlanRows) : 1;
  const PlanArgs a{b, f.columns, f.wanted, items_of(b, f), sc.row_pages, sc.group, sc.done, sc.counts, sc.prefix_items, sc.row_items};
  shared_plan_kernel<<<workgroups, kPlanThreads, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_attn_shared(const SharedBatch& b, const SharedScratch& sc, const void* q, int64_t ld, const KvLayout& kv, float* part_o,
                              float* part_ml, unsigned* spans_done, int max_spans, void* out, OperandLayout out_layout, hipStream_t s) {
  if (b.batch <= 0) return hipSuccess;
  // 8-bit pools hold value / scale: the key scale joins the softmax scale, the value scale the final division, behind the partials
  const float scale_log2 = 1.4426950408889634f / sqrtf((float)kv.head_dim) * (kv.fp8 ? kv.k_scale : 1.0f);
  const float out_scale = kv.fp8 ? kv.v_scale : 1.0f;
  const Form f = form_of(b.batch, b.n_groups, b.n_q_heads, b.n_kv_heads);
  const int64_t prefix_units = (int64_t)items_of(b, f) * b.n_kv_heads;
  const int64_t row_units = (int64_t)b.batch * ((b.max_pages_per_seq * 16 + b.span_len - 1) / b.span_len) * b.n_kv_heads;
  const bool rows_alone = rows_split(b.batch, b.n_kv_heads);
  // (workgroups of the sixteen-column kernel take one unit after another)
  auto grid_of = [](int64_t units, bool split) { return (unsigned)std::min<int64_t>(split ? units : (units + 3) / 4, 8 * kResident); };
#define TDP_COLUMNS_(DH, KV8, PREFIX, SPLIT, grid, items, count)                                                                         \
  attn_columns_kernel<DH, KV8, PREFIX, SPLIT><<<grid, 256, 0, s>>>((const bf16*)q, ld, b.n_q_heads, kv, items, count, b.block_tables,    \
                                                                   b.max_pages_per_seq, part_o, part_ml, spans_done, max_spans, b.span_len, \
                                                                   (bf16*)out, out_layout, scale_log2, out_scale)
#define TDP_PREFIX_(DH, NWC, KV8)                                                                                                   \
  attn_prefix_kernel<DH, NWC, KV8><<<(unsigned)prefix_units, 256, 0, s>>>((const bf16*)q, ld, b.n_q_heads, kv, sc.prefix_items, sc.counts, \
                                                                          b.block_tables, b.max_pages_per_seq, part_o, part_ml, max_spans, \
                                                                          scale_log2)
#define TDP_SHARED(DH, KV8)                                                                                   \
  do {                                                                                                        \
    if (b.n_groups > 0) {                                                                                     \
      if (f.columns == 16)                                                                                    \
        TDP_COLUMNS_(DH, KV8, true, true, grid_of(prefix_units, true), sc.prefix_items, sc.counts);           \
      else if (f.columns == 64) TDP_PREFIX_(DH, 2, KV8);                                                      \
      else TDP_PREFIX_(DH, 4, KV8);                                                                           \
    }                                                                                                         \
    const unsigned rows_grid = grid_of(row_units, rows_alone);                                                \
    if (rows_alone) TDP_COLUMNS_(DH, KV8, false, true, rows_grid, sc.row_items, sc.counts + 1);               \
    else TDP_COLUMNS_(DH, KV8, false, false, rows_grid, sc.row_items, sc.counts + 1);                         \
  } while (0)
  if (kv.head_dim == 128) {
    if (kv.fp8) TDP_SHARED(128, true); else TDP_SHARED(128, false);
  } else {
    if (kv.fp8) TDP_SHARED(64, true); else TDP_SHARED(64, false);
  }
#undef TDP_SHARED
#undef TDP_PREFIX_
#undef TDP_COLUMNS_
  return hipGetLastError();
}

}  // namespace tdp
