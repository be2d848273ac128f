// Block tables of a paged cache on the device: rows that continue other rows (fork, with reference counts and fresh pages), pages moved
// to the front of the pool (compact), and the copies of page contents that both ask for.
//
// Both decisions need "the k-th free page in order".  A survey notes a bit for every page and a count for every chunk of 4096 pages;
// whoever needs pages sums the counts in front of a chunk (1024 chunks at most) and the bits of its 64 words, a word to a lane.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stdio.h>

#include <algorithm>
#include <new>

#include "../../include/tdp.h"
#include "tdp_device.h"
#include "tdp_kernels.h"

namespace tdp {

int probe_fail(int code, const char* msg);  // sets the thread's error message (stage.hip)

namespace {

typedef unsigned long long u64;
constexpr int kChunk = 4096, kChunkWords = kChunk / 64, kChunksMost = 1024, kRowsMost = 8192;
constexpr int kPage = 16;

__device__ __forceinline__ int pages_of(int tokens) { return (tokens + kPage - 1) / kPage; }

// A lane's value plus those of the lanes in front of it.
__device__ __forceinline__ int wave_scan(int v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    const int up = __shfl_up(v, o, 64);
    if (lane >= o) v += up;
  }
  return v;
}
// The same over a workgroup of 1024, and the sum of all; `part` (LDS, 16) is used again only behind a barrier.
__device__ __forceinline__ int block_scan(int v, int* part, int* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  v = wave_scan(v);
  if (lane == 63) part[wave] = v;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < 16; ++w) {
    before += w < wave ? part[w] : 0;
    all += part[w];
  }
  *total = all;
  return v + before;
}

// before[c] = marked pages in the chunks in front of chunk c, c = 0 .. n; 256 threads.
__device__ __forceinline__ void sum_chunks(const int* counts, int n, int* before, int* part) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int v[4], own = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[i] = tid * 4 + i < n ? counts[tid * 4 + i] : 0;
    own += v[i];
  }
  const int incl = wave_scan(own);
  if (lane == 63) part[wave] = incl;
  __syncthreads();
  int at = incl - own;
#pragma unroll
  for (int w = 0; w < 3; ++w) at += w < wave ? part[w] : 0;
  if (tid == 0) before[0] = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    at += v[i];
    if (tid * 4 + i < n) before[tid * 4 + i + 1] = at;
  }
  __syncthreads();
}
// The last chunk with before[c] <= k (k below the number of marked pages).
__device__ __forceinline__ int chunk_of(const int* before, int n, int k) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (before[mid] <= k) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// One wave: give(k, page) for every marked page of chunk c whose number k among the marked pages lies in [first, last).
template <typename Give>
__device__ __forceinline__ void enumerate_chunk(const u64* marks, int c, int before, int first, int last, Give give) {
  u64 word = marks[(int64_t)c * kChunkWords + (threadIdx.x & 63)];
  const int own = __popcll(word);
  int k = before + wave_scan(own) - own;
  if (k >= last || k + own <= first) return;
  const int page0 = c * kChunk + (threadIdx.x & 63) * 64;
  while (word && k < last) {
    const int bit = __ffsll((long long)word) - 1;
    if (k >= first) give(k, page0 + bit);
    word &= word - 1;
    ++k;
  }
}

// ---- fork ------------------------------------------------------------------------------------------------------------------------

struct ForkArgs {
  const int32_t *parents, *src_tables, *src_lens, *add;
  int n_src, add_all, n_dst, width, num_pages, chunks;
  const int32_t* refs_in;
  int32_t *refs_out, *dst_tables, *dst_lens, *copies, *status;
  // scratch
  u64* marks;           // a bit for every free page
  int* counts;          // free pages of every chunk
  int* row_first;       // [n_dst] number of the row's first fresh page among all
  int* row_from;        // [n_dst] first table entry that is fresh; bit 30: it is a copy
  int* src_children;    // [n_src] rows that continue it, times two, plus 1 if one of them takes over the last page
  int* totals;          // fresh pages, refused rows
};
constexpr int kCopies = 1 << 30;

__device__ __forceinline__ int parent_of(const ForkArgs& a, int r) { return a.parents ? a.parents[r] : r < a.n_src ? r : -1; }

// Workgroup 0 looks at the rows, the others at 4096 pages each.  Nothing that the second kernel needs is read from refs again,
// so that it may change them in place.  Bound: launching, and loads that wait for each other: 3 us of 4 rows, 4 us of 512 rows and 8192 pages.
__global__ __launch_bounds__(1024) void pages_survey_kernel(const ForkArgs a) {
  __shared__ int part[16];
  __shared__ int bad;
  extern __shared__ int lds[];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (blockIdx.x > 0) {
    const int c = blockIdx.x - 1;
    int found = 0;
#pragma unroll
    for (int i = 0; i < kChunkWords / 16; ++i) {
      const int w = wave * (kChunkWords / 16) + i, p = c * kChunk + w * 64 + lane;
      const int refs = p < a.num_pages ? a.refs_in[p] : 1;
      if (p < a.num_pages && a.refs_out != a.refs_in) a.refs_out[p] = refs;
      const u64 word = __ballot(refs == 0);
      found += __popcll(word);
      if (lane == 0) a.marks[(int64_t)c * kChunkWords + w] = word;
    }
    if (lane == 0) part[wave] = found;
    __syncthreads();
    if (tid == 0) {
      for (int w = 1; w < 16; ++w) found += part[w];
      a.counts[c] = found;
    }
    return;
  }
  int* const first = lds;               // [n_src] the lowest row that continues it; -1: and takes over its last page
  int* const children = lds + a.n_src;  // [n_src]
  if (tid == 0) bad = 0;
  for (int s = tid; s < a.n_src; s += 1024) {
    first[s] = 0x7fffffff;
    children[s] = 0;
  }
  __syncthreads();
  for (int r = tid; r < a.n_dst; r += 1024) {
    const int p = parent_of(a, r);
    if (p >= 0 && p < a.n_src) {
      atomicMin(&first[p], r);
      atomicAdd(&children[p], 1);
    }
  }
  const int most = a.width * kPage;
  for (int s = tid; s < a.n_src; s += 1024)
    if (a.src_lens[s] < 0 || a.src_lens[s] > most) bad = 1;  // (all of them count as one: counted below where they are continued)
  __syncthreads();
  int base = 0, refused = 0;
  for (int r0 = 0; r0 < a.n_dst; r0 += 1024) {
    const int r = r0 + tid;
    int need = 0, from = 0, no = 0;
    if (r < a.n_dst) {
      const int p = parent_of(a, r), room = a.add ? a.add[r] : a.add_all;
      const bool known = p >= -1 && p < a.n_src;
      const int len = known && p >= 0 ? a.src_lens[p] : 0;
      no = !known || len < 0 || len > most || room < 0 || room > most - len;
      if (!no) {
        from = pages_of(len);
        if (len % kPage) {
          const int page = a.src_tables[(int64_t)p * a.width + len / kPage];
          no = page < 0 || page >= a.num_pages;
          if (!no && first[p] == r && a.refs_in[page] == 1) first[p] = -1;
          else from = len / kPage | kCopies;
        }
        need = no ? 0 : pages_of(len + room) - (from & ~kCopies);
      }
    }
    int total;
    const int incl = block_scan(need, part, &total);
    if (r < a.n_dst) {
      a.row_first[r] = base + incl - need;
      a.row_from[r] = from;
    }
    base += total;
    refused += __syncthreads_count(no);
  }
  for (int s = tid; s < a.n_src; s += 1024) a.src_children[s] = children[s] * 2 + (first[s] == -1);
  if (tid == 0) {
    a.totals[0] = base;
    a.totals[1] = refused ? refused : bad;
  }
}

// Workgroup i makes new row i and settles the references of old row i.  Bound: loads that wait for each other (the chunks' counts, the parent,
// its entries, their references): 3.5 us of 4 rows, 5 to 7.5 us of 512 rows of up to 90 pages.
__global__ __launch_bounds__(256) void pages_fork_kernel(const ForkArgs a) {
  __shared__ int before[kChunksMost + 1], part[4];
  const int tid = threadIdx.x, wave = tid >> 6, i = blockIdx.x;
  sum_chunks(a.counts, a.chunks, before, part);
  const int wanted = a.totals[0], refused = a.totals[1], free = before[a.chunks];
  const bool done = wanted <= free && !refused;
  if (i == 0 && tid == 0) {
    a.status[0] = max(0, wanted - free);
    a.status[1] = refused;
    a.status[2] = done ? wanted : 0;
    a.status[3] = free;
  }
  if (!done) {
    if (i < a.n_dst && tid < 2) a.copies[2 * (int64_t)i + tid] = -1;
    return;
  }
  if (i < a.n_src) {
    const int children = a.src_children[i] >> 1, kept = a.src_children[i] & 1, len = a.src_lens[i];
    const int32_t* const row = a.src_tables + (int64_t)i * a.width;
    const int full = len / kPage, change = children - 1;
    auto add = [&](int page, int n) {
      if (page >= 0 && page < a.num_pages) atomicAdd(&a.refs_out[page], n);
    };
    if (change)
      for (int e = tid; e < full; e += 256) add(row[e], change);
    if (tid == 0 && len % kPage && !kept) add(row[full], -1);
  }
  if (i >= a.n_dst) return;
  const int p = parent_of(a, i), len = p >= 0 ? a.src_lens[p] : 0, new_len = len + (a.add ? a.add[i] : a.add_all);
  const int from = a.row_from[i] & ~kCopies, held = pages_of(new_len), first = a.row_first[i], last = first + held - from;
  const bool copies = (a.row_from[i] & kCopies) != 0;
  const int32_t* const old = a.src_tables + (int64_t)max(p, 0) * a.width;
  int32_t* const row = a.dst_tables + (int64_t)i * a.width;
  for (int e = tid; e < a.width; e += 256)
    if (e < from) row[e] = old[e];
    else if (e >= held) row[e] = -1;
  if (last > first) {
    for (int c = chunk_of(before, a.chunks, first) + wave; c < a.chunks && before[c] < last; c += 4)
      enumerate_chunk(a.marks, c, before[c], first, last, [&](int k, int page) {
        row[from + k - first] = page;
        a.refs_out[page] = 1;
        if (k == first) a.copies[2 * (int64_t)i + 1] = copies ? page : -1;
      });
  } else if (tid == 64) {
    a.copies[2 * (int64_t)i + 1] = -1;
  }
  if (tid == 0) {
    a.copies[2 * (int64_t)i] = copies ? old[from] : -1;
    a.dst_lens[i] = new_len;
  }
}

// ---- compact ---------------------------------------------------------------------------------------------------------------------
//
// Five launches, each for what the whole of the one in front of it has to have found: how often the rows name a page; which pages are free, which
// only the rows hold; their order; the moves; the tables.  Of 5 rows 2.3, 2.2, 4.8, 3.5 and 2.2 us, of 256 rows 2.9, 4.5, 6.9, 5.1 and 2.4: launches
// and loads that wait for each other, with nothing that takes bandwidth before the copies.

struct CompactArgs {
  const int32_t *src_tables, *lens;
  int n_rows, width, num_pages, chunks, max_moves;
  const int32_t* refs_in;
  int32_t *refs_out, *dst_tables, *moves, *status;
  // scratch
  u64 *free_marks, *movable_marks;
  int *free_counts, *movable_counts, *used_counts;
  int* named;      // [num_pages] entries of the rows that name a page; zero between calls
  int* moved;      // [num_pages] the id that it has behind the call
  int *from, *to;  // [num_pages] the k-th highest movable page, the k-th lowest free one
  int* totals;     // refused rows; zero between calls
};

__global__ __launch_bounds__(256) void compact_count_kernel(const CompactArgs a) {
  const int r = blockIdx.x, len = a.lens[r];
  bool no = len < 0 || len > a.width * kPage;
  if (!no)
    for (int e = threadIdx.x; e < pages_of(len); e += 256) {
      const int page = a.src_tables[(int64_t)r * a.width + e];
      if (page >= 0 && page < a.num_pages) atomicAdd(&a.named[page], 1);
      else no = true;
    }
  if (__syncthreads_or(no) && threadIdx.x == 0) atomicAdd(&a.totals[0], 1);
}

__global__ __launch_bounds__(1024) void compact_survey_kernel(const CompactArgs a) {
  __shared__ int part[3][16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, c = blockIdx.x;
  int found[3] = {0, 0, 0};
#pragma unroll
  for (int i = 0; i < kChunkWords / 16; ++i) {
    const int w = wave * (kChunkWords / 16) + i, p = c * kChunk + w * 64 + lane;
    const bool in = p < a.num_pages;
    const int refs = in ? a.refs_in[p] : -1, named = in ? a.named[p] : 0;
    if (in) {
      a.named[p] = 0;
      a.moved[p] = p;
      if (a.refs_out != a.refs_in) a.refs_out[p] = refs;
    }
    const u64 free = __ballot(refs == 0), movable = __ballot(refs > 0 && refs == named);
    found[0] += __popcll(free);
    found[1] += __popcll(movable);
    found[2] += __popcll(__ballot(refs > 0));
    if (lane == 0) {
      a.free_marks[(int64_t)c * kChunkWords + w] = free;
      a.movable_marks[(int64_t)c * kChunkWords + w] = movable;
    }
  }
  if (lane == 0)
    for (int j = 0; j < 3; ++j) part[j][wave] = found[j];
  __syncthreads();
  if (tid < 3) {
    int sum = 0;
    for (int w = 0; w < 16; ++w) sum += part[tid][w];
    (tid == 0 ? a.free_counts : tid == 1 ? a.movable_counts : a.used_counts)[c] = sum;
  }
}

// A workgroup for four chunks: the ids of their free and movable pages, in the order of the moves.
__global__ __launch_bounds__(256) void compact_list_kernel(const CompactArgs a) {
  __shared__ int free_before[kChunksMost + 1], movable_before[kChunksMost + 1], part[4];
  sum_chunks(a.free_counts, a.chunks, free_before, part);
  sum_chunks(a.movable_counts, a.chunks, movable_before, part);
  const int c = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (c >= a.chunks) return;
  enumerate_chunk(a.free_marks, c, free_before[c], 0, a.max_moves, [&](int k, int page) { a.to[k] = page; });
  const int movable = movable_before[a.chunks];
  enumerate_chunk(a.movable_marks, c, movable_before[c], movable - a.max_moves, movable, [&](int k, int page) { a.from[movable - 1 - k] = page; });
}

__global__ __launch_bounds__(256) void compact_move_kernel(const CompactArgs a) {
  __shared__ int free_before[kChunksMost + 1], movable_before[kChunksMost + 1], used_before[kChunksMost + 1], part[4];
  sum_chunks(a.free_counts, a.chunks, free_before, part);
  sum_chunks(a.movable_counts, a.chunks, movable_before, part);
  sum_chunks(a.used_counts, a.chunks, used_before, part);
  const int k = blockIdx.x * 256 + threadIdx.x, refused = a.totals[0];
  const int most = refused ? 0 : min(a.max_moves, min(free_before[a.chunks], movable_before[a.chunks]));
  auto moves = [&](int j) { return j < most && a.to[j] < a.from[j]; };  // (true up to some j, false from there on)
  if (k == 0) {
    a.status[0] = 0;
    a.status[1] = refused;
    if (!moves(0)) a.status[2] = 0;
    a.status[3] = used_before[a.chunks];
  }
  if (k >= a.max_moves) return;
  const bool goes = moves(k);
  if (goes && !moves(k + 1)) a.status[2] = k + 1;
  a.moves[2 * (int64_t)k] = goes ? a.from[k] : -1;
  a.moves[2 * (int64_t)k + 1] = goes ? a.to[k] : -1;
  if (!goes) return;
  const int from = a.from[k], to = a.to[k];
  a.moved[from] = to;
  a.refs_out[to] = a.refs_out[from];
  a.refs_out[from] = 0;
}

__global__ __launch_bounds__(256) void compact_tables_kernel(const CompactArgs a) {
  const int r = blockIdx.x;
  if (r == 0 && threadIdx.x == 0) a.totals[0] = 0;
  const int held = pages_of(min(max(a.lens[r], 0), a.width * kPage));
  for (int e = threadIdx.x; e < a.width; e += 256) {
    const int64_t at = (int64_t)r * a.width + e;
    const int page = e < held ? a.src_tables[at] : -1;
    a.dst_tables[at] = page >= 0 && page < a.num_pages ? a.moved[page] : page;
  }
}

// ---- page contents ---------------------------------------------------------------------------------------------------------------

// A workgroup copies up to 16 KiB of one page of one pool of one layer.  Bound: HBM, 5.4 TB/s read and written (268 MB, 50 us).  The stores are
// non-temporal: what they would displace in the caches is worth more to the decode step behind than the pages themselves (copies of 26 MB,
// and with two layers of attention over 64 x 8 rows behind them that reads them: ordinary 19 and 303 us, so 7 and 289, the loads as well
// 10 and 289; of 105 MB and eight layers 40 and 1173, 26 and 1153, 40 and 1149).
constexpr int kCopyBytes = 16384;
__global__ __launch_bounds__(256) void pages_copy_kernel(uint8_t* k_pool, uint8_t* v_pool, int64_t layer_bytes, int64_t page_bytes,
                                                         int num_pages, const int32_t* __restrict__ pairs, int pieces) {
  const int i = blockIdx.x / pieces, piece = blockIdx.x - i * pieces;
  const int from = pairs[2 * (int64_t)i], to = pairs[2 * (int64_t)i + 1];
  if (from < 0 || from >= num_pages || to < 0 || to >= num_pages) return;
  uint8_t* const pool = ((blockIdx.y & 1) ? v_pool : k_pool) + (blockIdx.y >> 1) * layer_bytes;
  const int64_t begin = (int64_t)piece * kCopyBytes;
  const uint4* const src = reinterpret_cast<const uint4*>(pool + from * page_bytes + begin);
  uint4* const dst = reinterpret_cast<uint4*>(pool + to * page_bytes + begin);
  const int n = (int)(min((int64_t)kCopyBytes, page_bytes - begin) / 16);
  uint4 v[4];
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if ((int)threadIdx.x + 256 * j < n) v[j] = src[threadIdx.x + 256 * j];
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if ((int)threadIdx.x + 256 * j < n)
      __builtin_nontemporal_store(__builtin_bit_cast(i32x4, v[j]), reinterpret_cast<i32x4*>(dst) + threadIdx.x + 256 * j);
}

int fail_hip(hipError_t e, const char* what) {
  char buf[200];
  snprintf(buf, sizeof buf, "%s: %s", what, hipGetErrorString(e));
  return probe_fail(e == hipErrorOutOfMemory ? TDP_ENOMEM : TDP_EHIP, buf);
}

}  // namespace

hipError_t launch_kv_copy_pages(const KvLayout& kv, int64_t layer_bytes, int n_layers, const int32_t* pairs, int n, hipStream_t s) {
  if (n <= 0) return hipSuccess;
  const int64_t page_bytes = (int64_t)kv.n_kv_heads * kv.head_dim * 16 * (kv.fp8 ? 1 : 2);
  const int pieces = (int)((page_bytes + kCopyBytes - 1) / kCopyBytes);
  // (a launch counts its threads in 32 bits, and its layers in 16)
  const int64_t most = std::max<int64_t>(1, (1ll << 31) / 256 / (2 * std::min(n_layers, 1 << 14)) / pieces);
  for (int l = 0; l < n_layers; l += 1 << 14)
    for (int64_t first = 0; first < n; first += most) {
      const unsigned here = (unsigned)std::min<int64_t>(n - first, most);
      pages_copy_kernel<<<dim3(here * pieces, 2 * std::min(n_layers - l, 1 << 14)), 256, 0, s>>>(
          (uint8_t*)kv.k_pool + l * layer_bytes, (uint8_t*)kv.v_pool + l * layer_bytes, layer_bytes, page_bytes, kv.num_pages,
          pairs + 2 * first, pieces);
    }
  return hipGetLastError();
}

}  // namespace tdp

using namespace tdp;

struct tdp_pages {
  tdp_pages_config cfg;
  int device = 0, chunks = 0;
  u64* marks = nullptr;  // two bits for every page
  int* ints = nullptr;   // everything else
};

extern "C" {

int tdp_pages_create(const tdp_pages_config* cfg, tdp_pages** out) {
  if (!cfg || !out) return probe_fail(TDP_EINVAL, "null pointer");
  if (cfg->num_pages < 1 || cfg->num_pages > kChunk * kChunksMost) return probe_fail(TDP_EINVAL, "num_pages must be 1 .. 2^22");
  if (cfg->max_rows < 1 || cfg->max_rows > kRowsMost) return probe_fail(TDP_EINVAL, "max_rows must be 1 .. 8192");
  if (cfg->max_pages_per_seq < 1 || cfg->max_pages_per_seq > (1 << 16)) return probe_fail(TDP_EINVAL, "max_pages_per_seq must be 1 .. 2^16");
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess) return probe_fail(TDP_EHIP, "no HIP device");
  tdp_pages* h = new (std::nothrow) tdp_pages();
  if (!h) return probe_fail(TDP_ENOMEM, "host allocation failed");
  h->cfg = *cfg;
  h->device = dev;
  h->chunks = (cfg->num_pages + kChunk - 1) / kChunk;
  const size_t ints = ((size_t)3 * h->chunks + 3 + 3 * (size_t)cfg->max_rows + 4 * (size_t)cfg->num_pages) * sizeof(int);
  hipError_t e = hipMalloc((void**)&h->marks, (size_t)2 * h->chunks * kChunkWords * sizeof(u64));
  if (e == hipSuccess) e = hipMalloc((void**)&h->ints, ints);
  if (e == hipSuccess) e = hipMemset(h->ints, 0, ints);
  if (e == hipSuccess)
    e = hipFuncSetAttribute((const void*)pages_survey_kernel, hipFuncAttributeMaxDynamicSharedMemorySize, 2 * kRowsMost * (int)sizeof(int));
  if (e == hipSuccess) e = hipDeviceSynchronize();
  if (e != hipSuccess) {
    const int code = fail_hip(e, "tdp_pages_create");
    tdp_pages_destroy(h);
    return code;
  }
  *out = h;
  return TDP_OK;
}

void tdp_pages_destroy(tdp_pages* h) {
  if (!h) return;
  (void)hipDeviceSynchronize();
  if (h->marks) (void)hipFree(h->marks);
  if (h->ints) (void)hipFree(h->ints);
  delete h;
}

static int check_pages_device(const tdp_pages* h) {
  int dev = -1;
  const hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return fail_hip(e, "hipGetDevice");
  return dev == h->device ? TDP_OK : probe_fail(TDP_EINVAL, "the object was created on another device than the current one");
}

int tdp_pages_fork(tdp_pages* h, const int32_t* parents, const int32_t* src_tables, const int32_t* src_lens, int32_t n_src,
                   const int32_t* add, int32_t add_all, int32_t n_dst, const int32_t* refs_in, int32_t* refs_out, int32_t* dst_tables,
                   int32_t* dst_lens, int32_t* copies, int32_t* status, void* stream) {
  if (!h) return probe_fail(TDP_EINVAL, "null pages object");
  if (n_src < 0 || n_dst < 0) return probe_fail(TDP_EINVAL, "negative size");
  if (n_src > h->cfg.max_rows || n_dst > h->cfg.max_rows) return probe_fail(TDP_EINVAL, "rows exceed max_rows");
  if (!add && add_all < 0) return probe_fail(TDP_EINVAL, "add_all must be >= 0");
  if (!refs_in || !refs_out || !status) return probe_fail(TDP_EINVAL, "null pointer");
  if (n_src > 0 && (!src_tables || !src_lens)) return probe_fail(TDP_EINVAL, "null pointer");
  if (n_dst > 0 && (!dst_tables || !dst_lens || !copies)) return probe_fail(TDP_EINVAL, "null pointer");
  const int64_t W = h->cfg.max_pages_per_seq, N = h->cfg.num_pages;
  // (rows are made by workgroups of their own, which read what belongs to others)
  const Range in[] = {{parents, 4ll * n_dst}, {add, 4ll * n_dst}, {src_lens, 4ll * n_src}, {src_tables, 4 * W * n_src}, {refs_in == refs_out ? nullptr : refs_in, 4 * N}};
  const Range out[] = {{refs_out, 4 * N}, {dst_tables, 4 * W * n_dst}, {dst_lens, 4ll * n_dst}, {copies, 8ll * n_dst}, {status, 16}};
  if (any_meet(in, out)) return probe_fail(TDP_EINVAL, "outputs must not overlap inputs or one another (refs_out may be refs_in itself)");
  const int rc = check_pages_device(h);
  if (rc != TDP_OK) return rc;
  hipStream_t s = (hipStream_t)stream;
  int* const rows = h->ints + 3 * h->chunks + 3;
  const ForkArgs a{parents, src_tables, src_lens, add, n_src, add_all, n_dst, (int)W, (int)N, h->chunks, refs_in, refs_out, dst_tables, dst_lens,
                   copies, status, h->marks, h->ints, rows, rows + h->cfg.max_rows, rows + 2 * h->cfg.max_rows, h->ints + 3 * h->chunks};
  pages_survey_kernel<<<1 + h->chunks, 1024, 2 * (size_t)n_src * sizeof(int), s>>>(a);
  pages_fork_kernel<<<std::max(1, std::max(n_src, n_dst)), 256, 0, s>>>(a);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? TDP_OK : fail_hip(e, "tdp_pages_fork");
}

int tdp_pages_compact(tdp_pages* h, const int32_t* src_tables, const int32_t* lens, int32_t n_rows, int32_t max_moves, const int32_t* refs_in,
                      int32_t* refs_out, int32_t* dst_tables, int32_t* moves, int32_t* status, void* stream) {
  if (!h) return probe_fail(TDP_EINVAL, "null pages object");
  if (n_rows < 0) return probe_fail(TDP_EINVAL, "negative size");
  if (n_rows > h->cfg.max_rows) return probe_fail(TDP_EINVAL, "rows exceed max_rows");
  if (max_moves < 1 || max_moves > kChunk * kChunksMost) return probe_fail(TDP_EINVAL, "max_moves must be 1 .. 2^22");
  if (!refs_in || !refs_out || !moves || !status) return probe_fail(TDP_EINVAL, "null pointer");
  if (n_rows > 0 && (!src_tables || !lens || !dst_tables)) return probe_fail(TDP_EINVAL, "null pointer");
  const int64_t bytes = 4ll * h->cfg.max_pages_per_seq * n_rows, N = h->cfg.num_pages;
  const Range in[] = {{src_tables == dst_tables ? nullptr : src_tables, bytes}, {lens, 4ll * n_rows}, {refs_in == refs_out ? nullptr : refs_in, 4 * N}};
  const Range out[] = {{refs_out, 4 * N}, {dst_tables, bytes}, {moves, 8ll * max_moves}, {status, 16}};
  if (any_meet(in, out))
    return probe_fail(TDP_EINVAL, "outputs must not overlap inputs or one another (dst_tables may be src_tables itself, refs_out refs_in)");
  const int rc = check_pages_device(h);
  if (rc != TDP_OK) return rc;
  hipStream_t s = (hipStream_t)stream;
  int* const per_page = h->ints + 3 * h->chunks + 3 + 3 * h->cfg.max_rows;
  const CompactArgs a{src_tables, lens, n_rows, h->cfg.max_pages_per_seq, (int)N, h->chunks, max_moves, refs_in, refs_out, dst_tables, moves, status,
                      h->marks, h->marks + (int64_t)h->chunks * kChunkWords, h->ints, h->ints + h->chunks, h->ints + 2 * h->chunks,
                      per_page, per_page + N, per_page + 2 * N, per_page + 3 * N, h->ints + 3 * h->chunks + 2};
  if (n_rows > 0) compact_count_kernel<<<n_rows, 256, 0, s>>>(a);
  compact_survey_kernel<<<h->chunks, 1024, 0, s>>>(a);
  compact_list_kernel<<<(h->chunks + 3) / 4, 256, 0, s>>>(a);
  compact_move_kernel<<<(max_moves + 255) / 256, 256, 0, s>>>(a);
  if (n_rows > 0) compact_tables_kernel<<<n_rows, 256, 0, s>>>(a);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? TDP_OK : fail_hip(e, "tdp_pages_compact");
}

}  // extern "C"
