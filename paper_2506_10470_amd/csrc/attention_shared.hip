// Decode attention of rows that share a prefix (beams of a prompt, requests behind one system prompt): the keys and values of the pages on
// which the block tables of a group agree are read once for all (query head, row) pairs of the group, its columns.
//
// What is shared is found in the tables, not told: a group is rows that may share something, and its prefix is the leading pages that are the
// same in all of them, whole pages in front of every row's last token.  So the answer is that of ordinary decode attention whatever
// the groups are.  Partials (reference m, sum l, unnormalised output o, per span of the prefix) go to the first slots of every row
// and head; the decode kernel behind attends to what a row has of its own and combines all.
#include "tdp_device.h"
#include "tdp_kernels.h"

namespace tdp {
namespace {

// Columns of a workgroup's tile: 128, or 64 or 32 where groups are small (two or four waves then share a block's tokens out).
int tile_columns(int batch, int n_groups, int G) {
  const int64_t average = ((int64_t)batch * G + n_groups - 1) / n_groups;
  return average <= 32 ? 32 : average <= 64 ? 64 : 128;
}
// Spans wanted of one K/V head: the launch then has two to four workgroups for every one that the chip holds at once.
int spans_wanted(int n_kv_heads) { return (1024 + n_kv_heads - 1) / n_kv_heads; }

constexpr int kMinSpanPages = kDecodeSpanMin / 16;

// ---- plan ------------------------------------------------------------------------------------------------------------------------

// One workgroup per group: the pages that all its rows begin with.  Rows of length zero attend to nothing and do not count: what
// their tables hold is not looked at, and the group's pages are those of its first row with tokens (group_first).
__global__ __launch_bounds__(1024) void shared_prefix_kernel(const int32_t* __restrict__ group_starts, const int32_t* __restrict__ lens,
                                                             const int32_t* __restrict__ block_tables, int max_pages_per_seq, int batch,
                                                             const SharedRows rows, int32_t* __restrict__ row_pages,
                                                             int32_t* __restrict__ group_pages, int32_t* __restrict__ group_first) {
  __shared__ int most, longest, first, last;
  const int g = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int begin = min(max(group_starts[g], 0), batch), end = min(max(group_starts[g + 1], begin), batch);
  if (tid == 0) {
    most = 0x7fffffff;
    longest = 0;
    first = end;
    last = begin;
  }
  __syncthreads();
  for (int r = begin + tid; r < end; r += 1024) {
    const int n = rows.tokens(lens[r], max_pages_per_seq);
    if (n > 0) {
      atomicMin(&most, (n - 1) >> 4);
      atomicMax(&longest, n);
      atomicMin(&first, r);
      atomicMax(&last, r);
    }
  }
  __syncthreads();
  // the first difference between any row and the first of them; a wave compares four rows' 256 entries at a time
  const int limit = most, r0 = first, others = last - r0;  // (0: one row with tokens, or none)
  __syncthreads();
  if (others < 1) {
    if (tid == 0) most = 0;
  } else {
    constexpr int ROWS = 4, PART = 4;
    const int chunks = (limit + 64 * PART - 1) / (64 * PART), fours = (others + ROWS - 1) / ROWS;
    const int32_t* const base = block_tables + (int64_t)r0 * max_pages_per_seq;
    for (int i = wave; i < fours * chunks; i += 16) {
      const int c = i / fours, r = r0 + 1 + (i - c * fours) * ROWS;  // (low pages first)
      const int at = c * 64 * PART + lane;
      if (c * 64 * PART >= *(volatile int*)&most) break;
      int want[PART], got[ROWS][PART];
      bool in[ROWS];
#pragma unroll
      for (int u = 0; u < PART; ++u) want[u] = base[min(at + u * 64, limit - 1)];
#pragma unroll
      for (int j = 0; j < ROWS; ++j) {
        const int row = min(r + j, r0 + others);
        in[j] = rows.tokens(lens[row], max_pages_per_seq) > 0;
#pragma unroll
        for (int u = 0; u < PART; ++u) got[j][u] = block_tables[(int64_t)row * max_pages_per_seq + min(at + u * 64, limit - 1)];
      }
      int differs = 0x7fffffff;
#pragma unroll
      for (int u = PART - 1; u >= 0; --u)
#pragma unroll
        for (int j = 0; j < ROWS; ++j)
          if (in[j] && got[j][u] != want[u]) differs = min(at + u * 64, limit - 1);
      if (differs < limit) atomicMin(&most, differs);
    }
  }
  __syncthreads();
  // A short prefix is left to the rows where one of them has more than the shortest span behind it: there is little to save, and a row has
  // no more slots for partials than spans of that length.
  const int found = most;
  const int pages = found < kMinSpanPages && longest - found * 16 > kDecodeSpanMin ? 0 : found;
  for (int r = begin + tid; r < end; r += 1024) row_pages[r] = pages;
  if (tid == 0) {
    group_pages[g] = pages;
    group_first[g] = r0;
  }
}

// The work list of the prefix kernel: an item is a span of a group's prefix and a tile of its columns, two records
//   (first row, first column, columns of the group, span), (first page, pages, row whose table names them, 0),
// and (-1, ...) behind the last.  Spans are as long as the number wanted allows, and all of a group equally long.
__global__ __launch_bounds__(1024) void shared_list_kernel(const int32_t* __restrict__ group_starts, int n_groups, int batch, int G, int columns,
                                                           int wanted, const int32_t* __restrict__ group_pages, const int32_t* __restrict__ group_first,
                                                           int32_t* __restrict__ span_pages, int4* __restrict__ items, int max_items) {
  __shared__ long long work;
  __shared__ int part[16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  auto tiles_of = [&](int g) {
    const int begin = min(max(group_starts[g], 0), batch), end = min(max(group_starts[g + 1], begin), batch);
    return ((end - begin) * G + columns - 1) / columns;
  };
  if (tid == 0) work = 0;
  __syncthreads();
  for (int g = tid; g < n_groups; g += 1024)
    atomicAdd((unsigned long long*)&work, (unsigned long long)tiles_of(g) * (unsigned long long)group_pages[g]);
  __syncthreads();
  const int span = (int)max((long long)kMinSpanPages, (work + wanted - 1) / wanted);
  if (tid == 0) *span_pages = span;
  int base = 0;
  for (int g0 = 0; g0 < n_groups; g0 += 1024) {
    const int g = g0 + tid, pages = g < n_groups ? group_pages[g] : 0;
    const int spans = pages > 0 ? max(1, pages / span) : 0, tiles = spans ? tiles_of(g) : 0, own = spans * tiles;
    int at = own;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
      const int up = __shfl_up(at, o, 64);
      if (lane >= o) at += up;
    }
    __syncthreads();
    if (lane == 63) part[wave] = at;
    __syncthreads();
    int all = 0;
    at += base - own;
    for (int w = 0; w < 16; ++w) {
      at += w < wave ? part[w] : 0;
      all += part[w];
    }
    const int row = own ? min(max(group_starts[g], 0), batch) : 0, end = own ? min(max(group_starts[g + 1], row), batch) : 0;
    for (int i = 0; i < own && at + i < max_items; ++i) {
      const int s = i / tiles, first = (int)((int64_t)s * pages / spans);
      items[2 * (at + i)] = make_int4(row, (i - s * tiles) * columns, (end - row) * G, s);
      items[2 * (at + i) + 1] = make_int4(first, (int)((int64_t)(s + 1) * pages / spans) - first, group_first[g], 0);
    }
    base += all;
  }
  for (int i = base + tid; i < max_items; i += 1024) items[2 * i] = make_int4(-1, 0, 0, 0);
}

// ---- attention to the prefix -----------------------------------------------------------------------------------------------------

// One workgroup of four waves per (item, K/V head).  NWC waves have 32 columns each, and 4 / NWC waves share the tokens of a block out for
// the same columns.  A block of 64 tokens (128 for one wave of columns) of K and V^T is staged in LDS, double buffered and swizzled,
// and feeds the 32x32x16 MFMAs of all columns; scores are formed transposed, with their rows permuted so that a lane's elements are the
// consecutive tokens that it supplies to O^T += V^T P^T, as in the prefill kernel, whose masks are not needed here: a prefix is whole pages.
// Bound: reading the pages up to about a hundred columns, MFMA beyond.
template <int DH, int NWC, bool KV8>
__global__ __launch_bounds__(256, NWC == 1 ? 1 : 2) void attn_prefix_kernel(const bf16* __restrict__ q, int64_t ld, int n_q_heads, KvLayout kv,
                                                                            const int4* __restrict__ items,
                                                                            const int32_t* __restrict__ block_tables, int max_pages_per_seq,
                                                                            float* __restrict__ part_o, float* __restrict__ part_ml,
                                                                            int max_spans, float scale_log2) {
  constexpr int NWT = 4 / NWC;               // waves that share the tokens out
  constexpr int NH = NWC == 1 ? 4 : 2;       // 32-token halves of a block
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
  const int4 it = items[2 * item];
  if (it.x < 0) return;
  const int4 it2 = items[2 * item + 1];
  const int first_page = it2.x, n_pages = it2.y, n_tokens = n_pages * 16;
  const int32_t* const table = block_tables + (int64_t)it2.z * max_pages_per_seq + first_page;
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, kg = lane >> 5;
  const int wc = w % NWC, wt = w / NWC;

  // the lane's column; columns behind the last are computed as the last one and never stored
  const int col = it.y + wc * 32 + l32;
  const bool real = col < it.z;
  const int c = min(col, it.z - 1), row = it.x + c / G, head = kvh * G + c % G;
  const bool idle = it.y + wc * 32 >= it.z;  // (the whole wave)
  bf16x8 qf[KS];
  {
    const bf16* qp = q + (int64_t)row * ld + (int64_t)head * DH + kg * 8;
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
  constexpr int KP = KV8 ? NCH : NPG / 4, VP = KV8 ? NCH : 1;
  const int v_row = lane >> 2, v_chunk = (lane & 3) ^ ((v_row >> 2) & 3);
  int k_page[KP], v_page[VP];  // those that this thread asks for something of
  auto look_up = [&](int b) {
    auto id = [&](int i) { return table[min(b * NPG + i, n_pages - 1)]; };
    if constexpr (KV8) {
#pragma unroll
      for (int j = 0; j < NCH; ++j) {
        k_page[j] = id((tid + 256 * j) / (16 * CR));
        v_page[j] = id(256 * j / (DH * 4) * 2 + ((tid & 3) >> 1));
      }
    } else {
#pragma unroll
      for (int p = 0; p < KP; ++p) k_page[p] = id(w * KP + p);
      v_page[0] = id(w / WPH * 2 + (v_chunk >> 1));
    }
  };
  uint2 kraw[KV8 ? NCH : 1], vraw[KV8 ? NCH : 1];
  const unsigned k_lds = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char*)sK;
  const unsigned v_lds = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char*)sV;
  auto request = [&](unsigned lds_addr, const bf16* from) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds_addr), "v"(from) : "memory");
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
        kraw[j] = *reinterpret_cast<const uint2*>((const uint8_t*)kv.k_pool + ((int64_t)k_page[j] * Hkv + kvh) * HEAD + (kpiece * 16 + kt16) * 64 + kq * 8);
        vraw[j] = *reinterpret_cast<const uint2*>((const uint8_t*)kv.v_pool + (((int64_t)v_page[j] * Hkv + kvh) * DH + vr) * 16 + (vc & 1) * 8);
      }
    } else {
#pragma unroll
      for (int p = 0; p < KP; ++p) {
        const int pg = w * KP + p;  // of the block
        const bf16* kp = (const bf16*)kv.k_pool + ((int64_t)k_page[p] * Hkv + kvh) * HEAD;
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          const int slot = j * TPI + lane / CR, ktok = (pg & 1) * 16 + slot, kc = (lane % CR) ^ ((ktok / RWK) % CR);
          request(k_lds + ((buf * NH + (pg >> 1)) * HALF + ((pg & 1) * 16 + j * TPI) * DH) * 2, kp + (kc / 4) * 512 + slot * 32 + kc % 4 * 8);
        }
      }
      const int half = w / WPH, part = w % WPH;
      const bf16* vp = (const bf16*)kv.v_pool + ((int64_t)v_page[0] * Hkv + kvh) * HEAD + (part * (DH / WPH) + v_row) * 16 + (v_chunk & 1) * 8;
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
      bf16x8 vf[DT][2];  // on their way during the softmax
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int st = 0; st < 2; ++st) {
          const int r = d * 32 + l32;
          vf[d][st] = ld_bf16x8(vh + r * 32 + (((st * 2 + kg) ^ ((r >> 2) & 3)) << 3));
        }
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
        for (int st = 0; st < 2; ++st) o[d] = mfma32(vf[d][st], pb[st], o[d]);
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
  if (!real) return;
  const int64_t slot = ((int64_t)row * n_q_heads + head) * max_spans + it.w;
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *reinterpret_cast<f32x4*>(part_o + slot * DH + d * 32 + g * 8 + kg * 4) =
          f32x4{o[d][g * 4], o[d][g * 4 + 1], o[d][g * 4 + 2], o[d][g * 4 + 3]};
  if (kg == 0) *reinterpret_cast<float2*>(part_ml + slot * 2) = make_float2(m, lsum);
}

}  // namespace

int attn_prefix_items(int batch, int n_groups, int n_q_heads, int n_kv_heads) {
  const int G = n_q_heads / n_kv_heads;
  return (int)(((int64_t)batch * G) / tile_columns(batch, n_groups, G)) + n_groups + spans_wanted(n_kv_heads);
}
int attn_prefix_items_most(int max_batch, int n_q_heads, int n_kv_heads) {
  return max_batch * (n_q_heads / n_kv_heads) / 32 + max_batch + spans_wanted(n_kv_heads);
}

hipError_t launch_attn_shared_plan(const int32_t* group_starts, int n_groups, const int32_t* lens, int add, const int32_t* block_tables,
                                   int max_pages_per_seq, int batch, int n_q_heads, int n_kv_heads, const SharedScratch& sc, hipStream_t s) {
  const SharedRows rows{sc.row_pages, sc.span_pages, add};
  const int G = n_q_heads / n_kv_heads;
  shared_prefix_kernel<<<n_groups, 1024, 0, s>>>(group_starts, lens, block_tables, max_pages_per_seq, batch, rows, sc.row_pages, sc.group_pages,
                                             sc.group_first);
  shared_list_kernel<<<1, 1024, 0, s>>>(group_starts, n_groups, batch, G, tile_columns(batch, n_groups, G), spans_wanted(n_kv_heads), sc.group_pages,
                                        sc.group_first, sc.span_pages, sc.items, attn_prefix_items(batch, n_groups, n_q_heads, n_kv_heads));
  return hipGetLastError();
}

hipError_t launch_attn_prefix(const void* q, int64_t ld, int batch, int n_groups, int n_q_heads, const KvLayout& kv, const SharedScratch& sc,
                              const int32_t* block_tables, int max_pages_per_seq, float* part_o, float* part_ml, int max_spans,
                              hipStream_t s) {
  // 8-bit pools hold value / scale: the key scale joins the softmax scale, the value scale the final division, behind the partials
  const float scale_log2 = 1.4426950408889634f / sqrtf((float)kv.head_dim) * (kv.fp8 ? kv.k_scale : 1.0f);
  const unsigned grid = (unsigned)attn_prefix_items(batch, n_groups, n_q_heads, kv.n_kv_heads) * kv.n_kv_heads;
  const int columns = tile_columns(batch, n_groups, n_q_heads / kv.n_kv_heads);
#define TDP_PREFIX_(DH, NWC, KV8)                                                                                                   \
  attn_prefix_kernel<DH, NWC, KV8><<<grid, 256, 0, s>>>((const bf16*)q, ld, n_q_heads, kv, sc.items, block_tables, max_pages_per_seq, \
                                                        part_o, part_ml, max_spans, scale_log2)
#define TDP_PREFIX(DH, KV8)                          \
  do {                                               \
    if (columns == 32) TDP_PREFIX_(DH, 1, KV8);      \
    else if (columns == 64) TDP_PREFIX_(DH, 2, KV8); \
    else TDP_PREFIX_(DH, 4, KV8);                    \
  } while (0)
  if (kv.head_dim == 128) {
    if (kv.fp8) TDP_PREFIX(128, true); else TDP_PREFIX(128, false);
  } else {
    if (kv.fp8) TDP_PREFIX(64, true); else TDP_PREFIX(64, false);
  }
#undef TDP_PREFIX
#undef TDP_PREFIX_
  return hipGetLastError();
}

}  // namespace tdp
