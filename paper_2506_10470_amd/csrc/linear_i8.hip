// The product in 8-bit integers with a scale for each token and each output channel (tdp_linear_i8_*): quantisation of rows and of
// weights, and the object that holds the weights.  The product itself is the GEMM of gemm.hip on integers.
//
//   y[m, n] = s_x[m] s_w[n] sum_k c_x[m, k] c_w[k, n],    v = s c + e with |e| <= s / 2 before rounding,  s = max |v| / 127
//
// (Rounded in fp32, c and s add 381 u s, u = 2^-24: v * (127 / a) is off by 2 u of up to 127, and s by u.)  The sum is exact, so all that
// is lost is lost in the codes; the scales are common to a sum and stand outside it.
#include <math.h>
#include <stdio.h>
#include <string.h>

#include <new>

#include "../../include/tdp.h"
#include "tdp_device.h"
#include "tdp_kernels.h"

namespace tdp {

int probe_fail(int code, const char* msg);  // sets the thread's error message (stage.hip)

// What quantises a vector whose largest magnitude has these bits (magnitudes order as their bits do, infinities and NaN behind all).
struct Quantiser {
  float scale, up, inverse;
  __device__ __forceinline__ Quantiser(unsigned largest) {
    const float a = __uint_as_float(largest);
    const bool finite = largest < 0x7f800000u;
    up = a < 0x1p-100f ? 0x1p100f : 1.0f;
    inverse = finite && a > 0.f ? 127.0f / (a * up) : 0.f;
    scale = finite ? a / 127.0f : NAN;
  }
  __device__ __forceinline__ int code(float v) const { return inverse == 0.f ? 0 : (int)rintf(v * up * inverse); }
};
__device__ __forceinline__ unsigned magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// One workgroup per row, a thread per 8 elements (of rows longer than 8192 up to 4); the row is read once and kept in registers between the
// maximum and the codes (what lies beyond 32768 elements is read again).
template <bool F32_IN, bool NORM>
__global__ __launch_bounds__(1024) void quantise_rows_kernel(const void* __restrict__ x, int64_t ldx, const float* __restrict__ gain,
                                                             float eps, int K, int chunks_padded, uint8_t* __restrict__ codes,
                                                             OperandLayout lay, float* __restrict__ scales) {
  const int row = blockIdx.x, tid = threadIdx.x, threads = blockDim.x;
  const int chunks = K / 8;
  float ss = 0.f;
  unsigned largest = 0;
  auto load = [&](int c, float (&f)[8]) {
    if constexpr (F32_IN) {
      const f32x4* p = reinterpret_cast<const f32x4*>((const float*)x + (int64_t)row * ldx + c * 8);
      const f32x4 a = p[0], b = p[1];
#pragma unroll
      for (int i = 0; i < 4; ++i) f[i] = a[i], f[i + 4] = b[i];
    } else {
      const bf16x8 a = ld_bf16x8((const bf16*)x + (int64_t)row * ldx + c * 8);
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = (float)a[i];
    }
  };
  auto see = [&](int c, float (&f)[8]) {
    if constexpr (NORM) {
      const f32x4 g0 = *reinterpret_cast<const f32x4*>(gain + c * 8), g1 = *reinterpret_cast<const f32x4*>(gain + c * 8 + 4);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        ss += f[i] * f[i];
        f[i] *= i < 4 ? g0[i] : g1[i - 4];
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) largest = max(largest, magnitude(f[i]));
  };
  constexpr int KEEP = 4;
  float keep[KEEP][8];
#pragma unroll
  for (int k = 0; k < KEEP; ++k)
    if (tid + threads * k < chunks) load(tid + threads * k, keep[k]);
#pragma unroll
  for (int k = 0; k < KEEP; ++k)
    if (tid + threads * k < chunks) see(tid + threads * k, keep[k]);
  for (int c = tid + threads * KEEP; c < chunks; c += threads) {
    float f[8];
    load(c, f);
    see(c, f);
  }
  __shared__ float red_ss[16];
  __shared__ unsigned red_max[16];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) largest = max(largest, (unsigned)__shfl_xor((int)largest, o, 64));
  if constexpr (NORM) ss = wave_sum(ss);
  if ((tid & 63) == 0) {
    red_max[tid >> 6] = largest;
    red_ss[tid >> 6] = ss;
  }
  __syncthreads();
  ss = 0.f;
  for (int w = 0; w < threads / 64; ++w) {
    largest = max(largest, red_max[w]);
    ss += red_ss[w];
  }
  const Quantiser q(largest);
  if (tid == 0) scales[row] = NORM ? q.scale * (1.0f / sqrtf(ss / (float)K + eps)) : q.scale;
  auto emit = [&](int c, const float (&f)[8]) {
    unsigned w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      w[h] = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) w[h] |= (unsigned)(q.code(f[4 * h + i]) & 255) << (8 * i);
    }
    *reinterpret_cast<uint2*>(codes + 2 * operand_offset(lay, row, c * 4)) = make_uint2(w[0], w[1]);
  };
#pragma unroll
  for (int k = 0; k < KEEP; ++k)
    if (tid + threads * k < chunks) emit(tid + threads * k, keep[k]);
  for (int c = tid + threads * KEEP; c < chunks; c += threads) {
    float f[8], unused = ss;
    const unsigned seen = largest;
    load(c, f);
    see(c, f);
    ss = unused;
    largest = seen;
    emit(c, f);
  }
  for (int c = chunks + tid; c < chunks_padded; c += threads)
    *reinterpret_cast<uint2*>(codes + 2 * operand_offset(lay, row, c * 4)) = make_uint2(0u, 0u);
}

hipError_t launch_quantise_rows(const void* x, int x_is_f32, int64_t ldx, const float* gain, float eps, int M, int K, int64_t Kpad,
                                void* codes, float* scales, hipStream_t s) {
  if (M <= 0) return hipSuccess;
  const int waves = (K / 8 + 63) / 64, threads = 64 * (waves < 16 ? waves : 16);
  const OperandLayout lay = layout_paired(Kpad / 2);
#define TDP_QUANTISE(F32_IN, NORM) \
  quantise_rows_kernel<F32_IN, NORM><<<M, threads, 0, s>>>(x, ldx, gain, eps, K, (int)(Kpad / 8), (uint8_t*)codes, lay, scales)
  if (gain) TDP_QUANTISE(false, true);
  else if (x_is_f32) TDP_QUANTISE(true, false);
  else TDP_QUANTISE(false, false);
#undef TDP_QUANTISE
  return hipGetLastError();
}

// A wave's share of K in the two kernels below: `length` of `all` steps, contiguous, gone through in a circle from `turn` on.  (Shares
// start as far apart as shares are long, and groups of weight rows 128 K bytes: where K is a power of two all waves of the chip would ask
// the same few channels in step.  One row of 8192 x 8192 15.4 us without the turn.)
struct Share {
  int first, length, turn;
  __device__ __forceinline__ Share(int all, int of, int which, int group) {
    const int per = (all + of - 1) / of;
    first = which * per;
    length = max(0, min(per, all - first));
    turn = length > 0 ? (which + group) % length : 0;
  }
  __device__ __forceinline__ int step(int i) const { return first + (i + turn >= length ? i + turn - length : i + turn); }
};

// ---- one row or two --------------------------------------------------------------------------------------------------------------
// For a row or two a tile of 32 rows, its ring to fill, its partials to sum and two or three launches cost more than the weights are to
// read.  One launch instead: every workgroup quantises the rows itself into LDS and streams weights through registers, the first of them
// on their way meanwhile.  A wave takes four weight rows, in 1 KiB loads of four rows x four k-blocks of 64 codes, eight of them at a
// time, and a lane multiplies its 16 codes with those of every row by v_dot4_i32_i8; the lanes of a weight row are added up at the end.
// Where there are too few weight rows for the chip the waves of a workgroup share K (slices). Taken where one round of workgroups holds
// all weight rows (up to 16384 columns).  Calls of a captured graph, back to back: one row of 256 x 256 3.5 us (tiles 5.9), 4096 x 4096 6.2
// (11.6), 5120 x 7168 9.5 (14.3), 8192 x 8192 14.1 (19.3), 28672 x 8192 43 (44: 5.4 TB/s); two rows 4.3, 8.2, 11.3, 15.6, 44.  (By itself
// the smallest takes 4 to 5 in a trace.)  With more weight rows the tiles' longer runs of memory win: 4096 x 32000 26.0 (24.4), 8192 x
// 57344 in several turns 93 (72).  With four rows a workgroup's own quantisation costs what is saved (4096 x 4096 12 and 11).
constexpr int kFewRows = 2, kFewWaves = 8, kFewInFlight = 8, kFewLds = 128 * 1024;
struct FewRowsParams : FewRowsArgs {
  int slices, groups, blocks_k;  // waves that share K; groups of four weight rows; k-blocks
};

template <int MM, bool F32_IN, bool NORM>
__global__ __launch_bounds__(64 * kFewWaves) void few_rows_kernel(const FewRowsParams p) {
  constexpr int THREADS = 64 * kFewWaves;
  extern __shared__ __attribute__((aligned(16))) unsigned char few_smem[];
  __shared__ unsigned red_max[MM][kFewWaves];
  __shared__ float red_ss[MM][kFewWaves];
  __shared__ float x_scale[MM];
  __shared__ int part[kFewWaves][MM][4];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int turns = (p.blocks_k + 3) / 4, k_lds = turns * 256;  // of 256 codes
  const int slice = wave % p.slices;
  const int group = blockIdx.x * (kFewWaves / p.slices) + wave / p.slices;
  const int rr = (lane >> 2) & 3, kb = lane >> 4, c16 = (lane & 3) * 16;
  // this lane's weight row (past the last group: the last one's, for nothing)
  const int last = min(group, p.groups - 1), pair = last * 2 + (rr & 1);
  const int r = p.gated ? (pair / 32) * 64 + pair % 32 + (rr >> 1) * 32 : last * 4 + rr;
  const Share share(turns, p.slices, slice, __builtin_amdgcn_readfirstlane(r >> kWeightGroupShift));  // (a wave's rows are of one group)
  const uint8_t* const row_base =
      (const uint8_t*)p.W + (int64_t)(r >> kWeightGroupShift) * (p.Kpad << kWeightGroupShift) + (r & ((1 << kWeightGroupShift) - 1)) * 64 + c16;
  i32x4 w[kFewInFlight];
  auto fetch = [&](int t) {  // (a k-block behind the last: any, its codes are zero)
    const int block = 4 * t + kb;
    const int64_t at = (int64_t)(block < p.blocks_k ? block : 0) << (6 + kWeightGroupShift);
    return __builtin_nontemporal_load(reinterpret_cast<const i32x4*>(row_base + at));
  };
  // the rows' largest magnitudes (and sums of squares), then their codes
  auto load8 = [&](int m, int c, float (&f)[8]) {
    if constexpr (F32_IN) {
      const f32x4* q = reinterpret_cast<const f32x4*>((const float*)p.x + (int64_t)m * p.ldx + c * 8);
      const f32x4 a = q[0], b = q[1];
#pragma unroll
      for (int i = 0; i < 4; ++i) f[i] = a[i], f[i + 4] = b[i];
    } else {
      const bf16x8 a = ld_bf16x8((const bf16*)p.x + (int64_t)m * p.ldx + c * 8);
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = (float)a[i];
    }
  };
  auto gained = [&](int c, float (&f)[8]) {
    if constexpr (NORM) {
      const f32x4 g0 = *reinterpret_cast<const f32x4*>(p.gain + c * 8), g1 = *reinterpret_cast<const f32x4*>(p.gain + c * 8 + 4);
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] *= i < 4 ? g0[i] : g1[i - 4];
    }
  };
  const int chunks = p.K / 8;
  constexpr int KEEP = 2;  // chunks of a row that a thread keeps between maximum and codes (8192 elements of a row in all)
  float keep[MM][KEEP][8], ss[MM];
  unsigned largest[MM];
  auto see = [&](int m, int c, float (&f)[8]) {
    if constexpr (NORM) {
#pragma unroll
      for (int i = 0; i < 8; ++i) ss[m] += f[i] * f[i];
      gained(c, f);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) largest[m] = max(largest[m], magnitude(f[i]));
  };
#pragma unroll
  for (int m = 0; m < MM; ++m) {
    largest[m] = 0;
    ss[m] = 0.f;
#pragma unroll
    for (int k = 0; k < KEEP; ++k)
      if (m < p.M && tid + k * THREADS < chunks) load8(m, tid + k * THREADS, keep[m][k]);
  }
#pragma unroll
  for (int m = 0; m < MM; ++m)
#pragma unroll 2
    for (int c = tid + KEEP * THREADS; m < p.M && c < chunks; c += THREADS) {
      float f[8];
      load8(m, c, f);
      see(m, c, f);
    }
  // (behind the loads of the rows: loads are waited for in order)
#pragma unroll
  for (int u = 0; u < kFewInFlight; ++u)
    if (u < share.length) w[u] = fetch(share.step(u));
#pragma unroll
  for (int m = 0; m < MM; ++m)
#pragma unroll
    for (int k = 0; k < KEEP; ++k)
      if (m < p.M && tid + k * THREADS < chunks) see(m, tid + k * THREADS, keep[m][k]);
#pragma unroll
  for (int m = 0; m < MM; ++m) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) largest[m] = max(largest[m], (unsigned)__shfl_xor((int)largest[m], o, 64));
    if constexpr (NORM) ss[m] = wave_sum(ss[m]);
    if (lane == 0) {
      red_max[m][wave] = largest[m];
      red_ss[m][wave] = ss[m];
    }
  }
  __syncthreads();
#pragma unroll
  for (int m = 0; m < MM; ++m) {
    unsigned all = 0;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < kFewWaves; ++i) {
      all = max(all, red_max[m][i]);
      sum += red_ss[m][i];
    }
    const Quantiser q(all);
    if (tid == 0) x_scale[m] = NORM ? q.scale * (1.0f / sqrtf(sum / (float)p.K + p.eps)) : q.scale;
    auto put = [&](int c, const float (&f)[8]) {
      unsigned o[2] = {0u, 0u};
#pragma unroll
      for (int i = 0; i < 8; ++i) o[i / 4] |= (unsigned)(q.code(f[i]) & 255) << (8 * (i % 4));
      *reinterpret_cast<uint2*>(few_smem + m * k_lds + c * 8) = make_uint2(o[0], o[1]);
    };
    if (m < p.M) {
#pragma unroll
      for (int k = 0; k < KEEP; ++k)
        if (tid + k * THREADS < chunks) put(tid + k * THREADS, keep[m][k]);
#pragma unroll 2
      for (int c = tid + KEEP * THREADS; c < chunks; c += THREADS) {
        float f[8];
        load8(m, c, f);
        gained(c, f);
        put(c, f);
      }
    }
    for (int c = (m < p.M ? chunks : 0) + tid; c < k_lds / 8; c += THREADS)
      *reinterpret_cast<uint2*>(few_smem + m * k_lds + c * 8) = make_uint2(0u, 0u);
  }
  __syncthreads();
  int acc[MM];
#pragma unroll
  for (int m = 0; m < MM; ++m) acc[m] = 0;
  const uint8_t* const code = few_smem + kb * 64 + c16;
#pragma unroll 1
  for (int i = 0; i < share.length; i += kFewInFlight) {
#pragma unroll
    for (int u = 0; u < kFewInFlight; ++u) {
      if (i + u >= share.length) break;
      const int t = share.step(i + u);
      const i32x4 v = w[u];
#pragma unroll
      for (int m = 0; m < MM; ++m) {
        const i32x4 a = *reinterpret_cast<const i32x4*>(code + m * k_lds + t * 256);
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[m] = __builtin_amdgcn_sdot4(v[j], a[j], acc[m], false);
      }
      if (i + u + kFewInFlight < share.length) w[u] = fetch(share.step(i + u + kFewInFlight));
    }
  }
#pragma unroll
  for (int m = 0; m < MM; ++m)
    for (int o : {1, 2, 16, 32}) acc[m] += __shfl_xor(acc[m], o, 64);
  if (p.slices > 1) {
    if ((lane & 51) == 0)
#pragma unroll
      for (int m = 0; m < MM; ++m) part[wave][m][rr] = acc[m];
    __syncthreads();
#pragma unroll
    for (int m = 0; m < MM; ++m) {
      acc[m] = 0;
      for (int i = 0; i < p.slices; ++i) acc[m] += part[wave - slice + i][m][rr];
    }
  }
  // lane (weight row rr, i of 16) writes row i of the result
  const int m = kb * 4 + (lane & 3);
  float v = (float)acc[0] * p.w_scale[r] * x_scale[0];
#pragma unroll
  for (int i = 1; i < MM; ++i) v = m == i ? (float)acc[i] * p.w_scale[r] * x_scale[i] : v;
  int col = r;
  if (p.gated) {
    const float up = __shfl_xor(v, 8, 64);
    v = silu_f(v) * up;
    col = pair;
  }
  if (group >= p.groups || slice != 0 || m >= p.M || (p.gated && rr >= 2)) return;
  if (p.bias) v += p.bias[r];
  if (p.residual) v += p.out_f32 ? ((const float*)p.residual)[(int64_t)m * p.ldr + col] : (float)((const bf16*)p.residual)[(int64_t)m * p.ldr + col];
  if (p.out_f32) ((float*)p.out)[(int64_t)m * p.ldo + col] = v;
  else ((bf16*)p.out)[(int64_t)m * p.ldo + col] = (bf16)v;
}

// by rows, and fp32 rows, bf16 rows, normed bf16 rows
#define TDP_FEW(MM) {few_rows_kernel<MM, true, false>, few_rows_kernel<MM, false, false>, few_rows_kernel<MM, false, true>}
static void (*const kFewKernels[kFewRows][3])(FewRowsParams) = {TDP_FEW(1), TDP_FEW(2)};
#undef TDP_FEW

hipError_t few_rows_setup() {
  hipError_t e = hipSuccess;
  for (const auto& rows : kFewKernels)
    for (const auto& kernel : rows)
      if (e == hipSuccess)
        e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, kFewLds);
  return e;
}

static int few_rows_lds(int M, int64_t Kpad) { return M * (int)((Kpad + 255) / 256 * 256); }
static int few_rows_places(int lds) { return lds <= 72 * 1024 ? 512 : 256; }  // workgroups that the chip holds at once
static int few_rows_groups(int gated, int cols) { return gated ? cols / 2 : cols / 4; }
bool few_rows_fit(int M, int64_t Kpad, int gated, int cols) {
  if (M < 1 || M > kFewRows) return false;
  const int lds = few_rows_lds(M, Kpad);
  return lds <= kFewLds && few_rows_groups(gated, cols) <= few_rows_places(lds) * kFewWaves;
}

hipError_t launch_few_rows(const FewRowsArgs& a, hipStream_t s) {
  FewRowsParams p;
  (FewRowsArgs&)p = a;
  p.blocks_k = (int)(a.Kpad / 64);
  p.groups = few_rows_groups(a.gated, a.cols);
  const int turns = (p.blocks_k + 3) / 4, lds = few_rows_lds(a.M, a.Kpad), places = few_rows_places(lds);
  // slices until the groups fill the chip, as long as a wave has a few loads
  p.slices = 1;
  while (p.slices < kFewWaves && p.groups * p.slices * 2 <= places * kFewWaves && turns >= 4 * p.slices) p.slices *= 2;
  const int blocks = (p.groups * p.slices + kFewWaves - 1) / kFewWaves;
  kFewKernels[a.M - 1][a.gain ? 2 : a.x_is_f32 ? 0 : 1]<<<blocks, 64 * kFewWaves, lds, s>>>(p);
  return hipGetLastError();
}

// ---- a small batch ---------------------------------------------------------------------------------------------------------------
// From rows that are quantised: a workgroup takes up to 64 of them and 16 or 32 weight rows, its eight waves an eighth of K each, and
// adds up in LDS what split-K workgroups would leave as partials for a kernel behind them.  Weights and codes go straight from memory to
// the registers of the MFMAs (a fragment of weights, 16 rows x 64 codes, is 1 KiB of memory in one piece; codes come from L2), six
// k-steps ahead. Taken where one round of workgroups holds all weight rows without leaving many CUs a share less, and where the codes
// that a CU reads again stay below 512 KB (352 from 17 rows on): 3 rows of 4096 x 4096 7.9 us (tiles 11.3), 16 of 5120 x 7168 11.6
// (15.5), 48 15.2 (16.9), 64 of 2048 x 2048 8.5 (11.2), 16 of 28672 x 8192 42 (46).  Beyond: 48 of 28672 x 8192 57 (49), 64 of 16384 x
// 1024 28 (20), 3 of 8192 x 10240, 320 workgroups, 25 (21).  More than 64 rows, in parts of 64, where 256 workgroups hold all: 128 of
// 4096 x 4096 13.3 (17.4), 200 of 2048 x 2048 9.3 (11.5), 512 of 256 x 256 5.7 (6.9); 384 workgroups 333 of 2048 x 2048 14.4 (11.8).
// Level where K is 8192 (3 to 64 rows of 8192 x 8192 0.96 to 1.03 of the tiles' rate: groups of weight rows begin 1 MB apart).
constexpr int kSomeRows = 64, kSomeWaves = 8;  // rows to a workgroup at most
struct SomeRowsParams {
  const uint8_t *x, *W;  // codes: x_layout = layout_paired(Kpad / 2), layout_weights(Kpad / 2)
  OperandLayout x_layout;
  const float *x_scale, *w_scale, *bias;
  const void* residual;
  void* out;
  int64_t Kpad, ldr, ldo;
  int M, cols, gated, out_f32, steps;  // steps: k-blocks of 64
};

// MT tiles of 16 rows, NT of 16 weight rows (gated: gate and up rows of the same 16 columns)
template <int MT, int NT>
__global__ __launch_bounds__(64 * kSomeWaves) void some_rows_kernel(const SomeRowsParams p) {
  constexpr int AHEAD = 6;
  constexpr int PITCH = NT * 16 + 4;  // (a row of sums in LDS: 16-byte pieces, neighbouring rows in other banks)
  __shared__ __attribute__((aligned(16))) int sums[kSomeWaves][MT * 16][PITCH];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, kq = lane >> 4;
  const int block = blockIdx.x, m0 = blockIdx.y * kSomeRows;
  auto weight_row = [&](int nt) {  // the first of tile nt
    if (!p.gated) return (block * NT + nt) * 16;
    const int j = block * 16;
    return (j / 32) * 64 + j % 32 + nt * 32;
  };
  const Share share(p.steps, kSomeWaves, wave, weight_row(0) >> kWeightGroupShift);
  const uint8_t *wp[NT], *xp[MT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int r = weight_row(nt) + l16;
    wp[nt] = p.W + (int64_t)(r >> kWeightGroupShift) * (p.Kpad << kWeightGroupShift) + (r & ((1 << kWeightGroupShift) - 1)) * 64 + kq * 16;
  }
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const int m = min(m0 + mt * 16 + l16, p.M - 1);
    xp[mt] = p.x + 2 * operand_offset(p.x_layout, m, kq * 8);
  }
  i32x4 w[AHEAD][NT], x[AHEAD][MT], acc[NT][MT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) acc[nt][mt] = i32x4{0, 0, 0, 0};
  auto fetch = [&](int u, int i) {
    const int t = share.step(i);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
      w[u][nt] = __builtin_nontemporal_load(reinterpret_cast<const i32x4*>(wp[nt] + ((int64_t)t << (6 + kWeightGroupShift))));
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) x[u][mt] = *reinterpret_cast<const i32x4*>(xp[mt] + (int64_t)t * 128);
  };
#pragma unroll
  for (int u = 0; u < AHEAD; ++u)
    if (u < share.length) fetch(u, u);
#pragma unroll 1
  for (int i = 0; i < share.length; i += AHEAD) {
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      if (i + u >= share.length) break;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) acc[nt][mt] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[u][nt], x[u][mt], acc[nt][mt], 0, 0, 0);
      if (i + u + AHEAD < share.length) fetch(u, i + u + AHEAD);
    }
  }
  // a lane holds weight rows kq * 4 .. + 3 of row l16
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) *reinterpret_cast<i32x4*>(&sums[wave][mt * 16 + l16][nt * 16 + kq * 4]) = acc[nt][mt];
  __syncthreads();
  const int quads = (p.gated ? 1 : NT) * 4, row = tid / quads, q = (tid - row * quads) * 4, m = m0 + row;  // (at most 512 quads)
  const int col = (p.gated ? block * 16 : block * NT * 16) + q;
  if (row >= MT * 16 || m >= p.M || col >= p.cols) return;
  auto sum_at = [&](int n) {
    i32x4 s = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < kSomeWaves; ++i) s += *reinterpret_cast<const i32x4*>(&sums[i][row][n]);
    const f32x4 scale = *reinterpret_cast<const f32x4*>(p.w_scale + weight_row(n >> 4) + (n & 15));
    f32x4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = (float)s[e] * scale[e] * p.x_scale[m];
    return v;
  };
  f32x4 v = sum_at(q);
  if (NT == 2 && p.gated) {
    const f32x4 up = sum_at(16 + q);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = silu_f(v[e]) * up[e];
  }
  if (p.bias) v += *reinterpret_cast<const f32x4*>(p.bias + col);
  if (p.out_f32) {
    if (p.residual) v += *reinterpret_cast<const f32x4*>((const float*)p.residual + (int64_t)m * p.ldr + col);
    *reinterpret_cast<f32x4*>((float*)p.out + (int64_t)m * p.ldo + col) = v;
  } else {
    bf16x4 o;
    if (p.residual) {
      const bf16x4 r = *reinterpret_cast<const bf16x4*>((const bf16*)p.residual + (int64_t)m * p.ldr + col);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += (float)r[e];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = (bf16)v[e];
    *reinterpret_cast<bf16x4*>((bf16*)p.out + (int64_t)m * p.ldo + col) = o;
  }
}

// 32 weight rows to a workgroup where that leaves three quarters of the chip's CUs one.
static int some_rows_parts(int M) { return (M + kSomeRows - 1) / kSomeRows; }
static bool some_rows_two(int M, int gated, int cols) { return gated || (int64_t)((cols + 31) / 32) * some_rows_parts(M) >= 192; }
static int some_rows_grid(int M, int gated, int cols) { return some_rows_two(M, gated, cols) && !gated ? (cols + 31) / 32 : (cols + 15) / 16; }
bool some_rows_fit(int M, int64_t Kpad, int gated, int cols) {
  if (M < 1) return false;
  const int parts = some_rows_parts(M), grid = some_rows_grid(M, gated, cols), tiles = parts > 1 ? 4 : (M + 15) / 16;
  const int64_t all = (int64_t)grid * parts;
  if (all > (parts > 1 ? 256 : 512) || (all > 256 && all < 360)) return false;
  const int64_t codes = (all + 255) / 256 * tiles * 16 * Kpad;  // of the rows, that a CU reads
  return codes <= (tiles == 1 ? 512 : 352) * 1024;
}

hipError_t launch_some_rows(const SomeRowsParams& p, hipStream_t s) {
  const bool two = some_rows_two(p.M, p.gated, p.cols);
  const dim3 grid(some_rows_grid(p.M, p.gated, p.cols), some_rows_parts(p.M));
#define TDP_SOME(MT)                                                      \
  (two ? some_rows_kernel<MT, 2><<<grid, 64 * kSomeWaves, 0, s>>>(p)      \
       : some_rows_kernel<MT, 1><<<grid, 64 * kSomeWaves, 0, s>>>(p))
  switch (p.M > kSomeRows ? 4 : (p.M + 15) / 16) {
    case 1: TDP_SOME(1); break;
    case 2: TDP_SOME(2); break;
    case 3: TDP_SOME(3); break;
    default: TDP_SOME(4); break;
  }
#undef TDP_SOME
  return hipGetLastError();
}

// ---- weights (once, when they are set) --------------------------------------------------------------------------------------------
__device__ __forceinline__ float weight_at(const void* src, int kind, int64_t i) {
  return kind == kWeightF32 ? ((const float*)src)[i] : (float)((const bf16*)src)[i];
}

// The bits of every column's largest magnitude: a workgroup takes 64 columns x 512 rows.
__global__ __launch_bounds__(256) void column_max_kernel(const void* __restrict__ src, int kind, int64_t K, int64_t N, int64_t ld,
                                                         unsigned* __restrict__ column_max) {
  const int64_t n = (int64_t)blockIdx.x * 64 + (threadIdx.x & 63);
  const int64_t k0 = (int64_t)blockIdx.y * 512 + (threadIdx.x >> 6), k1 = min(K, (int64_t)blockIdx.y * 512 + 512);
  if (n >= N) return;
  unsigned largest = 0;
  for (int64_t k = k0; k < k1; k += 4) largest = max(largest, magnitude(weight_at(src, kind, k * ld + n)));
  atomicMax(column_max + n, largest);
}

// 16 codes of a weight row per thread, neighbouring threads in neighbouring columns of the source.
__global__ __launch_bounds__(256) void pack_weights_kernel(const void* __restrict__ src, int kind, const float* __restrict__ src_scales,
                                                           int64_t K, int64_t N, int64_t ld, int mode, uint8_t* __restrict__ dst,
                                                           OperandLayout lay, float* __restrict__ scales,
                                                           const unsigned* __restrict__ column_max) {
  const int64_t n = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int c = blockIdx.y;  // codes [16 c, 16 c + 16)
  if (n >= N) return;
  const int64_t r = mode == 0 ? n : (n / 32) * 64 + n % 32 + (mode == 2 ? 32 : 0);
  const Quantiser q(kind == kWeightCodes ? 0u : column_max[n]);
  unsigned w[4] = {0u, 0u, 0u, 0u};
  for (int i = 0; i < 16; ++i) {
    const int64_t k = (int64_t)c * 16 + i;
    if (k >= K) break;
    const int code = kind == kWeightCodes ? ((const int8_t*)src)[k * ld + n] : q.code(weight_at(src, kind, k * ld + n));
    w[i / 4] |= (unsigned)(code & 255) << (8 * (i % 4));
  }
  *reinterpret_cast<uint4*>(dst + 2 * operand_offset(lay, (int)r, c * 8)) = make_uint4(w[0], w[1], w[2], w[3]);
  if (c == 0) scales[r] = kind == kWeightCodes ? src_scales[n] : q.scale;
}

hipError_t launch_quantise_weights(const void* src, int kind, const float* src_scales, int64_t K, int64_t N, int64_t ld, int mode,
                                   void* dst, int64_t Kpad, float* scales, unsigned* column_max, hipStream_t s) {
  if (kind != kWeightCodes) {
    hipError_t e = hipMemsetAsync(column_max, 0, (size_t)N * sizeof(unsigned), s);
    if (e != hipSuccess) return e;
    column_max_kernel<<<dim3((unsigned)((N + 63) / 64), (unsigned)((K + 511) / 512)), 256, 0, s>>>(src, kind, K, N, ld, column_max);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  pack_weights_kernel<<<dim3((unsigned)((N + 255) / 256), (unsigned)(Kpad / 16)), 256, 0, s>>>(
      src, kind, src_scales, K, N, ld, mode, (uint8_t*)dst, layout_weights(Kpad / 2), scales, column_max);
  return hipGetLastError();
}

}  // namespace tdp

using namespace tdp;

struct tdp_linear_i8 {
  tdp_linear_i8_config cfg;
  int device = 0;
  int64_t Kpad = 0, Npad = 0;
  uint8_t* w = nullptr;        // [Npad][Kpad] codes in layout_weights(Kpad / 2)
  float* w_scale = nullptr;    // [Npad]
  float* bias = nullptr;       // [Npad]
  bool has_bias = false;
  uint8_t* codes = nullptr;    // [max_rows ^ 2][Kpad] codes of the call's rows
  float* x_scale = nullptr;    // [max_rows]
  float* ws = nullptr;         // split-K partials, int32
  int64_t ws_elems = 0;
  unsigned* column_max = nullptr;
  GemmPlan form{0, 0, 0};      // tile 0: planned
};

namespace {

int fail_hip(hipError_t e, const char* what) {
  char buf[256];
  snprintf(buf, sizeof buf, "%s: %s", what, hipGetErrorString(e));
  (void)hipGetLastError();  // (reported here; the next launch is not to be taken for the one that failed)
  return probe_fail(e == hipErrorOutOfMemory ? TDP_ENOMEM : TDP_EHIP, buf);
}

int64_t round_up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

// The object's memory is on one device; calls launch on the current one.
int check_device(const tdp_linear_i8* h) {
  int dev = -1;
  const hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return fail_hip(e, "hipGetDevice");
  if (dev != h->device) return probe_fail(TDP_EINVAL, "the object was created on another device than the current one");
  return TDP_OK;
}

// `bytes` from src, host or device, as device memory: src itself, or a copy in *tmp.
int on_device(const void* src, int mem, size_t bytes, const void** dev, void** tmp) {
  *dev = src;
  *tmp = nullptr;
  if (mem == TDP_DEVICE) return TDP_OK;
  hipError_t e = hipMalloc(tmp, bytes);
  if (e == hipSuccess) e = hipMemcpy(*tmp, src, bytes, hipMemcpyHostToDevice);
  if (e != hipSuccess) {
    if (*tmp) (void)hipFree(*tmp);
    return fail_hip(e, "weight copy");
  }
  *dev = *tmp;
  return TDP_OK;
}

int set_weights(tdp_linear_i8* h, const void* src, int kind, const float* scales, int mem, int64_t rows, int64_t cols) {
  if (!h || !src || (kind == kWeightCodes && !scales)) return probe_fail(TDP_EINVAL, "null pointer");
  if (mem != TDP_HOST && mem != TDP_DEVICE) return probe_fail(TDP_EINVAL, "mem must be TDP_HOST or TDP_DEVICE");
  const int64_t K = h->cfg.in_features, N = h->cfg.out_features;
  if (rows != K || cols != N) return probe_fail(TDP_EINVAL, "weight shape does not match the configuration");
  int rc = check_device(h);
  if (rc != TDP_OK) return rc;
  hipError_t e = hipDeviceSynchronize();  // (a source may come from any stream, and calls on any may still read what is replaced)
  if (e != hipSuccess) return fail_hip(e, "weight quantisation");
  const size_t size = kind == kWeightF32 ? 4 : kind == kWeightBf16 ? 2 : 1;
  const void *w = nullptr, *ws = nullptr;
  void *tmp = nullptr, *tmp_scales = nullptr;
  if ((rc = on_device(src, mem, (size_t)(K * N) * size, &w, &tmp)) != TDP_OK) return rc;
  if (kind == kWeightCodes && (rc = on_device(scales, mem, (size_t)N * 4, &ws, &tmp_scales)) != TDP_OK) {
    if (tmp) (void)hipFree(tmp);
    return rc;
  }
  for (int half = 0; half < (h->cfg.gated ? 2 : 1) && e == hipSuccess; ++half) {
    const int64_t cols_here = h->cfg.gated ? N / 2 : N, at = half * cols_here;
    e = launch_quantise_weights((const uint8_t*)w + at * size, kind, ws ? (const float*)ws + at : nullptr, K, cols_here, N,
                                h->cfg.gated ? 1 + half : 0, h->w, h->Kpad, h->w_scale, h->column_max, 0);
  }
  if (e == hipSuccess) e = hipDeviceSynchronize();
  if (tmp) (void)hipFree(tmp);
  if (tmp_scales) (void)hipFree(tmp_scales);
  return e == hipSuccess ? TDP_OK : fail_hip(e, "weight quantisation");
}

}  // namespace

extern "C" {

int tdp_linear_i8_create(const tdp_linear_i8_config* cfg, tdp_linear_i8** out) {
  if (!cfg || !out) return probe_fail(TDP_EINVAL, "null pointer");
  if (cfg->in_features < 8 || cfg->in_features % 8 || cfg->in_features > 131072)
    return probe_fail(TDP_EINVAL, "in_features must be a multiple of 8, at most 131072");
  if (cfg->gated != 0 && cfg->gated != 1) return probe_fail(TDP_EINVAL, "gated must be 0 or 1");
  const int unit = cfg->gated ? 8 : 4;
  if (cfg->out_features < unit || cfg->out_features % unit || cfg->out_features > (1 << 24))
    return probe_fail(TDP_EINVAL, "out_features must be a multiple of 4 (gated: of 8), at most 2^24");
  if (cfg->max_rows < 1 || cfg->max_rows > (1 << 21)) return probe_fail(TDP_EINVAL, "max_rows must be 1 .. 2^21");
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess) return probe_fail(TDP_EHIP, "no HIP device");
  tdp_linear_i8* h = new (std::nothrow) tdp_linear_i8();
  if (!h) return probe_fail(TDP_ENOMEM, "host allocation failed");
  h->cfg = *cfg;
  h->device = dev;
  h->Kpad = round_up(cfg->in_features, 128);
  h->Npad = cfg->gated ? 2 * round_up(cfg->out_features / 2, 128) : round_up(cfg->out_features, 256);
  const int64_t M = ((int64_t)cfg->max_rows + 1) & ~1ll;
  h->ws_elems = 8 * (M < 512 ? M : 512) * h->Npad;
  if (h->ws_elems > (64ll << 20)) h->ws_elems = 64ll << 20;
  hipError_t e = gemm_setup();
  if (e == hipSuccess) e = few_rows_setup();
  auto alloc = [&](auto** p, int64_t n, bool zero) {
    const size_t bytes = (size_t)n * sizeof(**p);
    if (e == hipSuccess) e = hipMalloc((void**)p, bytes);
    if (e == hipSuccess && zero) e = hipMemset(*p, 0, bytes);
  };
  alloc(&h->w, h->Npad * h->Kpad, true);
  alloc(&h->w_scale, h->Npad, true);
  alloc(&h->bias, h->Npad, true);
  alloc(&h->codes, M * h->Kpad, true);
  alloc(&h->x_scale, M, false);
  alloc(&h->ws, h->ws_elems, false);
  alloc(&h->column_max, cfg->out_features, false);
  if (e == hipSuccess) e = hipDeviceSynchronize();
  if (e != hipSuccess) {
    const int code = fail_hip(e, "tdp_linear_i8_create");
    tdp_linear_i8_destroy(h);
    return code;
  }
  *out = h;
  return TDP_OK;
}

void tdp_linear_i8_destroy(tdp_linear_i8* h) {
  if (!h) return;
  (void)hipDeviceSynchronize();
  void* ptrs[] = {h->w, h->w_scale, h->bias, h->codes, h->x_scale, h->ws, h->column_max};
  for (void* p : ptrs)
    if (p) (void)hipFree(p);
  delete h;
}

int tdp_linear_i8_set_weight(tdp_linear_i8* h, const void* src, int32_t dtype, int32_t mem, int64_t rows, int64_t cols) {
  if (dtype != TDP_F32 && dtype != TDP_BF16) return probe_fail(TDP_EINVAL, "dtype must be TDP_F32 or TDP_BF16");
  return set_weights(h, src, dtype == TDP_F32 ? kWeightF32 : kWeightBf16, nullptr, mem, rows, cols);
}

int tdp_linear_i8_set_codes(tdp_linear_i8* h, const int8_t* codes, const float* scales, int32_t mem, int64_t rows, int64_t cols) {
  return set_weights(h, codes, kWeightCodes, scales, mem, rows, cols);
}

int tdp_linear_i8_set_bias(tdp_linear_i8* h, const void* src, int32_t dtype, int32_t mem, int64_t n) {
  if (!h || !src) return probe_fail(TDP_EINVAL, "null pointer");
  if (dtype != TDP_F32 && dtype != TDP_BF16) return probe_fail(TDP_EINVAL, "dtype must be TDP_F32 or TDP_BF16");
  if (mem != TDP_HOST && mem != TDP_DEVICE) return probe_fail(TDP_EINVAL, "mem must be TDP_HOST or TDP_DEVICE");
  if (h->cfg.gated) return probe_fail(TDP_EINVAL, "a gated product has no bias");
  if (n != h->cfg.out_features) return probe_fail(TDP_EINVAL, "bias length does not match the configuration");
  int rc = check_device(h);
  if (rc != TDP_OK) return rc;
  hipError_t e = hipDeviceSynchronize();  // (as in set_weights)
  if (e != hipSuccess) return fail_hip(e, "bias conversion");
  const void* dev = nullptr;
  void* tmp = nullptr;
  if ((rc = on_device(src, mem, (size_t)n * (dtype == TDP_F32 ? 4 : 2), &dev, &tmp)) != TDP_OK) return rc;
  e = launch_convert_vec(dev, dtype == TDP_F32, n, h->bias, 0);
  if (e == hipSuccess) e = hipDeviceSynchronize();
  if (tmp) (void)hipFree(tmp);
  if (e != hipSuccess) return fail_hip(e, "bias conversion");
  h->has_bias = true;
  return TDP_OK;
}

int tdp_linear_i8_set_form(tdp_linear_i8* h, int32_t tile, int32_t splits) {
  if (!h) return probe_fail(TDP_EINVAL, "null linear object");
  if (tile == 0) {
    h->form = GemmPlan{0, 0, 0};
    return TDP_OK;
  }
  const GemmPlan form{tile, splits, 0};
  if (!gemm_form_fits_integers(form, 1, h->Npad, h->Kpad / 2, h->ws_elems)) return probe_fail(TDP_EINVAL, "no such form of this product");
  h->form = form;
  return TDP_OK;
}

int tdp_linear_i8_run(tdp_linear_i8* h, const void* x, int32_t x_dtype, int64_t ld_x, int32_t M, const void* residual, int64_t ld_residual,
                      void* out, int32_t out_dtype, int64_t ld_out, void* stream) {
  if (!h) return probe_fail(TDP_EINVAL, "null linear object");
  if (M < 0) return probe_fail(TDP_EINVAL, "negative size");
  if (M > h->cfg.max_rows) return probe_fail(TDP_EINVAL, "M exceeds max_rows");
  if ((x_dtype != TDP_F32 && x_dtype != TDP_BF16) || (out_dtype != TDP_F32 && out_dtype != TDP_BF16))
    return probe_fail(TDP_EINVAL, "dtypes must be TDP_F32 or TDP_BF16");
  if (M == 0) return TDP_OK;
  if (!x || !out) return probe_fail(TDP_EINVAL, "null pointer");
  if (residual && h->cfg.gated) return probe_fail(TDP_EINVAL, "a gated product has no residual");
  const int K = h->cfg.in_features, cols = h->cfg.gated ? h->cfg.out_features / 2 : h->cfg.out_features;
  const int x_size = x_dtype == TDP_F32 ? 4 : 2, out_size = out_dtype == TDP_F32 ? 4 : 2;
  if (ld_x < K || ld_x * x_size % 16 || ((uintptr_t)x & 15)) return probe_fail(TDP_EINVAL, "rows of x must be 16-byte aligned and hold in_features");
  auto aligned = [&](const void* p, int64_t ld) { return ld >= cols && ld % 4 == 0 && ((uintptr_t)p & (4 * out_size - 1)) == 0; };
  if (!aligned(out, ld_out)) return probe_fail(TDP_EINVAL, "rows of out must be aligned to four elements and hold the result");
  if (residual && !aligned(residual, ld_residual))
    return probe_fail(TDP_EINVAL, "rows of residual must be aligned to four elements and hold the result");
  if (h->form.tile && !gemm_form_fits_integers(h->form, M, h->Npad, h->Kpad / 2, h->ws_elems))
    return probe_fail(TDP_EINVAL, "the partials of this form exceed the workspace");
  int rc = check_device(h);
  if (rc != TDP_OK) return rc;
  hipStream_t s = (hipStream_t)stream;
  hipError_t e = hipSuccess;
  if (!h->form.tile && few_rows_fit(M, h->Kpad, h->cfg.gated, cols)) {
    e = launch_few_rows({x, x_dtype == TDP_F32, ld_x, nullptr, 0.f, M, K, h->Kpad, h->w, h->w_scale, h->has_bias ? h->bias : nullptr,
                         h->cfg.gated, cols, residual, ld_residual, out, out_dtype == TDP_F32, ld_out}, s);
    return e == hipSuccess ? TDP_OK : fail_hip(e, "tdp_linear_i8_run");
  }
  e = launch_quantise_rows(x, x_dtype == TDP_F32, ld_x, nullptr, 0.f, M, K, h->Kpad, h->codes, h->x_scale, s);
  if (e == hipSuccess && !h->form.tile && some_rows_fit(M, h->Kpad, h->cfg.gated, cols)) {
    e = launch_some_rows({h->codes, h->w, layout_paired(h->Kpad / 2), h->x_scale, h->w_scale, h->has_bias ? h->bias : nullptr, residual,
                          out, h->Kpad, ld_residual, ld_out, M, cols, h->cfg.gated, out_dtype == TDP_F32, (int)(h->Kpad / 64)}, s);
  } else if (e == hipSuccess) {
    GemmArgs g;
    memset(&g, 0, sizeof(g));
    g.A = h->codes; g.a_layout = layout_paired(h->Kpad / 2); g.a_scale = h->x_scale;
    g.W = h->w; g.w_scale = h->w_scale; g.Kpad = h->Kpad / 2; g.Npad = h->Npad;
    g.M = M; g.N_store = cols; g.out = out; g.ldo = ld_out; g.out_f32 = out_dtype == TDP_F32;
    g.bias = h->has_bias ? h->bias : nullptr;
    g.residual = residual; g.ldr = ld_residual; g.residual_f32 = g.out_f32;
    g.epilogue = h->cfg.gated ? EPI_SWIGLU : residual ? EPI_RESIDUAL : EPI_STORE;
    g.workspace = h->ws; g.workspace_elems = h->ws_elems; g.form = h->form;
    try {
      e = launch_gemm(g, s);
    } catch (...) {  // (the plan is remembered)
      return probe_fail(TDP_ENOMEM, "host allocation failed");
    }
  }
  return e == hipSuccess ? TDP_OK : fail_hip(e, "tdp_linear_i8_run");
}

}  // extern "C"
