// The product in 8-bit integers with a scale for each token and each output channel (tdp_linear_i8_*): quantisation of rows and of
// weights, and the object that holds the weights.  The product itself is the GEMM of gemm.hip on integers.
//
//   y[m, n] = s_x[m] s_w[n] sum_k c_x[m, k] c_w[k, n],    v = s c + e with |e| <= s / 2,  s = max |v| / 127
//
// The sum is exact, so all that is lost is lost in the codes; the scales are common to a sum and stand outside it.
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
  if (gain) {
    if (x_is_f32) TDP_QUANTISE(true, true);
    else TDP_QUANTISE(false, true);
  } else {
    if (x_is_f32) TDP_QUANTISE(true, false);
    else TDP_QUANTISE(false, false);
  }
#undef TDP_QUANTISE
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
  const size_t size = kind == kWeightF32 ? 4 : kind == kWeightBf16 ? 2 : 1;
  const void *w = nullptr, *ws = nullptr;
  void *tmp = nullptr, *tmp_scales = nullptr;
  if ((rc = on_device(src, mem, (size_t)(K * N) * size, &w, &tmp)) != TDP_OK) return rc;
  if (kind == kWeightCodes && (rc = on_device(scales, mem, (size_t)N * 4, &ws, &tmp_scales)) != TDP_OK) {
    if (tmp) (void)hipFree(tmp);
    return rc;
  }
  hipError_t e = hipSuccess;
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
  if (cfg->max_rows < 1 || cfg->max_rows > (1 << 24)) return probe_fail(TDP_EINVAL, "max_rows must be 1 .. 2^24");
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
  const void* dev = nullptr;
  void* tmp = nullptr;
  if ((rc = on_device(src, mem, (size_t)n * (dtype == TDP_F32 ? 4 : 2), &dev, &tmp)) != TDP_OK) return rc;
  hipError_t e = launch_convert_vec(dev, dtype == TDP_F32, n, h->bias, 0);
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
  hipError_t e = launch_quantise_rows(x, x_dtype == TDP_F32, ld_x, nullptr, 0.f, M, K, h->Kpad, h->codes, h->x_scale, s);
  if (e == hipSuccess) {
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
