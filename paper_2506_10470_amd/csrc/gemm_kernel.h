// The GEMM kernel and its epilogues, as templates (see gemm.hip for the product they make and for the choice among them).
#pragma once
#include <math.h>

#include <type_traits>

#include "tdp_device.h"
#include "tdp_kernels.h"

namespace tdp {

struct GemmParams {
  static constexpr bool kIntegers = false, kStatistics = false;
  const bf16* A;
  const bf16* W;
  bf16* out;
  const void* residual;  // bf16, or fp32 when res_f32
  const float* bias;     // fp32 [Npad] or null
  float* ws;
  OperandLayout a_lay, w_lay, u_lay;
  int64_t Kpad, Npad, ldo, ldr;
  int M, N_store, epilogue, out_f32, res_f32;
  int k_tiles_total, k_tiles_per_split, splits;
  int k_tiles_per_chunk;  // 0, or (splits = 1, small tiles) the K range is summed in chunks of this many k-tiles
  int tiles_m, tiles_n;
  // order of the tiles, see gemm_tile_of_block: bands of band_h + 1 (the first n_tall) or band_h rows of tiles; an
  // XCD takes `chunks` runs of `chunk` tiles, and an eighth of the `rest` tiles behind them
  int band_h, n_tall, chunk_shift, chunks, rest;
  unsigned per_split_inv, tall_inv, low_inv, h_tall_inv, h_low_inv;  // see divide
};
// What the two epilogues that only one projection has need on top.  Their kernels are instances of their own (the type of the
// parameters selects the epilogue): as run-time branches of every instance they cost the others registers, 16 -> 24 spilled ones
// of a 256 x 256 tile, 3 to 4 more and 17 scalar ones of the other tiles of 256 weight rows.
struct GemmRotateParams : GemmParams {
  PrefillRotation rot;
};
struct GemmMaxParams : GemmParams {
  float* row_max;  // [M][2 tiles_n]
};
struct GemmStatsParams : GemmParams {
  static constexpr bool kStatistics = true;
  RowStatistics stats;
};
// Operands of 8-bit integers: 64 codes where 32 bf16 stood, byte for byte the same tiles, rings and fragments (offsets and strides count
// pairs of codes), v_mfma_i32_16x16x64_i8 in the place of v_mfma_f32_16x16x32_bf16 - the same cycles for twice the products.  The
// accumulators are int32 in the registers of the fp32 ones, and so are the partials of a split: a sum over K is exact (a lane's
// |sum| <= 127 * 128 K - weights may hold -128 - which K <= 2^17 keeps below 2^31), so a result does not depend on the plan or on the
// batch around it.
struct GemmIntParams : GemmParams {
  static constexpr bool kIntegers = true;
  const float* a_scale;  // [M]
  const float* w_scale;  // [Npad], by weight row
};
struct GemmIntStatsParams : GemmIntParams {
  static constexpr bool kStatistics = true;
  RowStatistics stats;
};

// Residual add and store of four consecutive output columns (plain / residual epilogues).
__device__ __forceinline__ void store_row4(const GemmParams& p, int m, int n, float (&v)[4]) {
  if (p.bias) {
    const f32x4 b = *reinterpret_cast<const f32x4*>(p.bias + n);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] += b[e];
  }
  if (p.epilogue == EPI_RESIDUAL) {
    if (p.res_f32) {
      const f32x4 r = *reinterpret_cast<const f32x4*>((const float*)p.residual + (int64_t)m * p.ldr + n);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += r[e];
    } else {
      const bf16x4 r = *reinterpret_cast<const bf16x4*>((const bf16*)p.residual + (int64_t)m * p.ldr + n);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += (float)r[e];
    }
  }
  if (p.out_f32) {
    *reinterpret_cast<f32x4*>((float*)p.out + (int64_t)m * p.ldo + n) = f32x4{v[0], v[1], v[2], v[3]};
  } else {
    bf16x4 o;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = (bf16)v[e];
    *reinterpret_cast<bf16x4*>(p.out + (int64_t)m * p.ldo + n) = o;
  }
}

__device__ __forceinline__ void store_values4(const GemmParams& p, int m, int n, const float (&v)[4]) {
  if (p.out_f32) {
    *reinterpret_cast<f32x4*>((float*)p.out + (int64_t)m * p.ldo + n) = f32x4{v[0], v[1], v[2], v[3]};
  } else {
    bf16x4 o;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = (bf16)v[e];
    *reinterpret_cast<bf16x4*>(p.out + (int64_t)m * p.ldo + n) = o;
  }
}

// Epilogue of the GEMM kernel (16x16 accumulator tiles): a lane holds, for each (wt, at), output columns
// n..n+3 of row m, with m = row0 + at*16 + l16 and n = col0 + wt*16 + kq*4.  Gate and up rows
// alternate in blocks of 32 weight rows, i.e. tiles wt, wt+1 (gate) pair with wt+2, wt+3 (up).
template <int AT, int WT>
__device__ __forceinline__ void gemm_epilogue16(const GemmParams& p, f32x4 (&acc)[WT][AT], int row0, int col0,
                                                int l16, int kq, int split) {
#pragma unroll
  for (int at = 0; at < AT; ++at) {
    const int m = row0 + at * 16 + l16;
    if (m >= p.M) continue;
    if (p.splits > 1) {
      float* dst = p.ws + ((int64_t)split * p.M + m) * p.Npad;
#pragma unroll
      for (int wt = 0; wt < WT; ++wt) *reinterpret_cast<f32x4*>(dst + col0 + wt * 16 + kq * 4) = acc[wt][at];
    } else if (p.epilogue == EPI_SWIGLU) {
#pragma unroll
      for (int wt = 0; wt < WT; wt += 4)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int j = (col0 + wt * 16) / 2 + h * 16 + kq * 4;
          if (j < p.N_store) {
            bf16x4 o;
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = (bf16)(silu_f(acc[wt + h][at][e]) * acc[wt + h + 2][at][e]);
            *reinterpret_cast<bf16x4*>(p.out + operand_offset(p.u_lay, m, j)) = o;
          }
        }
    } else {
#pragma unroll
      for (int wt = 0; wt < WT; ++wt) {
        const int n = col0 + wt * 16 + kq * 4;
        if (n < p.N_store) {
          float v[4] = {acc[wt][at][0], acc[wt][at][1], acc[wt][at][2], acc[wt][at][3]};
          store_row4(p, m, n, v);
        }
      }
    }
  }
}

// The plain fp32 epilogue with the largest element of every row among the wave's 16 WT columns (unsplit, no bias; minus infinity
// where there is nothing but NaN).  The exchanges between lanes, two round trips through LDS for each row block, come behind all stores
// and are in flight together: made block by block in front of the next one's stores they took most of what the maxima save (see
// tdp_lm_head).  (Accumulators are read block by block; all read ahead they spill.)
template <int AT, int WT>
__device__ __forceinline__ void gemm_epilogue16_max(const GemmMaxParams& p, f32x4 (&acc)[WT][AT], int row0, int col0,
                                                    int l16, int kq) {
  float mx[AT];
#pragma unroll
  for (int at = 0; at < AT; ++at) {
    const int m = row0 + at * 16 + l16;
    float* out = (float*)p.out + (int64_t)m * p.ldo;
    mx[at] = -INFINITY;
#pragma unroll
    for (int wt = 0; wt < WT; ++wt) {
      const int n = col0 + wt * 16 + kq * 4;
      asm volatile("" : "+a"(acc[wt][at]));
      if (m < p.M && n < p.N_store) {
        const f32x4 v = acc[wt][at];
        *reinterpret_cast<f32x4*>(out + n) = v;
        mx[at] = fmaxf(fmaxf(mx[at], fmaxf(v[0], v[1])), fmaxf(v[2], v[3]));
      }
    }
  }
#pragma unroll
  for (int at = 0; at < AT; ++at) mx[at] = fmaxf(mx[at], __shfl_xor(mx[at], 16, 64));
#pragma unroll
  for (int at = 0; at < AT; ++at) mx[at] = fmaxf(mx[at], __shfl_xor(mx[at], 32, 64));
#pragma unroll
  for (int at = 0; at < AT; ++at) {
    const int m = row0 + at * 16 + l16;
    if (kq == 0 && m < p.M) p.row_max[(int64_t)m * (2 * p.tiles_n) + col0 / (16 * WT)] = mx[at];
  }
}

// The epilogue of an unsplit QKV projection in prefill: bias, rotation, one rounding; queries and values go to the bf16 rows, keys to
// their slots.  A wave's columns are whole heads (16 WT = 128: one of 128 channels or two of 64), so a lane holds both channels of
// its pairs: tile t of a head and tile t + H, H = head_dim / 32.  Bound: the stores, and two look-ups in a row (a token's position,
// then its (cos, sin)), asked for two row blocks at a time.  Against
// an fp32 projection that a kernel of its own reads back (19346 tokens of 70B: 2364 + 219 us; 7959 of 7B: 705 + 128; 6713 of Qwen: 467 +
// 52) the projection is no longer: 2325, 711, 441.
template <int AT, int WT, int H>
__device__ __forceinline__ void gemm_epilogue16_rotate(const GemmRotateParams& p, f32x4 (&acc)[WT][AT], int row0, int col0,
                                                       int l16, int kq) {
  const PrefillRotation& r = p.rot;
  constexpr int DH = 32 * H, AB = 2;
  const bool odd = kq & 1;  // channels 4 .. 7 of eight
  int2 where[AT];
#pragma unroll
  for (int at = 0; at < AT; ++at) where[at] = r.token_pages[min(row0 + at * 16 + l16, p.M - 1)];
#pragma unroll
  for (int hd = 0; hd < WT / (2 * H); ++hd) {
    const int col = col0 + hd * DH, head = col / DH, kvh = head - r.n_q_heads;
    if (kvh >= 2 * r.kv.n_kv_heads) continue;  // padding
    f32x4 bias[2 * H];
    if (p.bias) {
#pragma unroll
      for (int t = 0; t < 2 * H; ++t) bias[t] = *reinterpret_cast<const f32x4*>(p.bias + col + t * 16 + kq * 4);
    }
    const bool value = kvh >= r.kv.n_kv_heads;
#pragma unroll
    for (int a0 = 0; a0 < AT; a0 += AB) {
      float4 cs[AB][H][2];
      if (!value) {
#pragma unroll
        for (int ab = 0; ab < AB; ++ab) {
          if (a0 + ab >= AT) break;
          const float4* table = reinterpret_cast<const float4*>(r.rope_table + (int64_t)where[a0 + ab].x * (DH / 2) + kq * 4);
#pragma unroll
          for (int t = 0; t < H; ++t) {
            cs[ab][t][0] = table[t * 8];
            cs[ab][t][1] = table[t * 8 + 1];
          }
        }
      }
#pragma unroll
      for (int ab = 0; ab < AB; ++ab) {
        const int at = a0 + ab;
        if (at >= AT) break;
        const int m = row0 + at * 16 + l16;
        if (m >= p.M) continue;
        bf16* row = (bf16*)r.qkv + (int64_t)m * r.ld + col + kq * 4;
        const int64_t page = where[at].y;
        const int slot = where[at].x & 15;
#pragma unroll
        for (int t = 0; t < H; ++t) {
          asm volatile("" : "+a"(acc[hd * 2 * H + t][at]), "+a"(acc[hd * 2 * H + t + H][at]));  // (not all read ahead: they would spill)
          f32x4 a = acc[hd * 2 * H + t][at], b = acc[hd * 2 * H + t + H][at];
          if (p.bias) {
            a += bias[t];
            b += bias[t + H];
          }
          float lo[4] = {a[0], a[1], a[2], a[3]}, hi[4] = {b[0], b[1], b[2], b[3]};
          if (!value) {
            const float4 c0 = cs[ab][t][0], c1 = cs[ab][t][1];
            rotate_pair(a[0], b[0], make_float2(c0.x, c0.y), 0, lo[0], hi[0]);  // (channel 0 and 4, ... of eight are alike but for 3)
            rotate_pair(a[1], b[1], make_float2(c0.z, c0.w), 1, lo[1], hi[1]);
            rotate_pair(a[2], b[2], make_float2(c1.x, c1.y), 2, lo[2], hi[2]);
            rotate_pair(a[3], b[3], make_float2(c1.z, c1.w), odd ? 7 : 3, lo[3], hi[3]);
          }
          bf16x4 l4, h4;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            l4[e] = (bf16)lo[e];
            h4[e] = (bf16)hi[e];
          }
          if (value || kvh < 0) {
            *reinterpret_cast<bf16x4*>(row + t * 16) = l4;
            *reinterpret_cast<bf16x4*>(row + (t + H) * 16) = h4;
          } else {
            const int c = t * 16 + kq * 4;
            uint8_t* pool = (uint8_t*)r.kv.k_pool;
            *reinterpret_cast<bf16x4*>(pool + k_pool_byte(r.kv, page, kvh, slot, 2 * c)) = l4;
            *reinterpret_cast<bf16x4*>(pool + k_pool_byte(r.kv, page, kvh, slot, 2 * c + DH)) = h4;
          }
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  }
}

// The residual epilogue of a whole tile (no split-K, no bias): out = acc + residual.  The residual of
// half the wave's tile is requested in one go - addresses clamped into the matrix instead of guarded,
// so that nothing but loads stands between the first request and the last - and only then added and
// stored: fetched row block by row block behind guards, the loads of one row block were all that
// was ever in flight, and the eight round trips took 45 us per 256 x 256 tile against 12 us for the
// epilogue without a residual (measured; the registers that held the operand fragments are free here).
template <int AT, int WT>
__device__ __forceinline__ void gemm_epilogue16_residual(const GemmParams& p, f32x4 (&acc)[WT][AT], int row0,
                                                         int col0, int l16, int kq) {
  constexpr int AB = AT > 4 ? (AT + 1) / 2 : AT;  // row blocks per batch
  const int n_last = p.N_store - 4;
#pragma unroll
  for (int a0 = 0; a0 < AT; a0 += AB) {
    f32x4 r[AB][WT];
#pragma unroll
    for (int ab = 0; ab < AB; ++ab) {
      if (a0 + ab >= AT) break;
      const int m = min(row0 + (a0 + ab) * 16 + l16, p.M - 1);
#pragma unroll
      for (int wt = 0; wt < WT; ++wt) {
        const int n = min(col0 + wt * 16 + kq * 4, n_last);
        if (p.res_f32) {
          r[ab][wt] = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>((const float*)p.residual + (int64_t)m * p.ldr + n));
        } else {
          const bf16x4 t = *reinterpret_cast<const bf16x4*>((const bf16*)p.residual + (int64_t)m * p.ldr + n);
          r[ab][wt] = f32x4{(float)t[0], (float)t[1], (float)t[2], (float)t[3]};
        }
      }
    }
#pragma unroll
    for (int ab = 0; ab < AB; ++ab) {
      if (a0 + ab >= AT) break;
      const int m = row0 + (a0 + ab) * 16 + l16;
#pragma unroll
      for (int wt = 0; wt < WT; ++wt) {
        const int n = col0 + wt * 16 + kq * 4;
        if (m < p.M && n < p.N_store) {
          const f32x4 v = acc[wt][a0 + ab] + r[ab][wt];
          if (p.out_f32) {
            *reinterpret_cast<f32x4*>((float*)p.out + (int64_t)m * p.ldo + n) = v;
          } else {
            bf16x4 o;
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = (bf16)v[e];
            *reinterpret_cast<bf16x4*>(p.out + (int64_t)m * p.ldo + n) = o;
          }
        }
      }
    }
  }
}

// Four int32 sums in an accumulator's registers -> the values they stand for.  (Conversion and two products round three times in
// fp32, 2^-22 in all at most.)
__device__ __forceinline__ f32x4 scaled(f32x4 acc, f32x4 w_scale, float a_scale) {
  const i32x4 c = __builtin_bit_cast(i32x4, acc);
  f32x4 v;
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = (float)c[e] * w_scale[e] * a_scale;
  return v;
}

// The epilogues of a product of integers (plain, residual, gated; bf16 or fp32 results).  Scales, and in gemm_epilogue16_residual's manner
// half a tile's residual, are requested in one go, with addresses clamped into the matrix, in front of the arithmetic.
template <int AT, int WT>
__device__ __forceinline__ void gemm_epilogue16_int(const GemmIntParams& p, f32x4 (&acc)[WT][AT], int row0, int col0,
                                                    int l16, int kq, int split) {
  if (p.splits > 1) {
#pragma unroll
    for (int at = 0; at < AT; ++at) {
      const int m = row0 + at * 16 + l16;
      if (m >= p.M) continue;
      float* dst = p.ws + ((int64_t)split * p.M + m) * p.Npad;
#pragma unroll
      for (int wt = 0; wt < WT; ++wt) *reinterpret_cast<f32x4*>(dst + col0 + wt * 16 + kq * 4) = acc[wt][at];
    }
    return;
  }
  f32x4 ws[WT];
  float as[AT];
#pragma unroll
  for (int wt = 0; wt < WT; ++wt) ws[wt] = *reinterpret_cast<const f32x4*>(p.w_scale + col0 + wt * 16 + kq * 4);
#pragma unroll
  for (int at = 0; at < AT; ++at) as[at] = p.a_scale[min(row0 + at * 16 + l16, p.M - 1)];
  if (p.epilogue == EPI_SWIGLU) {
#pragma unroll
    for (int at = 0; at < AT; ++at) {
      const int m = row0 + at * 16 + l16;
#pragma unroll
      for (int wt = 0; wt < WT; wt += 4)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int j = (col0 + wt * 16) / 2 + h * 16 + kq * 4;
          asm volatile("" : "+a"(acc[wt + h][at]), "+a"(acc[wt + h + 2][at]));  // (not all read ahead: they would spill)
          if (m < p.M && j < p.N_store) {
            const f32x4 g = scaled(acc[wt + h][at], ws[wt + h], as[at]), u = scaled(acc[wt + h + 2][at], ws[wt + h + 2], as[at]);
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = silu_f(g[e]) * u[e];
            store_values4(p, m, j, v);
          }
        }
    }
    return;
  }
  if (p.epilogue == EPI_RESIDUAL) {
    constexpr int AB = AT > 4 ? (AT + 1) / 2 : AT;  // row blocks per batch
    const int n_last = p.N_store - 4;
#pragma unroll
    for (int a0 = 0; a0 < AT; a0 += AB) {
      f32x4 r[AB][WT];
#pragma unroll
      for (int ab = 0; ab < AB; ++ab) {
        if (a0 + ab >= AT) break;
        const int m = min(row0 + (a0 + ab) * 16 + l16, p.M - 1);
#pragma unroll
        for (int wt = 0; wt < WT; ++wt) {
          const int n = min(col0 + wt * 16 + kq * 4, n_last);
          if (p.res_f32) {
            r[ab][wt] = *reinterpret_cast<const f32x4*>((const float*)p.residual + (int64_t)m * p.ldr + n);
          } else {
            const bf16x4 t = *reinterpret_cast<const bf16x4*>((const bf16*)p.residual + (int64_t)m * p.ldr + n);
            r[ab][wt] = f32x4{(float)t[0], (float)t[1], (float)t[2], (float)t[3]};
          }
        }
      }
#pragma unroll
      for (int ab = 0; ab < AB; ++ab) {
        if (a0 + ab >= AT) break;
        const int m = row0 + (a0 + ab) * 16 + l16;
#pragma unroll
        for (int wt = 0; wt < WT; ++wt) {
          const int n = col0 + wt * 16 + kq * 4;
          asm volatile("" : "+a"(acc[wt][a0 + ab]));
          if (m < p.M && n < p.N_store) {
            f32x4 v = scaled(acc[wt][a0 + ab], ws[wt], as[a0 + ab]);
            if (p.bias) v += *reinterpret_cast<const f32x4*>(p.bias + n);
            v += r[ab][wt];
            float o[4] = {v[0], v[1], v[2], v[3]};
            store_values4(p, m, n, o);
          }
        }
      }
    }
    return;
  }
#pragma unroll
  for (int at = 0; at < AT; ++at) {
    const int m = row0 + at * 16 + l16;
#pragma unroll
    for (int wt = 0; wt < WT; ++wt) {
      const int n = col0 + wt * 16 + kq * 4;
      asm volatile("" : "+a"(acc[wt][at]));
      if (m < p.M && n < p.N_store) {
        f32x4 v = scaled(acc[wt][at], ws[wt], as[at]);
        if (p.bias) v += *reinterpret_cast<const f32x4*>(p.bias + n);
        float o[4] = {v[0], v[1], v[2], v[3]};
        store_values4(p, m, n, o);
      }
    }
  }
}

// The statistics of every row among the wave's 16 WT columns, for log-probabilities (LogSum), and the logit of the row's given token
// where it is among them.  A lane makes them of its own 4 WT logits in registers, relative to its own largest; the four lanes of
// a row are joined behind all rows' arithmetic, with the exchanges of all row blocks in flight.  Logits are stored if the call
// needs them later.
template <int AT, int WT, typename Params>
__device__ __forceinline__ void gemm_epilogue16_stats(const Params& p, f32x4 (&acc)[WT][AT], int row0, int col0,
                                                      int l16, int kq) {
  const RowStatistics& st = p.stats;
  f32x4 ws[WT];
  float as[AT];
  if constexpr (Params::kIntegers) {
#pragma unroll
    for (int wt = 0; wt < WT; ++wt) ws[wt] = *reinterpret_cast<const f32x4*>(p.w_scale + col0 + wt * 16 + kq * 4);
#pragma unroll
    for (int at = 0; at < AT; ++at) as[at] = p.a_scale[min(row0 + at * 16 + l16, p.M - 1)];
  }
  int target[AT];
#pragma unroll
  for (int at = 0; at < AT; ++at) target[at] = st.targets ? st.targets[min(row0 + at * 16 + l16, p.M - 1)] : -1;
  LogSum sum[AT];
#pragma unroll
  for (int at = 0; at < AT; ++at) {
    const int m = row0 + at * 16 + l16;
    f32x4 z[WT];
#pragma unroll
    for (int wt = 0; wt < WT; ++wt) {
      const int n = col0 + wt * 16 + kq * 4;
      asm volatile("" : "+a"(acc[wt][at]));
      z[wt] = acc[wt][at];
      if constexpr (Params::kIntegers) z[wt] = scaled(z[wt], ws[wt], as[at]);
      if (n >= p.N_store) {
        z[wt] = f32x4{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
      } else if (m < p.M) {
        if (st.store) *reinterpret_cast<f32x4*>((float*)p.out + (int64_t)m * p.ldo + n) = z[wt];
        const unsigned e = (unsigned)(target[at] - n);
        if (e < 4u) st.target_logit[m] = e == 0 ? z[wt][0] : e == 1 ? z[wt][1] : e == 2 ? z[wt][2] : z[wt][3];
      }
    }
    float mx = -INFINITY;
#pragma unroll
    for (int wt = 0; wt < WT; ++wt) mx = fmaxf(fmaxf(mx, fmaxf(z[wt][0], z[wt][1])), fmaxf(z[wt][2], z[wt][3]));
    sum[at] = LogSum{mx, 0.f, 0.f};
    const float r = reference_of(mx);
#pragma unroll
    for (int wt = 0; wt < WT; ++wt)
#pragma unroll
      for (int e = 0; e < 4; ++e) add_distance(sum[at], z[wt][e] - r);
    __builtin_amdgcn_sched_barrier(0);
  }
#pragma unroll
  for (int o = 16; o < 64; o *= 2) {
    LogSum other[AT];
#pragma unroll
    for (int at = 0; at < AT; ++at) other[at] = of_lane(sum[at], o);
#pragma unroll
    for (int at = 0; at < AT; ++at) join(sum[at], other[at]);
  }
#pragma unroll
  for (int at = 0; at < AT; ++at) {
    const int m = row0 + at * 16 + l16;
    if (kq == 0 && m < p.M) {
      const int64_t i = (int64_t)m * (2 * p.tiles_n) + col0 / (16 * WT);
      st.max[i] = sum[at].max;
      st.sum[i] = sum[at].sum;
      st.weighted[i] = sum[at].weighted;
    }
  }
}

// Workgroup -> (tile_m, tile_n, split).  The tiles are put in one order - by split, by band of up to four rows of
// tiles, and inside a band column by column - so that any run of consecutive tiles is a compact block: the
// workgroups that make it share a band's activation panels and as few weight panels as there can be.
// Workgroups are dealt round-robin to the 8 XCDs, each with its own L2: an XCD takes runs of as many
// tiles as it has slots, the eight XCDs' runs side by side, and what is left is divided evenly.  Every
// workgroup but the last few of the grid has a tile.  (An earlier numbering gave an XCD rectangles of tiles whose
// corners could lie outside the matrix: the workgroups that found nothing to do sat at regular ids, and
// as the dispatcher hands out ids to the four shader engines of an XCD in turn, two of them got all the
// work: with three or six rows of tiles a launch took twice its time, 121 us against 61 at M = 384 on 10240 x 8192.)
// (The look-up stands in front of a workgroup's first request, so its divisions are by multiplication: x / d =
// umulhi(x, ceil(2^32 / d)) while x * d < 2^32, 0 standing for d = 1 and for divisors where that does not hold.)
__device__ __forceinline__ int divide(int x, int d, unsigned inv) {
  return inv ? (int)__umulhi((unsigned)x, inv) : d == 1 ? x : x / d;
}
__device__ __forceinline__ bool gemm_tile_of_block(const GemmParams& p, int& tile_m, int& tile_n, int& split) {
  const int xcd = blockIdx.x & 7;
  int local = blockIdx.x >> 3;
  int t;
  const int whole = p.chunks << p.chunk_shift;  // tiles of this XCD that come in whole runs
  if (local < whole) {
    const int run = local >> p.chunk_shift;
    t = ((run * 8 + xcd) << p.chunk_shift) + (local - (run << p.chunk_shift));
  } else {
    local -= whole;
    const int q = p.rest >> 3, r = p.rest & 7;
    if (local >= q + (xcd < r ? 1 : 0)) return false;
    t = whole * 8 + xcd * q + min(xcd, r) + local;
  }
  const int per_split = p.tiles_m * p.tiles_n;
  split = divide(t, per_split, p.per_split_inv);
  t -= split * per_split;
  const int tall = (p.band_h + 1) * p.tiles_n, low = p.band_h * p.tiles_n;  // tiles per band
  if (t < p.n_tall * tall) {
    const int band = divide(t, tall, p.tall_inv);
    t -= band * tall;
    tile_n = divide(t, p.band_h + 1, p.h_tall_inv);
    tile_m = band * (p.band_h + 1) + t - tile_n * (p.band_h + 1);
  } else {
    t -= p.n_tall * tall;
    const int band = divide(t, low, p.low_inv);
    t -= band * low;
    tile_n = divide(t, p.band_h, p.h_low_inv);
    tile_m = p.n_tall * (p.band_h + 1) + band * p.band_h + t - tile_n * p.band_h;
  }
  return true;
}

// The same pipeline on v_mfma_f32_16x16x32_bf16: a stage of 32 k is exactly one MFMA k-step, a wave
// tile of (TM*32) x (TN*32) is (TM*2) x (TN*2) accumulators of four registers.  Operand bytes read
// from LDS per flop are the same as with 32x32x16 tiles, but the accumulator traffic in the
// register file is half, and on a power-limited part that buys clock: with random operands an
// MFMA-only loop sustains 2.16 PFLOP/s with 16x16x32 against 1.89 with 32x32x16 (measured).
// Fragments of stage t+1 are read under the MFMAs of stage t (two register sets, the stage loop
// is unrolled by two); one barrier per stage, at its start.
//
// WNT: the weight tiles are requested as non-temporal.  With a single row of tiles (M up to the tile's
// rows: the decode sizes) every weight byte is read by exactly one workgroup, so keeping it in L2
// only evicts what is shared - the activation panel, the split-K partials.  Measured at M = 32 ... 256
// on the 70B shapes: +6 to +12 % on the down projection, +2 to +8 % on gate/up, +1 to +4 % on QKV and
// O.  With more tile rows the weights are shared through L2 and the hint costs 5-10 % on the large
// shapes; the one exception that pays is two tile rows on a wide projection without split-K (gate/up at
// M = 512: the two readers of a weight tile are neighbours in the order of the tiles and run at the same
// time, so the second read still finds the line): -1.8 %.
//
// Tiles of up to 128 x 128 can sum K in chunks (see sum_order_splits): a second set of accumulators (which costs 128 x 128
// its second workgroup per CU, so there are two forms of that).
template <int AT, int WT, int NS>
constexpr bool kChunked = AT * WT <= 12 || (AT == 4 && WT == 4 && NS == 9);

// A workgroup of four waves (2 x 2) makes a tile of BM = 32 AT rows x BN = 32 WT weight rows; a wave, AT x WT
// accumulators.
template <int AT, int WT, int NS, bool WNT, typename Params>
__global__ __launch_bounds__(256) void gemm_mi16_kernel(const Params p) {
  constexpr int BM = AT * 32, BN = WT * 32, BK = 32;
  constexpr int CPR = BK / 8;         // 16-byte chunks per row
  // Rows that share one swizzle value.  A fragment read of this kernel is 16 rows x 4 chunks (lane =
  // chunk * 16 + row); measured with SQ_LDS_BANK_CONFLICT on that pattern: the chunk position must
  // turn every 2 rows to be conflict free (4 LDS cycles per ds_read_b128); turning every 4 rows -
  // right for the 32 rows x 2 chunks of the 32x32 kernels - costs 8 cycles per read here.
  constexpr int RW = 2;
  constexpr int RPI = 64 / CPR;       // rows per DMA instruction
  // DMA instructions per wave and stage.  Where the 2 AT row blocks of the activations do not divide by four, the
  // last waves request rows of the tile a second time, into ring rows that nothing reads (BMR > BM).
  constexpr int IPA = (BM / RPI + 3) / 4, IPW = BN / RPI / 4;
  constexpr int BMR = IPA * 4 * RPI;
  constexpr int STAGE = (BMR + BN) * BK;
  static_assert(WT % 4 == 0, "gate/up pairing");
  extern __shared__ __attribute__((aligned(16))) unsigned char smem_raw[];
  bf16* smem = reinterpret_cast<bf16*>(smem_raw);  // [NS][BMR + BN][BK]

  int tile_m, tile_n, split;
  if (!gemm_tile_of_block(p, tile_m, tile_n, split)) return;
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm0 = (wave >> 1) * (AT * 16);
  const int wn0 = (wave & 1) * (WT * 16);
  const int l16 = lane & 15;
  const int kq = lane >> 4;
  const int m0 = tile_m * BM;
  const int n0 = tile_n * BN;
  const int kt_begin = split * p.k_tiles_per_split * 2;
  int kt_end = kt_begin + p.k_tiles_per_split * 2;
  if (kt_end > p.k_tiles_total * 2) kt_end = p.k_tiles_total * 2;
  const int n_stages = kt_end - kt_begin;  // even: two stages per 64-wide k-tile

  // DMA addressing: a wave-uniform 64-bit base per operand, which moves one k-stage per request,
  // plus loop-invariant 32-bit per-lane byte offsets (scalar base + vector offset needs no vector
  // arithmetic per load).
  typedef const __attribute__((address_space(1))) char* gptr;
  const int r_in = lane / CPR;
  // Instruction j of an operand lands 1 KiB further on in LDS than instruction 0; that distance
  // rides in the instruction's immediate offset, which also moves the global address, so it is
  // taken out of the per-lane offsets again.  The per-lane offset is zero-extended by the hardware
  // and must not go negative: a constant bias keeps it positive and is subtracted from the bases.
  constexpr int kImmBias = 3 * 1024;
  const int valid = min(BM, p.M - m0), spread = (1 << (31 - __builtin_clz(valid))) - 1;
  unsigned a_goff[IPA];  // bytes
#pragma unroll
  for (int j = 0; j < IPA; ++j) {
    const int row = (wave * IPA + j) * RPI + r_in;
    const int c_sw = (lane % CPR) ^ ((row / RW) % CPR);
    // rows past M are computed but never stored; they re-read the tile's valid rows in turn (all of
    // them reading the last valid row makes one hot line for every workgroup of the launch)
    const int m = row < valid ? row : row & spread;
    a_goff[j] = 2u * (unsigned)(operand_row_offset(p.a_lay, m) + c_sw * 8) + (unsigned)(kImmBias - j * 1024);
  }
  // weight rows need no clamp; the swizzle term (row / RW) % CPR does not depend on the row block j
  // (RPI is a multiple of RW * CPR)
  static_assert(RPI % (RW * CPR) == 0, "the swizzle repeats per row block");
  unsigned w_goff[IPW];
#pragma unroll
  for (int j = 0; j < IPW; ++j) {
    const int row = (wave * IPW + j) * RPI + r_in;
    const int c_sw = (lane % CPR) ^ ((row / RW) % CPR);
    w_goff[j] = 2u * (unsigned)(operand_row_offset(p.w_lay, row) + c_sw * 8) + (unsigned)(kImmBias - j * 1024);
  }
  const int64_t a_step = 2 * p.a_lay.kb, w_step = 2 * p.w_lay.kb;  // bytes per k-stage
  // the stage being requested: global bases, index and ring slot; past the last stage the bases
  // stay put, so the tail re-fetches the last stage (valid memory, never read)
  gptr a_req = (gptr)(p.A + operand_row_offset(p.a_lay, m0) + (int64_t)kt_begin * p.a_lay.kb) - kImmBias;
  gptr w_req = (gptr)(p.W + operand_row_offset(p.w_lay, n0) + (int64_t)kt_begin * p.w_lay.kb) - kImmBias;
  int req_t = 0, req_slot = 0;
  constexpr int N_DMA = IPA + IPW;
  // One DMA instruction: 64 lanes x 16 bytes from (scalar base + per-lane byte offset) into 1 KiB
  // of LDS at lds_addr.  Written as assembly to get the scalar-base form (no vector address
  // arithmetic per load); M0 carries the LDS address, and every DMA of this kernel goes through
  // here, so nothing else depends on M0.
  auto dma_aim = [](unsigned lds_addr) { asm volatile("s_mov_b32 m0, %0\n\ts_nop 0" ::"s"(lds_addr) : "memory"); };
#define TDP_DMA16(lane_off, base, imm) \
  asm volatile("global_load_lds_dwordx4 %0, %1 offset:%2" ::"v"(lane_off), "s"(base), "n"(imm) : "memory")
#define TDP_DMA16W(lane_off, base, imm)                                                                              \
  do {                                                                                                               \
    if constexpr (WNT)                                                                                               \
      asm volatile("global_load_lds_dwordx4 %0, %1 offset:%2 nt" ::"v"(lane_off), "s"(base), "n"(imm) : "memory");   \
    else                                                                                                             \
      asm volatile("global_load_lds_dwordx4 %0, %1 offset:%2" ::"v"(lane_off), "s"(base), "n"(imm) : "memory");      \
  } while (0)
  const unsigned ring_base = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char*)smem_raw;
  static_assert(IPA <= 4 && IPW <= 4, "immediate offsets up to 3 KiB");
  // instruction j of the requested stage: activations first, then weights; M0 is aimed at the
  // wave's first KiB of each operand once per stage
  auto dma_one = [&](int j) {
    const unsigned ring = ring_base + req_slot * (STAGE * 2);
    if (j == 0) dma_aim(ring + (wave * IPA * RPI * BK) * 2);
    if (j == IPA) dma_aim(ring + (BMR * BK + wave * IPW * RPI * BK) * 2);
    switch (j < IPA ? j : j - IPA) {
      case 0: if (j < IPA) TDP_DMA16(a_goff[0], a_req, 0); else TDP_DMA16W(w_goff[0], w_req, 0); break;
      case 1: if (j < IPA) TDP_DMA16(a_goff[1 % IPA], a_req, 1024); else TDP_DMA16W(w_goff[1 % IPW], w_req, 1024); break;
      case 2: if (j < IPA) TDP_DMA16(a_goff[2 % IPA], a_req, 2048); else TDP_DMA16W(w_goff[2 % IPW], w_req, 2048); break;
      default: if (j < IPA) TDP_DMA16(a_goff[3 % IPA], a_req, 3072); else TDP_DMA16W(w_goff[3 % IPW], w_req, 3072); break;
    }
  };
#undef TDP_DMA16
#undef TDP_DMA16W
  auto dma_advance = [&]() {
    ++req_t;
    if (req_t < n_stages) {
      a_req += a_step;
      w_req += w_step;
    }
    req_slot = req_slot + 1 == NS ? 0 : req_slot + 1;
  };
  auto dma_stage = [&]() {
#pragma unroll
    for (int j = 0; j < N_DMA; ++j) dma_one(j);
    dma_advance();
  };

  f32x4 acc[WT][AT];
#pragma unroll
  for (int wt = 0; wt < WT; ++wt)
#pragma unroll
    for (int at = 0; at < AT; ++at) acc[wt][at] = f32x4{0.f, 0.f, 0.f, 0.f};

  // fragment reads: lane (l16, kq) supplies row l16 of a 16-row tile, k = kq*8 .. +8 of the stage
  // Tile wt / at lies 16 rows = 16 * BK elements further on and 16 is a multiple of RW * CPR, so
  // the swizzle term is the lane's alone: one base per operand, the rest are immediate offsets.
  static_assert(16 % (RW * CPR) == 0, "swizzle repeats every 16 rows");
  const int swz = (kq ^ ((l16 / RW) % CPR)) << 3;
  const int w_off = (BMR + wn0 + l16) * BK + swz;
  const int a_off = (wm0 + l16) * BK + swz;
  bf16x8 wf[2][WT], af[2][AT];
  constexpr int PENDING = (NS - 2) * N_DMA;
  int rd_slot = 0;  // ring slot of the stage whose fragments are read next
  int w_next = w_off, a_next = a_off;  // this lane's fragments in that slot (element offsets into smem)
  auto read_frags = [&](int set) {
    const bf16* base = smem + rd_slot * STAGE;
#pragma unroll
    for (int wt = 0; wt < WT; ++wt) wf[set][wt] = ld_bf16x8(base + w_off + wt * 16 * BK);
#pragma unroll
    for (int at = 0; at < AT; ++at) af[set][at] = ld_bf16x8(base + a_off + at * 16 * BK);
  };
  // One stage: its fragments are in register set `set`; the next stage was requested NS-2
  // barriers ago.  The MFMAs are inline assembly so that every accumulator stays in place in its
  // AGPRs (left to itself the register allocator shuttles the 64 accumulator tuples through
  // VGPRs); issue order is therefore explicit: everything that is not an MFMA - the WT + AT fragment reads
  // and the N_DMA requests of the stages ahead, then the stage's bookkeeping - goes behind single MFMAs, a
  // few instructions at a time, so that it issues while the matrix pipe is busy instead of in a gap of
  // the MFMA stream, and is pinned there by scheduling barriers.
  constexpr int N_MFMA = AT * WT;
  constexpr bool GROUPED = AT >= 4 && AT <= WT && N_DMA <= WT;  // a weight read, an activation read, a request per MFMA group
  constexpr int N_OPS = WT + AT + N_DMA;
  auto stage = [&](int set) {
    // vmcnt: this wave's loads of the next stage have landed; lgkmcnt: its reads of this stage are
    // complete, so after the barrier this stage's buffer may be refilled and the next one read
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(PENDING) : "memory");
#pragma unroll
    for (int i = 0; i < N_MFMA; ++i) {
      const int wt = i / AT, at = i % AT;
      if constexpr (Params::kIntegers)
        asm volatile("v_mfma_i32_16x16x64_i8 %0, %1, %2, %0" : "+a"(acc[wt][at]) : "v"(wf[set][wt]), "v"(af[set][at]));
      else
        asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(acc[wt][at]) : "v"(wf[set][wt]), "v"(af[set][at]));
      if constexpr (GROUPED) {
        if (at < 3) __builtin_amdgcn_sched_barrier(0);
        if (at == 0) wf[set ^ 1][wt] = ld_bf16x8(smem + w_next + wt * 16 * BK);
        if (at == 1 && wt < AT) af[set ^ 1][wt] = ld_bf16x8(smem + a_next + wt * 16 * BK);
        if (at == 2 && wt < N_DMA) dma_one(wt);
        if (at < 3) __builtin_amdgcn_sched_barrier(0);
      } else {
        // operations first .. last - 1 of the list (weight reads, activation reads, requests) are this MFMA's
        const int first = (i * N_OPS + N_MFMA - 2) / (N_MFMA - 1), last = ((i + 1) * N_OPS + N_MFMA - 2) / (N_MFMA - 1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int op = first; op < last && op < N_OPS; ++op) {
          if (op < WT) wf[set ^ 1][op] = ld_bf16x8(smem + w_next + op * 16 * BK);
          else if (op < WT + AT) af[set ^ 1][op - WT] = ld_bf16x8(smem + a_next + (op - WT) * 16 * BK);
          else dma_one(op - WT - AT);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      // the bookkeeping, behind MFMAs of the last group that carry nothing else: the request side moves on one
      // stage, and so do the fragment offsets.  (The empty statements make the new values exist here
      // rather than wherever their next use is.)
      if (i == (GROUPED ? (WT - 1) * AT + 3 : N_MFMA - 1)) {
        __builtin_amdgcn_sched_barrier(0);
        ++req_t;
        if (req_t < n_stages) {
          a_req += a_step;
          w_req += w_step;
        }
        asm volatile("" : "+s"(a_req), "+s"(w_req), "+s"(req_t));
        __builtin_amdgcn_sched_barrier(0);
      }
      if (i == (GROUPED ? (WT - 1) * AT + (AT > 4 ? 4 : 3) : N_MFMA - 1)) {
        __builtin_amdgcn_sched_barrier(0);
        req_slot = req_slot + 1 == NS ? 0 : req_slot + 1;
        rd_slot = rd_slot + 1 == NS ? 0 : rd_slot + 1;
        asm volatile("" : "+s"(req_slot), "+s"(rd_slot));
        __builtin_amdgcn_sched_barrier(0);
      }
      if (i == (GROUPED ? (WT - 1) * AT + (AT > 5 ? 5 : AT > 4 ? 4 : 3) : N_MFMA - 1)) {
        __builtin_amdgcn_sched_barrier(0);
        w_next = rd_slot * STAGE + w_off;
        a_next = rd_slot * STAGE + a_off;
        asm volatile("" : "+v"(w_next), "+v"(a_next));
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };

  if (n_stages > 0) {
#pragma unroll
    for (int t = 0; t < NS - 1; ++t) dma_stage();
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(PENDING) : "memory");
    read_frags(0);
    rd_slot = 1 % NS;
    w_next = rd_slot * STAGE + w_off;
    a_next = rd_slot * STAGE + a_off;
    dma_stage();
  }
  if constexpr (kChunked<AT, WT, NS> && !Params::kIntegers) {
    // In chunks: what split-K workgroups would leave as partials is added up here in the same order (the requests run on
    // across the ends of the chunks).
    const int chunk = p.k_tiles_per_chunk > 0 ? 2 * p.k_tiles_per_chunk : n_stages;
    f32x4 total[WT][AT];
    for (int t = 0; t < n_stages;) {
      const int end = min(t + chunk, n_stages);
      const bool first = t == 0;
      for (; t < end; t += 2) {
        stage(0);
        stage(1);
      }
      if (end == n_stages && first) break;  // one chunk: the accumulators are the sum
      asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");  // MFMA -> accumulator read, which the compiler cannot see
#pragma unroll
      for (int wt = 0; wt < WT; ++wt)
#pragma unroll
        for (int at = 0; at < AT; ++at) {
          // (pinned on both sides: the accumulators live in the inline MFMAs' registers)
          asm volatile("" : "+a"(acc[wt][at]));
          total[wt][at] = first ? acc[wt][at] : total[wt][at] + acc[wt][at];
          acc[wt][at] = end == n_stages ? total[wt][at] : f32x4{0.f, 0.f, 0.f, 0.f};
          asm volatile("" : "+a"(acc[wt][at]));
        }
      asm volatile("s_nop 7" ::: "memory");  // accumulator write -> MFMA
    }
  } else {
    for (int t = 0; t < n_stages; t += 2) {
      stage(0);
      stage(1);
    }
  }
  // loads still in flight target LDS only; they must land before the workgroup's LDS is released.
  // The nops cover the MFMA -> accumulator-read distance, which the compiler cannot see.
  asm volatile("s_waitcnt vmcnt(0)\n\ts_nop 15\n\ts_nop 15" ::: "memory");
  if constexpr (std::is_same_v<Params, GemmRotateParams>) {
    if (p.rot.kv.head_dim == 128) gemm_epilogue16_rotate<AT, WT, 4>(p, acc, m0 + wm0, n0 + wn0, l16, kq);
    else gemm_epilogue16_rotate<AT, WT, 2>(p, acc, m0 + wm0, n0 + wn0, l16, kq);
  } else if constexpr (std::is_same_v<Params, GemmMaxParams>) {
    gemm_epilogue16_max<AT, WT>(p, acc, m0 + wm0, n0 + wn0, l16, kq);
  } else if constexpr (Params::kStatistics) {
    gemm_epilogue16_stats<AT, WT>(p, acc, m0 + wm0, n0 + wn0, l16, kq);
  } else if constexpr (Params::kIntegers) {
    gemm_epilogue16_int<AT, WT>(p, acc, m0 + wm0, n0 + wn0, l16, kq, split);
  } else if (p.splits == 1 && p.epilogue == EPI_RESIDUAL && !p.bias && p.N_store >= 4) {
    gemm_epilogue16_residual<AT, WT>(p, acc, m0 + wm0, n0 + wn0, l16, kq);
  } else {
    gemm_epilogue16<AT, WT>(p, acc, m0 + wm0, n0 + wn0, l16, kq, split);
  }
}

// The tiles: rows / 32, weight rows / 32, ring slots, workgroups per CU, and the matrix pipe's part in us of a 32-wide stage of one
// tile on a CU (see plan_cost in gemm.hip).
#define TDP_GEMM_TILES(X)                                                     \
  X(8, 8, 4, 1, 0.425)                      /* 1: 256 x 256 */                 \
  X(4, 8, 6, 1, 0.252)                      /* 2: 128 x 256 */                 \
  X(4, 4, 4, 2, 0.129)                      /* 3: 128 x 128 */                 \
  /* 224, 192, 160 x 256 */                                                   \
  X(7, 8, 4, 1, 0.346) X(6, 8, 5, 1, 0.337) X(5, 8, 5, 1, 0.266)              \
  /* 256, 224, 160, 96 x 128 */                                               \
  X(8, 4, 6, 1, 0.244) X(7, 4, 6, 1, 0.202) X(5, 4, 7, 1, 0.168) X(3, 4, 8, 1, 0.097) \
  /* 128 x 128 with one workgroup per CU (sums in chunks); 64, 32 x 128 */    \
  X(4, 4, 9, 1, 0.129)                                                        \
  X(2, 4, 6, 2, 0.079) X(1, 4, 4, 3, 0.0415)

// The kernels of one kind of parameters, tile by tile, with ordinary and with non-temporal weight requests.  Kinds are compiled in files
// of their own.
struct GemmKernels {
  const void* of[2];
};
const GemmKernels* gemm_statistics_kernels();      // gemm_stats.hip
const GemmKernels* gemm_int_kernels();             // gemm_int.hip
const GemmKernels* gemm_int_statistics_kernels();  // gemm_int.hip

template <int AT, int WT, int NS, bool WNT, typename Params>
static const void* kernel_of() {
  if constexpr (std::is_same_v<Params, GemmRotateParams> && WT != 8) return nullptr;
  else if constexpr (Params::kIntegers && AT == 4 && WT == 4 && NS == 9) return nullptr;  // (kChunksOnlyTile)
  else return reinterpret_cast<const void*>(&gemm_mi16_kernel<AT, WT, NS, WNT, Params>);
}
#define TDP_KERNELS(AT, WT, NS, PARAMS) {{kernel_of<AT, WT, NS, false, PARAMS>(), kernel_of<AT, WT, NS, true, PARAMS>()}}

}  // namespace tdp
