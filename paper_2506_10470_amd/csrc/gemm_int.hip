// The GEMM kernels of 8-bit integers.
#include "gemm_kernel.h"

namespace tdp {

#define TDP_TILE(AT, WT, NS, ...) TDP_KERNELS(AT, WT, NS, GemmIntParams),
const GemmKernels* gemm_int_kernels() {
  static const GemmKernels kernels[] = {TDP_GEMM_TILES(TDP_TILE)};
  return kernels;
}
#undef TDP_TILE

#define TDP_TILE(AT, WT, NS, ...) TDP_KERNELS(AT, WT, NS, GemmIntStatsParams),
const GemmKernels* gemm_int_statistics_kernels() {
  static const GemmKernels kernels[] = {TDP_GEMM_TILES(TDP_TILE)};
  return kernels;
}
#undef TDP_TILE

}  // namespace tdp
