// The GEMM kernels whose epilogue makes the statistics of log-probabilities.
#include "gemm_kernel.h"

namespace tdp {

#define TDP_TILE(AT, WT, NS, ...) TDP_KERNELS(AT, WT, NS, GemmStatsParams),
const GemmKernels* gemm_statistics_kernels() {
  static const GemmKernels kernels[] = {TDP_GEMM_TILES(TDP_TILE)};
  return kernels;
}
#undef TDP_TILE

}  // namespace tdp
