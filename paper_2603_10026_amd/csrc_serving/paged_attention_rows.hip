// Launches of paged_rows.h alone: batches without long chunks of new tokens.
#include "paged_rows.h"

namespace rf {

namespace {

template <int D, int NR, bool FP8>
__global__ __launch_bounds__(kWaves* kWave, 2) void paged_rows_kernel(const PagedArgs a) {
  __shared__ __attribute__((aligned(16))) unsigned char smem[rows_lds_bytes<D, NR, FP8>()];
  __shared__ ShareScratch scratch;
  paged_rows<D, NR, FP8>(a, blockIdx.x, smem, &scratch);
}

}  // namespace

hipError_t launch_paged_rows(const PagedArgs& a, bool fp8, hipStream_t s) {
  const int64_t grid = rows_blocks(a);
  if (grid > UINT32_MAX / (kWaves * kWave)) return hipErrorInvalidValue;
#define RF_ROWS(DD, NN, F8) \
  hipLaunchKernelGGL((paged_rows_kernel<DD, NN, F8>), dim3((unsigned)grid), dim3(kWaves * kWave), 0, s, a)
#define RF_ROWS_D(DD)                                                                        \
  if (a.deal.rows_log2 == 4) { if (fp8) RF_ROWS(DD, 1, true); else RF_ROWS(DD, 1, false); } \
  else { if (fp8) RF_ROWS(DD, 2, true); else RF_ROWS(DD, 2, false); }
  if (a.p.d == 128) {
    RF_ROWS_D(128);
  } else {
    RF_ROWS_D(64);
  }
#undef RF_ROWS_D
#undef RF_ROWS
  return hipGetLastError();
}

}  // namespace rf
