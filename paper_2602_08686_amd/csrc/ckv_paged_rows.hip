// Attention over pages for few columns (ckv_paged_few.h): its kernels.
#include "ckv_paged_few.h"

namespace ckv {

template <int DT, int DH, int WAVES, bool STREAM>
__global__ void __launch_bounds__(WAVES *kWave, WAVES / 4) paged_rows_kernel(PagedArgs a) {
  attend_rows<DT, DH, WAVES, STREAM>(a);
}

template <int DT, int DH, int WAVES>
static void launch_rows_attention(const PagedArgs &a, hipStream_t stream) {
  // rows that one workgroup only reads are used once
  if (a.col_tiles == 1) hipLaunchKernelGGL((paged_rows_kernel<DT, DH, WAVES, true>), dim3((unsigned)a.workgroups), dim3(WAVES * kWave), 0, stream, a);
  else hipLaunchKernelGGL((paged_rows_kernel<DT, DH, WAVES, false>), dim3((unsigned)a.workgroups), dim3(WAVES * kWave), 0, stream, a);
}

void launch_paged_rows(const PagedArgs &a, bool bf16, int d, hipStream_t stream) {
  if (bf16 && d == 128) launch_rows_attention<CKV_BF16, 128, rows_waves(CKV_BF16, 128)>(a, stream);
  else if (bf16) launch_rows_attention<CKV_BF16, 64, rows_waves(CKV_BF16, 64)>(a, stream);
  else if (d == 128) launch_rows_attention<CKV_F32, 128, rows_waves(CKV_F32, 128)>(a, stream);
  else launch_rows_attention<CKV_F32, 64, rows_waves(CKV_F32, 64)>(a, stream);
}

}  // namespace ckv
