// Attention of trees of drafted tokens over pages (ckv_paged_tree_attention): the kernels of ckv_paged_few.h and ckv_paged_tile.h with a mask among the
// new tokens. Rows in front of them are seen by all, so the mask is looked at in the blocks of 32 rows that hold new ones alone: a column's 32 bits
// of such a block are two words of its token's, shifted, as the new rows begin anywhere in a block. The words come into LDS as rows do, ahead of their block.
// Weights in bf16 enter the second product in two terms, for many columns too, so that a token's result is as near to 64 bits as that of a one-token step.
// Measured, bf16, 32/8 heads of 128: 16 tokens of 16 sequences over up to 560 rows a head 13.9 us (a token 11.4), 60 tokens, batch 4, 32768 rows 217 us, 593
// TFLOP/s of the visible pairs' products, 500 tokens, batch 2, 4099 rows 105 us, 566; f32, 14/2 heads of 64, 33 tokens, 1501 rows 18.1 us.
// 32/8 heads of 64: 60 tokens, batch 4, 32768 rows 151, 500, batch 2, 4099 rows 79; f32, 100 tokens, batch 2, 4099 rows 158 with heads of 128, 85 of 64.
#include "ckv_paged_few.h"
#include "ckv_paged_tile.h"

namespace ckv {

template <int DT, int DH, int WAVES, bool STREAM>
__global__ void __launch_bounds__(WAVES *kWave, WAVES / 4) tree_rows_kernel(TreeArgs a) {
  attend_rows<DT, DH, WAVES, STREAM>(a);
}
template <int DT, int DH, int WAVES, int GROUPS>
__global__ void __launch_bounds__(WAVES *kWave, tile_occupancy(DT, DH, WAVES)) tree_tile_kernel(TreeArgs a) {
  attend_tile<DT, DH, WAVES, GROUPS>(a);
}

template <int DT, int DH, int WAVES>
static void launch_rows_tree(const TreeArgs &a, hipStream_t stream) {
  if (a.col_tiles == 1) hipLaunchKernelGGL((tree_rows_kernel<DT, DH, WAVES, true>), dim3((unsigned)a.workgroups), dim3(WAVES * kWave), 0, stream, a);
  else hipLaunchKernelGGL((tree_rows_kernel<DT, DH, WAVES, false>), dim3((unsigned)a.workgroups), dim3(WAVES * kWave), 0, stream, a);
}
template <int DT, int DH, int WAVES, int GROUPS = 1>
static void launch_tile_tree(const TreeArgs &a, hipStream_t stream) {
  hipLaunchKernelGGL((tree_tile_kernel<DT, DH, WAVES, GROUPS>), dim3((unsigned)a.workgroups), dim3(WAVES * kWave), 0, stream, a);
}
template <int DT, int DH>
static void launch_tree_of(const TreeArgs &a, const PagedPlan &plan, hipStream_t stream) {
  if (plan.by_rows) launch_rows_tree<DT, DH, rows_waves(DT, DH)>(a, stream);
  else if (plan.halves) launch_tile_tree<CKV_BF16, DH, 8, 2>(a, stream);
  else if (plan.tile_cols == 256) launch_tile_tree<DT, DH, 8>(a, stream);
  else launch_tile_tree<DT, DH, 4>(a, stream);
}

void launch_tree(const TreeArgs &a, const PagedPlan &plan, bool bf16, int d, hipStream_t stream) {
  if (bf16 && d == 128) launch_tree_of<CKV_BF16, 128>(a, plan, stream);
  else if (bf16) launch_tree_of<CKV_BF16, 64>(a, plan, stream);
  else if (d == 128) launch_tree_of<CKV_F32, 128>(a, plan, stream);
  else launch_tree_of<CKV_F32, 64>(a, plan, stream);
}

}  // namespace ckv
