// Dense attention, a warp a row (see dense_rows.cuh), and the kernel that joins the parts of rows whose keys were cut.
#include "common.h"
#include "dense.h"
#include "dense_rows.cuh"

namespace fastar {

template <class T, int D, bool PAGED>
__global__ void __launch_bounds__(128) dense_rows_kernel(const DenseArgs a) {
  chain_wait();
  const int64_t row = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 5);
  if (row >= static_cast<int64_t>(a.T) * a.H) return;
  const int t = static_cast<int>(row / a.H), head = static_cast<int>(row % a.H);
  for (int b = 0; b < a.B; ++b) {
    if (t < a.cu[b] || t >= a.cu[b + 1]) continue;
    DenseSeq s;
    const int r = seq_of(a, b, s);
    if (r < 0 && a.status) record_status(a.status, kErrBounds);
    if (r <= 0) continue;
    dense_row_whole<T, D, PAGED>(a, b, t, head, s, 0);
  }
}

int launch_dense_rows(const DenseArgs& a, int D, bool fp16, cudaStream_t st) {
  const dim3 grid(static_cast<unsigned>((static_cast<int64_t>(a.T) * a.H + 3) / 4));
  void (*kern)(DenseArgs);
  if (a.kc) kern = fp16 ? (D == 128 ? dense_rows_kernel<__half, 128, true> : dense_rows_kernel<__half, 64, true>)
                        : (D == 128 ? dense_rows_kernel<__nv_bfloat16, 128, true> : dense_rows_kernel<__nv_bfloat16, 64, true>);
  else kern = fp16 ? (D == 128 ? dense_rows_kernel<__half, 128, false> : dense_rows_kernel<__half, 64, false>)
                   : (D == 128 ? dense_rows_kernel<__nv_bfloat16, 128, false> : dense_rows_kernel<__nv_bfloat16, 64, false>);
  return launch_chained(kern, grid, 128, 0, st, a) == cudaSuccess ? FASTAR_OK : FASTAR_ERR_CUDA;
}

}  // namespace fastar
