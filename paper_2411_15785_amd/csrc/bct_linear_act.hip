// The matrix-core projections of many token rows with bias, activation, residual and fp32 outputs in their epilogue: the kernel of
// bct_linear_rows.hip with an EpilogueTerm.  It is applied to the fp32 sums where they are written out, so it costs no pass
// over memory of its own.
#include "bct_linear_rows.h"

namespace bct {

hipError_t launch_linear_rows_act(const void* x, const void* w, const void* residual, const LinearOut& dst, uint32_t rows,
                                  uint32_t K, uint32_t N, bool x_tiled, bool out_tiled, hipStream_t s, const EpilogueTerm& term) {
  if (x_tiled) launch_rows<false, true>(x, w, nullptr, residual, dst, rows, K, N, out_tiled, s, term);
  else launch_rows<false, false>(x, w, nullptr, residual, dst, rows, K, N, out_tiled, s, term);
  return hipGetLastError();
}

}  // namespace bct
