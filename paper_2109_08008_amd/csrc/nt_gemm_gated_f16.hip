// Gated projections on the tiles of nt_gemm_phased.h for one element type (a unit each, to build in
// parallel).
#include "nt_gemm_phased.h"

namespace nt {

hipError_t gemm_gated_f16(const void* A, int lda, const void* Bt, int M, int N, int K, const GemmEpi& epi, hipStream_t s,
                      int bm) {
  return epi.lnf_colsum ? launch_gated<f16, true>(A, lda, Bt, M, N, K, epi, s, bm)
                        : launch_gated<f16, false>(A, lda, Bt, M, N, K, epi, s, bm);
}

}  // namespace nt
