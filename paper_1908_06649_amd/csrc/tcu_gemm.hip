// The blocked product of Theorem 2 and Corollary 1: instances of the kernels of
// tcu_gemm_tiles.h for every input and output type.
#include "tcu_gemm_tiles.h"

namespace tcu {

hipError_t launch_rect(int dtype, int s, const RectArgs &a, hipStream_t stream, int num_cus) {
  // A single contiguous strip times a single block is one native call.
  if (a.K == s && a.N == s && a.lda == s && a.ldb == s && a.ldc == s)
    return launch_tall(dtype, s, a.A, a.M, a.B, a.C, a.accum, stream, num_cus);
  switch (dtype) {
    case TCU_F16_F32: return launch_dt<TCU_F16_F32>(a, stream, num_cus);
    case TCU_BF16_F32: return launch_dt<TCU_BF16_F32>(a, stream, num_cus);
    case TCU_BF16_BF16: return launch_dt<TCU_BF16_BF16>(a, stream, num_cus);
    case TCU_I8_I32: return launch_dt<TCU_I8_I32>(a, stream, num_cus);
  }
  return hipErrorInvalidValue;
}

}  // namespace tcu
