// The tiles of products of e5m2 (A) and e5m2 (B)
#include "gemm_fp8_kernels.h"

namespace als {
template int gemm_fp8_launch<1, 1>(Fp8Args, int, Fp8Out, hipStream_t);
}
