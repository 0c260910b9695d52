// peri_norm_bf16.cu -- the Peri-LN kernels for bf16 throughout.
#include "peri_norm_forward.cuh"
#include "peri_norm_backward.cuh"

namespace mtdao {
template cudaError_t launch_peri_forward<Bf16, Bf16>(const NormArgs &, bool, cudaStream_t);
template cudaError_t launch_peri_backward<Bf16, Bf16>(const NormArgs &, bool, cudaStream_t);
}  // namespace mtdao
