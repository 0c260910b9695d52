// peri_norm_mixed.cu -- the Peri-LN kernels for an fp32 stream and bf16 branches.
#include "peri_norm_forward.cuh"
#include "peri_norm_backward.cuh"

namespace mtdao {
template cudaError_t launch_peri_forward<float, Bf16>(const NormArgs &, bool, cudaStream_t);
template cudaError_t launch_peri_backward<float, Bf16>(const NormArgs &, bool, cudaStream_t);
}  // namespace mtdao
