// peri_norm_f32.cu -- the Peri-LN kernels for an fp32 stream and fp32 branches.
#include "peri_norm_forward.cuh"
#include "peri_norm_backward.cuh"

namespace mtdao {
template cudaError_t launch_peri_forward<float, float>(const NormArgs &, bool, cudaStream_t);
template cudaError_t launch_peri_backward<float, float>(const NormArgs &, bool, cudaStream_t);
}  // namespace mtdao
