// The kernels of limited_kernels.cuh for f16 logits (a file a type: they take a minute to compile).
#include "limited_kernels.cuh"

namespace gto {

cudaError_t launch_limited_f16(const LimitedArgs& a, bool tree, int sms, cudaStream_t stream, int64_t* launches) {
  return limited_as<F16>(a, tree, sms, stream, launches);
}

}  // namespace gto
