// The kernels of limited_kernels.cuh for bf16 logits (a file a type: they take a minute to compile).
#include "limited_kernels.cuh"

namespace gto {

cudaError_t launch_limited_bf16(const LimitedArgs& a, bool tree, int sms, cudaStream_t stream, int64_t* launches) {
  return limited_as<Bf16>(a, tree, sms, stream, launches);
}

}  // namespace gto
