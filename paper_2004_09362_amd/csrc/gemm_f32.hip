// gemm_f32.hip -- the tiled matrix product (gemm.hpp) for operands of type float.
#include "gemm.hpp"

namespace ar {

int launch_gemm_f32(const GemmArgs& g, bool a_kmajor, bool b_kmajor, bool aligned, int32_t shape, void* stream) {
  return launch_gemm_of<float>(g, a_kmajor, b_kmajor, aligned, shape, stream);
}

int launch_gemm_pair_f32(const GemmArgs& x, const GemmArgs& w, bool aligned, int32_t shape, void* stream) {
  return launch_pair_of<float>(x, w, aligned, shape, stream);
}

}  // namespace ar
