// gemm_f16.hip -- the tiled matrix product (gemm.hpp) for operands of type f16.
#include "gemm.hpp"

namespace ar {

int launch_gemm_f16(const GemmArgs& g, bool a_kmajor, bool b_kmajor, bool aligned, int32_t shape, void* stream) {
  return launch_gemm_of<f16>(g, a_kmajor, b_kmajor, aligned, shape, stream);
}

int launch_gemm_pair_f16(const GemmArgs& x, const GemmArgs& w, bool aligned, int32_t shape, void* stream) {
  return launch_pair_of<f16>(x, w, aligned, shape, stream);
}

}  // namespace ar
