// The layer norm's kernels for rows that start anywhere.
#include "layernorm_forward.cuh"

namespace prm {

int layernorm_shifted(const LayerNormArgs& a, const __nv_bfloat16*, cudaStream_t stream) {
  return a.drop.threshold ? run_layernorm<__nv_bfloat16, true, true>(a, stream) : run_layernorm<__nv_bfloat16, false, true>(a, stream);
}
int layernorm_shifted(const LayerNormArgs& a, const float*, cudaStream_t stream) {
  return a.drop.threshold ? run_layernorm<float, true, true>(a, stream) : run_layernorm<float, false, true>(a, stream);
}

}  // namespace prm
