// sample_bf16.cu -- the filtered draw on bf16 logits.
#include "sample.cuh"

namespace dm {

cudaError_t launch_draw_bf16(const DrawParams& p, int rows, cudaStream_t stream) {
  return launch_draw_type<__nv_bfloat16>(p, rows, stream);
}

}  // namespace dm
