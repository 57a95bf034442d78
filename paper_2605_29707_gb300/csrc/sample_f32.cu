// sample_f32.cu -- the filtered draw on f32 logits.
#include "sample.cuh"

namespace dm {

cudaError_t launch_draw_f32(const DrawParams& p, int rows, cudaStream_t stream) {
  return launch_draw_type<float>(p, rows, stream);
}

}  // namespace dm
