// sample_f16.cu -- the filtered draw on f16 logits.
#include "sample.cuh"

namespace dm {

cudaError_t launch_draw_f16(const DrawParams& p, int rows, cudaStream_t stream) {
  return launch_draw_type<__half>(p, rows, stream);
}

}  // namespace dm
