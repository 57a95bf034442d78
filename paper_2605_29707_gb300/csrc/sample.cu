// sample.cu -- the filtered draw (sample.cuh) by element type.
#include "kernels.h"

namespace dm {

cudaError_t launch_filtered_draw(const DrawParams& p, int dtype, int rows, cudaStream_t stream) {
  if (rows <= 0 || rows > 0x7fffffff / 8) return cudaErrorInvalidValue;
  if (p.V > kMaxRowVocab) return cudaErrorInvalidValue;
  if (dtype == kF32) return launch_draw_f32(p, rows, stream);
  if (dtype == kBf16) return launch_draw_bf16(p, rows, stream);
  return launch_draw_f16(p, rows, stream);
}

}  // namespace dm
