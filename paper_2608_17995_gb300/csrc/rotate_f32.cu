// rotate_f32.cu — norm and rotation of fp32 heads.
#include "rotate.cuh"

namespace avits {
namespace rotate {

cudaError_t launch_f32(const Rotate& a, int form, bool append, int lanes, int grid,
                       cudaStream_t s) {
  return launch_type<float>(a, form, append, lanes, grid, s);
}

}  // namespace rotate
}  // namespace avits
