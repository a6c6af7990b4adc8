// rotate_f32.cu — norm and rotation of fp32 heads.
#include "rotate.cuh"

namespace avits {
namespace rotate {

cudaError_t launch_f32(const Rotate& a, bool append, const Cut& c, cudaStream_t s) {
  return launch_type<float>(a, append, c, s);
}

}  // namespace rotate
}  // namespace avits
