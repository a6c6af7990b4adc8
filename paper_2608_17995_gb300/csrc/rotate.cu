// rotate.cu — norm and rotation of bf16 heads, and the launch of both types.
#include "rotate.cuh"

namespace avits {

cudaError_t launch_norm_rotate(const RotateCall& call, bool append, int num_sms,
                               unsigned int* status, cudaStream_t s) {
  using namespace rotate;
  Rotate a{};
  a.r = call;
  const int es = call.dt == AVITS_BF16 ? 2 : 4, half = call.rot.rot / 2;
  Cut c{};
  // pieces that halves are whole numbers of, if 32 lanes hold the row, two to a lane
  c.bytes = 16;
  if (!call.rot.interleaved) {
    while (half * es % c.bytes) c.bytes /= 2;
    if (c.bytes < 4 || (es == 4 && c.bytes < 8) || call.d * es / c.bytes > 64) c.bytes = 2;
  }
  c.form = call.rot.interleaved ? kPairs : c.bytes == 2 ? kHalvesAny : kHalves;
  if (c.form == kHalvesAny) c.bytes = 16;
  a.pieces = call.d * es / c.bytes;
  c.lanes = c.bytes < 16 ? 16 : 4;
  while (2 * c.lanes < a.pieces) c.lanes *= 2;
  const int per = 32 / c.lanes;
  a.q_steps = (call.H + per - 1) / per;
  a.k_steps = (call.Hkv + per - 1) / per;
  a.steps = a.q_steps + a.k_steps * (append ? 2 : 1);
  a.inv_d = 1.f / (float)call.d;
  // a warp for each token, or several where tokens are too few to fill the SMs
  a.parts = 1;
  while (a.parts < a.steps && (long long)call.tokens * a.parts < 32ll * num_sms) a.parts *= 2;
  if (a.parts > a.steps) a.parts = a.steps;
  a.first[0] = 0;
  for (int x = 1; x < 4; ++x)
    a.first[x] = x < call.rot.axes ? a.first[x - 1] + call.rot.sections[x - 1] : 1 << 30;
  a.seq = FastDiv::of(call.N);
  a.part = FastDiv::of(a.parts);
  a.page = FastDiv::of(append ? call.cache.page_size : 1);
  a.status = status;
  const long long units = (long long)call.tokens * a.parts;
  c.grid = (int)((units + kRotWarps - 1) / kRotWarps);
  return call.dt == AVITS_BF16 ? launch_type<__nv_bfloat16>(a, append, c, s)
                               : launch_f32(a, append, c, s);
}

}  // namespace avits
