// rotate.cu — norm and rotation of bf16 heads, and the launch of both types.
#include "rotate.cuh"

namespace avits {

cudaError_t launch_norm_rotate(const RotateCall& call, bool append, int num_sms,
                               unsigned int* status, cudaStream_t s) {
  using namespace rotate;
  Rotate a{};
  a.r = call;
  const int E = call.dt == AVITS_BF16 ? 8 : 4;
  a.pieces = call.d / E;
  const int half = call.rot.rot / 2;
  const int form = call.rot.interleaved ? kPairs : half % E == 0 ? kHalves : kHalvesAny;
  int lanes = 4;                   // of a row: two pieces each
  while (2 * lanes < a.pieces) lanes *= 2;
  const int per = 32 / lanes;
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
  const int grid = (int)((units + kRotWarps - 1) / kRotWarps);
  return call.dt == AVITS_BF16 ? launch_type<__nv_bfloat16>(a, form, append, lanes, grid, s)
                               : launch_f32(a, form, append, lanes, grid, s);
}

}  // namespace avits
