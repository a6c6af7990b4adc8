// rotate.cu — norm and rotation of bf16 heads, and the launch of both types.
#include "rotate.cuh"

#include <climits>

namespace avits {

namespace {

// Warps of a token: the fewest rounds of warps, each as long as its steps and about three more
// for the angles.  Tokens of 48 bf16 heads of 128, us with 1, 2, 4, .. warps: 512 of them 5.6
// with 4, 7.0 with 8, 7.6 with 12; 2048 13.8, 14.9, 15.9, 20.2; 4096 25.0, 23.9, 28.6; 8192 41.9, 42.9.
// 1554 of 20 fp32 heads of 80 9.0, 7.6, 7.7, 9.1.
constexpr int kAnglesSteps = 3;
constexpr int kWarpsBf16 = 20, kWarpsF32 = 32;      // on an SM at once, by registers

int parts_of(const rotate::Rotate& a, int es, int num_sms) {
  const long long once = (long long)num_sms * (es == 2 ? kWarpsBf16 : kWarpsF32);
  long long least = LLONG_MAX;
  int best = 1;
  for (int n = 1;; n = 2 * n < a.steps ? 2 * n : a.steps) {
    const long long rounds = (a.r.tokens * (long long)n + once - 1) / once;
    const long long cost = rounds * (kAnglesSteps + (a.steps + n - 1) / n);
    if (cost < least) {
      least = cost;
      best = n;
    }
    if (n >= a.steps) return best;
  }
}

}  // namespace

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
  a.parts = parts_of(a, es, num_sms);
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
