// api.cu — the C ABI of libavits (see include/avits.h): host-side argument
// checks, workspace sizing and dispatch to the kernels.  Nothing here
// allocates device memory or synchronises, except avits_device_status().
#include <algorithm>
#include <climits>
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <string>

#include "avits_common.cuh"
#include "avits_internal.h"

namespace avits {

__device__ unsigned int g_status = 0u;

namespace {

thread_local std::string t_last_error;

constexpr int kMaxDevices = 64;
unsigned int* g_status_ptr[kMaxDevices] = {};

int num_sms_current() {
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return 0;
  if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
  return n;
}

avits_status cuda_status(cudaError_t e) {
  if (e == cudaSuccess) return AVITS_OK;
  t_last_error = cudaGetErrorString(e);
  cudaGetLastError();   // clear a non-sticky error
  return AVITS_ERR_CUDA;
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool valid_dtype(avits_dtype dt) { return dt == AVITS_F32 || dt == AVITS_BF16; }

// A mixed input in bilinear mode needs the cell map of its frame: an even
// frame, token indices that fit the map entry, and the workspace.
bool mixed_bilinear_ok(avits_upmode mode, const int32_t* pos_in, int B, int M, int gh, int gw,
                       const void* ws, size_t ws_bytes) {
  if (mode != AVITS_UP_BILINEAR || !pos_in) return true;
  if ((gh & 1) || (gw & 1) || M > (1 << 28) - 1) return false;
  return ws && aligned16(ws) && ws_bytes >= merge_workspace_bytes(B, gh, gw);
}

// Whether the rows of `width` elements that a view of up to 3 axes has (extents n,
// strides st >= 0) lie apart.  Views of a dense tensor nest: each stride passes all
// that the smaller ones reach.  Others are searched for two rows that meet: over the
// differences of the two shorter axes' indexes, the third's is then given; where
// those are more than 2^22 the view counts as one whose rows meet.
struct Axis {
  int64_t n, st;
};
bool rows_apart(int64_t width, Axis a, Axis b, Axis c = {1, 0}) {
  Axis ax[3] = {a, b, c};
  for (Axis& x : ax)
    if (x.n == 1) x.st = 0;
  std::sort(ax, ax + 3, [](const Axis& x, const Axis& y) { return x.st < y.st; });
  __int128 reach = width;
  bool nested = true;
  for (const Axis& x : ax) {
    if (x.n == 1) continue;
    nested = nested && x.st >= reach;
    reach += (__int128)(x.n - 1) * x.st;
  }
  if (nested) return true;
  std::sort(ax, ax + 3, [](const Axis& x, const Axis& y) { return x.n < y.n; });
  if (ax[0].n * ax[1].n > (1 << 22)) return false;
  const __int128 st = ax[2].st;
  for (int64_t i = 0; i < ax[0].n; ++i)
    for (int64_t j = 1 - ax[1].n; j < ax[1].n; ++j) {
      const __int128 off = (__int128)i * ax[0].st + (__int128)j * ax[1].st;
      const bool same = i == 0 && j == 0;          // the two rows differ in the third axis alone
      if (st == 0) {
        if (off < width && off > -width && (!same || ax[2].n > 1)) return false;
        continue;
      }
      const __int128 k0 = off / st;                // the nearest differences
      for (__int128 k = k0 - 1; k <= k0 + 1; ++k) {
        const __int128 d = off - k * st;
        if (k > -ax[2].n && k < ax[2].n && !(same && k == 0) && d < width && d > -width) return false;
      }
    }
  return true;
}
// What is written may not lie over itself: the rows of weights, of the pages.
bool weights_apart(const avits_kv_cache& c) {
  return rows_apart(c.max_len, {c.B, c.acc_sb}, {c.Hkv, c.acc_sh});
}
bool pages_apart(const avits_kv_cache& c) {
  return rows_apart(c.d, {c.num_pages, c.k_sp}, {c.page_size, c.k_st}, {c.Hkv, c.k_sh}) &&
         rows_apart(c.d, {c.num_pages, c.v_sp}, {c.page_size, c.v_st}, {c.Hkv, c.v_sh});
}

// A cache's description: INVALID_ARG for what cannot be one, UNSUPPORTED for a
// layout that the kernels' 16-byte accesses do not take.
avits_status check_cache(const avits_kv_cache* c) {
  if (!c || !c->k_pages || !c->v_pages || !c->block_table || !c->lens) return AVITS_ERR_INVALID_ARG;
  if (c->dt != AVITS_F32 && c->dt != AVITS_BF16) return AVITS_ERR_INVALID_ARG;
  if (c->B <= 0 || c->Hkv <= 0 || c->d <= 0 || c->num_pages <= 0 || c->page_size <= 0 ||
      c->max_len <= 0)
    return AVITS_ERR_INVALID_ARG;
  if (c->k_sp < 0 || c->k_st < 0 || c->k_sh < 0 || c->v_sp < 0 || c->v_st < 0 || c->v_sh < 0)
    return AVITS_ERR_INVALID_ARG;
  if (c->table_sb < 0) return AVITS_ERR_INVALID_ARG;
  if (c->acc && (c->acc_sb < 0 || c->acc_sh < 0 || (c->Hkv > 1 && c->acc_sh < c->max_len) ||
                 (c->B > 1 && c->acc_sb < c->max_len)))
    return AVITS_ERR_INVALID_ARG;
  const int per16 = c->dt == AVITS_BF16 ? 8 : 4;
  if (c->d > 256 || c->d % per16) return AVITS_ERR_UNSUPPORTED;
  if (c->max_len > (1 << 30) || c->page_size > (1 << 30) || c->B > (1 << 24) ||
      c->Hkv > (1 << 16) || (int64_t)c->B * c->Hkv > (1 << 26))
    return AVITS_ERR_UNSUPPORTED;
  if (!aligned16(c->k_pages) || !aligned16(c->v_pages)) return AVITS_ERR_UNSUPPORTED;
  for (int64_t st : {c->k_sp, c->k_st, c->k_sh, c->v_sp, c->v_st, c->v_sh})
    if (st % per16) return AVITS_ERR_UNSUPPORTED;
  return AVITS_OK;
}

bool rotary_ok(const avits_rotary* r, int d, const void* positions) {
  if (!r || r->rot < 0 || r->rot % 2 || r->rot > d) return false;
  if (r->rot == 0) return true;
  if (!r->freq || !positions || r->axes < 1 || r->axes > 4 || !(std::fabs(r->magnitude) < 3.0e38f))
    return false;
  int64_t pairs = 0;
  for (int i = 0; i < r->axes; ++i) {
    if (r->sections[i] < 0) return false;
    pairs += r->sections[i];
  }
  return pairs == r->rot / 2;
}
bool norm_ok(int norm, const void* q_weight, const void* k_weight, float eps) {
  return norm ? eps >= 0.f && eps < 3.0e38f : !q_weight && !k_weight;
}
bool same_strides(const int64_t* a, const int64_t* b, int64_t n0, int64_t n1, int64_t n2) {
  return (n0 == 1 || a[0] == b[0]) && (n1 == 1 || a[1] == b[1]) && (n2 == 1 || a[2] == b[2]);
}

// Arguments one after the other, 8 bytes each.
struct Packed {
  const char* at;
  bool ok = true;
  int64_t i64() {
    int64_t x;
    std::memcpy(&x, at, 8);
    at += 8;
    return x;
  }
  int i32() {
    const int64_t x = i64();
    ok = ok && x >= INT32_MIN && x <= INT32_MAX;
    return (int)x;
  }
  float f32() {
    double x;
    std::memcpy(&x, at, 8);
    at += 8;
    return (float)x;
  }
  template <typename T>
  T* ptr() { return reinterpret_cast<T*>((uintptr_t)i64()); }
};

}  // namespace

// The device address of g_status on the current device, looked up once per
// device.  Concurrent first calls store the same value.
unsigned int* status_word() {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return nullptr;
  unsigned int* p = __atomic_load_n(&g_status_ptr[dev], __ATOMIC_ACQUIRE);
  if (!p) {
    void* q = nullptr;
    if (cudaGetSymbolAddress(&q, g_status) != cudaSuccess) {
      cudaGetLastError();
      return nullptr;
    }
    p = static_cast<unsigned int*>(q);
    __atomic_store_n(&g_status_ptr[dev], p, __ATOMIC_RELEASE);
  }
  return p;
}

}  // namespace avits

using namespace avits;

extern "C" {

const char* avits_version(void) { return "0.1.0"; }

const char* avits_status_string(avits_status s) {
  switch (s) {
    case AVITS_OK: return "ok";
    case AVITS_ERR_INVALID_ARG: return "invalid argument";
    case AVITS_ERR_UNSUPPORTED: return "unsupported combination";
    case AVITS_ERR_CUDA: return "CUDA error";
    case AVITS_ERR_TIMEOUT: return "device wait timed out";
    case AVITS_ERR_NAN: return "NaN in fused score";
    case AVITS_ERR_COVERAGE: return "mixed sequence does not tile the frame";
    case AVITS_ERR_PAGE: return "cache length or page number out of range";
  }
  return "unknown status";
}

const char* avits_last_error_string(void) { return t_last_error.c_str(); }

size_t avits_score_spatial_workspace(avits_dtype dt, int B, int H, int M, int Nk, int d) {
  if (B <= 0 || H <= 0 || M <= 0 || Nk <= 0 || d <= 0) return 0;
  if (dt != AVITS_BF16 || (d != 64 && d != 128)) return 0;
  return spatial_tc_workspace(B, H, M, Nk, d, num_sms_current());
}

avits_status avits_score_spatial(const void* q_img, const void* k_all, avits_dtype dt, int B,
                                 int H, int M, int Nk, int L, int d, int64_t q_sb, int64_t q_sh,
                                 int64_t q_sn, int64_t k_sb, int64_t k_sh, int64_t k_sn,
                                 float softmax_scale, float weight, int accumulate, float* A,
                                 float* lse_opt, void* workspace, size_t ws_bytes, void* stream) {
  AVITS_RANGE();
  if (!q_img || !k_all || !A || !valid_dtype(dt)) return AVITS_ERR_INVALID_ARG;
  if (B <= 0 || H <= 0 || M <= 0 || Nk <= 0 || d <= 0 || L < 0 || L > Nk || Nk < M)
    return AVITS_ERR_INVALID_ARG;
  if (!(softmax_scale > 0.f) || !(softmax_scale < 3.0e38f)) return AVITS_ERR_INVALID_ARG;
  if (q_sn < d || k_sn < d || q_sh < 0 || k_sh < 0 || q_sb < 0 || k_sb < 0)
    return AVITS_ERR_INVALID_ARG;
  SpatialArgs a{q_img, k_all, dt, B, H, M, Nk, L, d, q_sb, q_sh, q_sn, k_sb, k_sh, k_sn,
                softmax_scale, weight, accumulate ? 1 : 0, A, lse_opt, workspace, ws_bytes,
                status_word()};
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (spatial_tc_eligible(a)) {
    const int sms = num_sms_current();
    if (ws_bytes < spatial_tc_workspace(B, H, M, Nk, d, sms) || !workspace)
      return AVITS_ERR_INVALID_ARG;
    return cuda_status(launch_spatial_tc(a, sms, s));
  }
  if (d > 256) return AVITS_ERR_UNSUPPORTED;
  return cuda_status(launch_spatial_simt(a, num_sms_current(), s));
}

avits_status avits_score_spatial_lse(const void* q_img, const void* k_txt, avits_dtype dt, int B,
                                     int H, int M, int L, int d, int64_t q_sb, int64_t q_sh,
                                     int64_t q_sn, int64_t k_sb, int64_t k_sh, int64_t k_sn,
                                     const float* lse_all, float softmax_scale, float weight,
                                     int accumulate, float* A, float* lse_opt, void* workspace,
                                     size_t ws_bytes, void* stream) {
  AVITS_RANGE();
  if (!q_img || !k_txt || !lse_all || !A || !valid_dtype(dt)) return AVITS_ERR_INVALID_ARG;
  if (B <= 0 || H <= 0 || M <= 0 || L <= 0 || d <= 0) return AVITS_ERR_INVALID_ARG;
  if (!(softmax_scale > 0.f) || !(softmax_scale < 3.0e38f)) return AVITS_ERR_INVALID_ARG;
  if (q_sn < d || k_sn < d || q_sh < 0 || k_sh < 0 || q_sb < 0 || k_sb < 0)
    return AVITS_ERR_INVALID_ARG;
  SpatialArgs a{q_img, k_txt, dt, B, H, M, L, L, d, q_sb, q_sh, q_sn, k_sb, k_sh, k_sn,
                softmax_scale, weight, accumulate ? 1 : 0, A, lse_opt, workspace, ws_bytes,
                status_word()};
  a.lse_all = lse_all;
  if (!spatial_tc_eligible(a)) return AVITS_ERR_UNSUPPORTED;
  const int sms = num_sms_current();
  if (ws_bytes < spatial_tc_workspace(B, H, M, L, d, sms) || !workspace)
    return AVITS_ERR_INVALID_ARG;
  return cuda_status(launch_spatial_tc(a, sms, static_cast<cudaStream_t>(stream)));
}

avits_status avits_score_spatial_keymask(const void* q_img, const void* k_all, avits_dtype dt,
                                         int B, int H, int M, int Nk, int d, int64_t q_sb,
                                         int64_t q_sh, int64_t q_sn, int64_t k_sb, int64_t k_sh,
                                         int64_t k_sn, const uint8_t* text_mask,
                                         float softmax_scale, float weight, int accumulate,
                                         float* A, float* lse_opt, void* workspace,
                                         size_t ws_bytes, void* stream) {
  AVITS_RANGE();
  if (!q_img || !k_all || !A || !text_mask || !valid_dtype(dt)) return AVITS_ERR_INVALID_ARG;
  if (B <= 0 || H <= 0 || M <= 0 || Nk <= 0 || d <= 0 || Nk < M) return AVITS_ERR_INVALID_ARG;
  if (!(softmax_scale > 0.f) || !(softmax_scale < 3.0e38f)) return AVITS_ERR_INVALID_ARG;
  if (q_sn < d || k_sn < d || q_sh < 0 || k_sh < 0 || q_sb < 0 || k_sb < 0)
    return AVITS_ERR_INVALID_ARG;
  SpatialArgs a{q_img, k_all, dt, B, H, M, Nk, 0, d, q_sb, q_sh, q_sn, k_sb, k_sh, k_sn,
                softmax_scale, weight, accumulate ? 1 : 0, A, lse_opt, workspace, ws_bytes,
                status_word(), text_mask};
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (spatial_tc_eligible(a)) {
    const int sms = num_sms_current();
    if (ws_bytes < spatial_tc_workspace(B, H, M, Nk, d, sms) || !workspace)
      return AVITS_ERR_INVALID_ARG;
    return cuda_status(launch_spatial_tc(a, sms, s));
  }
  if (d > 256) return AVITS_ERR_UNSUPPORTED;
  return cuda_status(launch_spatial_simt(a, num_sms_current(), s));
}

size_t avits_attention_forward_workspace(int B, int H, int Mq) {
  if (B <= 0 || H <= 0 || Mq <= 0) return 0;
  return attention_tc_workspace(B, H, Mq);
}

avits_status avits_attention_forward(const void* q, const void* k, const void* v, avits_dtype dt,
                                     int B, int H, int Mq, int Nk, int L, int d,
                                     const int64_t* q_str, const int64_t* k_str,
                                     const int64_t* v_str, const int64_t* o_str,
                                     float softmax_scale, void* o, float* lse_opt, float weight,
                                     int accumulate, float* A, void* workspace, size_t ws_bytes,
                                     void* stream) {
  AVITS_RANGE();
  if (!q || !k || !v || !o || !valid_dtype(dt)) return AVITS_ERR_INVALID_ARG;
  if (B <= 0 || H <= 0 || Mq <= 0 || Nk <= 0 || d <= 0 || L < 0 || L > Nk)
    return AVITS_ERR_INVALID_ARG;
  if (!(softmax_scale > 0.f) || !(softmax_scale < 3.0e38f)) return AVITS_ERR_INVALID_ARG;
  AttnArgs a{};
  a.q = q; a.k = k; a.v = v; a.o = o;
  a.B = B; a.H = H; a.Mq = Mq; a.Nk = Nk; a.L = L; a.d = d;
  const int64_t* given[4] = {q_str, k_str, v_str, o_str};
  for (int i = 0; i < 4; ++i) {
    const int64_t rows = (i == 1 || i == 2) ? Nk : Mq;
    if (given[i]) {
      for (int j = 0; j < 3; ++j) a.str[i][j] = given[i][j];
      if (a.str[i][2] < d || a.str[i][1] < 0 || a.str[i][0] < 0) return AVITS_ERR_INVALID_ARG;
    } else {
      a.str[i][2] = d;
      a.str[i][1] = rows * d;
      a.str[i][0] = (int64_t)H * rows * d;
    }
  }
  a.scale = softmax_scale;
  a.weight = weight;
  a.accumulate = accumulate ? 1 : 0;
  a.A = A;
  a.lse = lse_opt;
  a.ws = workspace;
  a.status = status_word();
  if (A && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 7u) ||
            ws_bytes < attention_tc_workspace(B, H, Mq)))
    return AVITS_ERR_INVALID_ARG;
  if (dt != AVITS_BF16) return AVITS_ERR_UNSUPPORTED;
  if (A && H > 255) return AVITS_ERR_UNSUPPORTED;   // the head count of the fixed-point sum
  if ((long long)B * H * ((Mq + 255) / 256) >= (1ll << 31)) return AVITS_ERR_UNSUPPORTED;
  if (!attention_tc_layout_ok(a)) return AVITS_ERR_UNSUPPORTED;
  return cuda_status(launch_attention_tc(a, num_sms_current(), static_cast<cudaStream_t>(stream)));
}

avits_status avits_score_temporal(const void* h_t, const void* h_prev, avits_dtype dt, int B,
                                  int N, int D, float eps, float* V, void* stream) {
  AVITS_RANGE();
  if (!h_t || !h_prev || !V || !valid_dtype(dt)) return AVITS_ERR_INVALID_ARG;
  if (B <= 0 || N <= 0 || D <= 0 || !(eps >= 0.f)) return AVITS_ERR_INVALID_ARG;
  return cuda_status(launch_temporal(h_t, h_prev, dt, B, N, D, eps, V, num_sms_current(),
                                     status_word(), static_cast<cudaStream_t>(stream)));
}

avits_status avits_score_spatiotemporal(const void* q_img, const void* k_all, avits_dtype dt,
                                        int B, int H, int M, int Nk, int L, int d, int64_t q_sb,
                                        int64_t q_sh, int64_t q_sn, int64_t k_sb, int64_t k_sh,
                                        int64_t k_sn, float softmax_scale, float weight,
                                        int accumulate, float* A, float* lse_opt, void* workspace,
                                        size_t ws_bytes, const void* h_t, const void* h_prev,
                                        int D, float eps, float* V, void* stream) {
  AVITS_RANGE();
  if (!q_img || !k_all || !A || !h_t || !h_prev || !V || !valid_dtype(dt))
    return AVITS_ERR_INVALID_ARG;
  if (B <= 0 || H <= 0 || M <= 0 || Nk <= 0 || d <= 0 || L < 0 || L > Nk || Nk < M || D <= 0)
    return AVITS_ERR_INVALID_ARG;
  if (!(softmax_scale > 0.f) || !(softmax_scale < 3.0e38f) || !(eps >= 0.f))
    return AVITS_ERR_INVALID_ARG;
  if (q_sn < d || k_sn < d || q_sh < 0 || k_sh < 0 || q_sb < 0 || k_sb < 0)
    return AVITS_ERR_INVALID_ARG;
  SpatialArgs a{q_img, k_all, dt, B, H, M, Nk, L, d, q_sb, q_sh, q_sn, k_sb, k_sh, k_sn,
                softmax_scale, weight, accumulate ? 1 : 0, A, lse_opt, workspace, ws_bytes,
                status_word()};
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const int sms = num_sms_current();
  if (spatial_tc_eligible(a)) {
    if (ws_bytes < spatial_tc_workspace(B, H, M, Nk, d, sms) || !workspace)
      return AVITS_ERR_INVALID_ARG;
    unsigned int* st = a.status;
    const float beside_us = spatial_tc_estimate_us(B, H, M, Nk, d, sms);
    const LaunchHook temporal = [=](cudaStream_t ss) {
      return launch_temporal_overlapped(h_t, h_prev, dt, B, M, D, eps, V, sms, st, beside_us, ss);
    };
    return cuda_status(launch_spatial_tc(a, sms, s, &temporal));
  }
  if (d > 256) return AVITS_ERR_UNSUPPORTED;
  cudaError_t e = launch_spatial_simt(a, num_sms_current(), s);
  if (e == cudaSuccess) e = launch_temporal(h_t, h_prev, dt, B, M, D, eps, V, sms, a.status, s);
  return cuda_status(e);
}

avits_status avits_score_temporal_var(const void* const* snaps, int n_t, avits_dtype dt, int B,
                                      int N, int D, float* V, void* stream) {
  AVITS_RANGE();
  if (!snaps || !V || !valid_dtype(dt)) return AVITS_ERR_INVALID_ARG;
  if (n_t < 2 || n_t > kMaxSnapshots || B <= 0 || N <= 0 || D <= 0) return AVITS_ERR_INVALID_ARG;
  for (int i = 0; i < n_t; ++i)
    if (!snaps[i]) return AVITS_ERR_INVALID_ARG;
  return cuda_status(launch_temporal_var(snaps, n_t, dt, B, N, D, V, num_sms_current(),
                                         static_cast<cudaStream_t>(stream)));
}

avits_status avits_fuse_select(const float* A, const float* V, int B, int M, float alpha,
                               float eps_norm, int k, float* S_opt, int32_t* sel_idx,
                               uint8_t* sel_mask_opt, int32_t* tok_offset, void* stream) {
  AVITS_RANGE();
  return avits_fuse_select_perturbed(A, V, nullptr, B, M, alpha, eps_norm, k, S_opt, sel_idx,
                                     sel_mask_opt, tok_offset, stream);
}

avits_status avits_fuse_select_perturbed(const float* A, const float* V, const float* perturb,
                                         int B, int M, float alpha, float eps_norm, int k,
                                         float* S_opt, int32_t* sel_idx, uint8_t* sel_mask_opt,
                                         int32_t* tok_offset, void* stream) {
  AVITS_RANGE();
  if (!A || !V || !tok_offset || (k > 0 && !sel_idx)) return AVITS_ERR_INVALID_ARG;
  if (B <= 0 || M <= 0 || M > kSelectMaxM || k < 0 || k > M) return AVITS_ERR_INVALID_ARG;
  if (!(alpha >= 0.f && alpha <= 1.f) || !(eps_norm >= 0.f)) return AVITS_ERR_INVALID_ARG;
  return cuda_status(launch_fuse_select(A, V, perturb, B, M, alpha, eps_norm, k, S_opt, sel_idx,
                                        sel_mask_opt, tok_offset, status_word(),
                                        static_cast<cudaStream_t>(stream)));
}

avits_status avits_selective_upsample(const void* latent, avits_dtype dt, int B, int M,
                                      int grid_h, int grid_w, int C, int p,
                                      const int32_t* pos_in_opt, const int32_t* span_in_opt,
                                      const uint8_t* sel_mask, const int32_t* tok_offset, int k,
                                      avits_upmode mode, void* out_latent, int32_t* out_pos,
                                      int32_t* out_span, int32_t* out_src_tok,
                                      int8_t* out_src_sub, void* workspace, size_t ws_bytes,
                                      void* stream) {
  AVITS_RANGE();
  if (!latent || !sel_mask || !tok_offset || !out_latent || !out_pos || !out_span ||
      !out_src_tok || !out_src_sub || !valid_dtype(dt))
    return AVITS_ERR_INVALID_ARG;
  if (B <= 0 || M <= 0 || grid_h <= 0 || grid_w <= 0 || C <= 0 || k < 0 || k > M)
    return AVITS_ERR_INVALID_ARG;
  if (p != 2) return AVITS_ERR_UNSUPPORTED;
  if ((pos_in_opt == nullptr) != (span_in_opt == nullptr)) return AVITS_ERR_INVALID_ARG;
  if (!pos_in_opt && (int64_t)grid_h * grid_w != M) return AVITS_ERR_INVALID_ARG;
  if (mode != AVITS_UP_NEAREST && mode != AVITS_UP_BILINEAR) return AVITS_ERR_INVALID_ARG;
  if (!aligned16(latent) || !aligned16(out_latent)) return AVITS_ERR_INVALID_ARG;
  if (!mixed_bilinear_ok(mode, pos_in_opt, B, M, grid_h, grid_w, workspace, ws_bytes))
    return AVITS_ERR_INVALID_ARG;
  return cuda_status(launch_upsample(latent, dt, B, M, grid_h, grid_w, C, pos_in_opt, span_in_opt,
                                     sel_mask, tok_offset, k, mode, out_latent, out_pos, out_span,
                                     out_src_tok, out_src_sub, workspace, status_word(),
                                     static_cast<cudaStream_t>(stream)));
}

size_t avits_selective_upsample_workspace(avits_upmode mode, int B, int grid_h, int grid_w) {
  if (mode != AVITS_UP_BILINEAR || B <= 0 || grid_h <= 0 || grid_w <= 0) return 0;
  return merge_workspace_bytes(B, grid_h, grid_w);
}

avits_status avits_select_upsample(const float* A, const float* V, const float* perturb, int B,
                                   int M, float alpha, float eps_norm, int k, float* S_opt,
                                   int32_t* sel_idx, uint8_t* sel_mask, int32_t* tok_offset,
                                   const void* latent, avits_dtype dt, int grid_h, int grid_w,
                                   int C, int p, const int32_t* pos_in_opt,
                                   const int32_t* span_in_opt, avits_upmode mode,
                                   void* out_latent, int32_t* out_pos, int32_t* out_span,
                                   int32_t* out_src_tok, int8_t* out_src_sub, void* workspace,
                                   size_t ws_bytes, void* stream) {
  AVITS_RANGE();
  if (!A || !V || !tok_offset || !sel_mask || (k > 0 && !sel_idx)) return AVITS_ERR_INVALID_ARG;
  if (B <= 0 || M <= 0 || M > kSelectMaxM || k < 0 || k > M) return AVITS_ERR_INVALID_ARG;
  if (!(alpha >= 0.f && alpha <= 1.f) || !(eps_norm >= 0.f)) return AVITS_ERR_INVALID_ARG;
  if (!latent || !out_latent || !out_pos || !out_span || !out_src_tok || !out_src_sub ||
      !valid_dtype(dt))
    return AVITS_ERR_INVALID_ARG;
  if (grid_h <= 0 || grid_w <= 0 || C <= 0) return AVITS_ERR_INVALID_ARG;
  if (p != 2) return AVITS_ERR_UNSUPPORTED;
  if ((pos_in_opt == nullptr) != (span_in_opt == nullptr)) return AVITS_ERR_INVALID_ARG;
  if (!pos_in_opt && (int64_t)grid_h * grid_w != M) return AVITS_ERR_INVALID_ARG;
  if (mode != AVITS_UP_NEAREST && mode != AVITS_UP_BILINEAR) return AVITS_ERR_INVALID_ARG;
  if (!aligned16(latent) || !aligned16(out_latent)) return AVITS_ERR_INVALID_ARG;
  if (!mixed_bilinear_ok(mode, pos_in_opt, B, M, grid_h, grid_w, workspace, ws_bytes))
    return AVITS_ERR_INVALID_ARG;
  return cuda_status(launch_select_upsample(
      A, V, perturb, B, M, alpha, eps_norm, k, S_opt, sel_idx, sel_mask, tok_offset,
      status_word(), latent, dt, grid_h, grid_w, C, pos_in_opt, span_in_opt, mode, out_latent,
      out_pos, out_span, out_src_tok, out_src_sub, workspace, static_cast<cudaStream_t>(stream)));
}

size_t avits_merge_final_workspace(avits_upmode mode, int B, int full_h, int full_w) {
  if ((mode != AVITS_UP_NEAREST && mode != AVITS_UP_BILINEAR) || B <= 0 || full_h <= 0 ||
      full_w <= 0)
    return 0;
  return merge_workspace_bytes(B, full_h, full_w);
}

avits_status avits_merge_final(const void* mixed, avits_dtype dt, int B, int N, const int32_t* pos,
                               const int32_t* span, int full_h, int full_w, int C, int p,
                               avits_upmode mode, void* out_full, void* workspace,
                               size_t ws_bytes, void* stream) {
  AVITS_RANGE();
  if (!mixed || !pos || !span || !out_full || !valid_dtype(dt)) return AVITS_ERR_INVALID_ARG;
  if (B <= 0 || N <= 0 || full_h <= 0 || full_w <= 0 || C <= 0) return AVITS_ERR_INVALID_ARG;
  if (p != 2) return AVITS_ERR_UNSUPPORTED;
  if (mode != AVITS_UP_NEAREST && mode != AVITS_UP_BILINEAR) return AVITS_ERR_INVALID_ARG;
  if (!aligned16(mixed) || !aligned16(out_full)) return AVITS_ERR_INVALID_ARG;
  if (mode == AVITS_UP_BILINEAR && ((full_h & 1) || (full_w & 1) || N > (1 << 28) - 1))
    return AVITS_ERR_INVALID_ARG;
  if (!workspace || !aligned16(workspace) ||
      ws_bytes < avits_merge_final_workspace(mode, B, full_h, full_w))
    return AVITS_ERR_INVALID_ARG;
  return cuda_status(launch_merge(mixed, dt, B, N, pos, span, full_h, full_w, C, mode, out_full,
                                  workspace, status_word(), static_cast<cudaStream_t>(stream)));
}

avits_status avits_cache_append(const avits_kv_cache* cache, const void* k_new, const void* v_new,
                                int T, const int32_t* cu_new, int64_t k_st, int64_t k_sh,
                                int64_t v_st, int64_t v_sh, void* stream) {
  AVITS_RANGE();
  if (T < 0 || !cu_new || (T > 0 && (!k_new || !v_new))) return AVITS_ERR_INVALID_ARG;
  if (k_st < 0 || k_sh < 0 || v_st < 0 || v_sh < 0) return AVITS_ERR_INVALID_ARG;
  const avits_status ok = check_cache(cache);
  if (ok != AVITS_OK) return ok;
  if (T == 0) return AVITS_OK;
  if (!pages_apart(*cache) || (cache->acc && !weights_apart(*cache))) return AVITS_ERR_INVALID_ARG;
  const int per16 = cache->dt == AVITS_BF16 ? 8 : 4;
  if (!aligned16(k_new) || !aligned16(v_new) || k_st % per16 || k_sh % per16 || v_st % per16 ||
      v_sh % per16)
    return AVITS_ERR_UNSUPPORTED;
  if (cache->k_pages == cache->v_pages) return AVITS_ERR_INVALID_ARG;
  return cuda_status(launch_cache_append(*cache, k_new, v_new, T, cu_new, k_st, k_sh, v_st, v_sh,
                                         status_word(), static_cast<cudaStream_t>(stream)));
}

size_t avits_cache_attention_workspace(const avits_kv_cache* cache, int H, int weights) {
  if (check_cache(cache) != AVITS_OK || H <= 0 || H % cache->Hkv ||
      !cache_attention_sizes_ok(*cache, H) || weights < AVITS_WEIGHTS_NONE ||
      weights > AVITS_WEIGHTS_ADD)
    return 0;
  return cache_attention_workspace(*cache, H, weights != AVITS_WEIGHTS_NONE, num_sms_current());
}

avits_status avits_cache_attention(const avits_kv_cache* cache, const void* q, int H,
                                   int64_t q_sb, int64_t q_sh, float softmax_scale, void* o,
                                   int64_t o_sb, int64_t o_sh, float* lse_opt, int weights,
                                   float weight, void* workspace, size_t ws_bytes, void* stream) {
  AVITS_RANGE();
  if (!q || !o || H <= 0 || q_sb < 0 || q_sh < 0 || o_sb < 0 || o_sh < 0)
    return AVITS_ERR_INVALID_ARG;
  if (!(softmax_scale > 0.f) || !(softmax_scale < 3.0e38f)) return AVITS_ERR_INVALID_ARG;
  if (weights < AVITS_WEIGHTS_NONE || weights > AVITS_WEIGHTS_ADD) return AVITS_ERR_INVALID_ARG;
  const avits_status ok = check_cache(cache);
  if (ok != AVITS_OK) return ok;
  if (H % cache->Hkv || (weights != AVITS_WEIGHTS_NONE && !cache->acc))
    return AVITS_ERR_INVALID_ARG;
  if ((H > 1 && o_sh < cache->d) || (cache->B > 1 && o_sb < cache->d)) return AVITS_ERR_INVALID_ARG;
  if (!cache_attention_sizes_ok(*cache, H)) return AVITS_ERR_UNSUPPORTED;
  if (!rows_apart(cache->d, {cache->B, o_sb}, {H, o_sh}) ||
      (weights != AVITS_WEIGHTS_NONE && !weights_apart(*cache)))
    return AVITS_ERR_INVALID_ARG;
  const int sms = num_sms_current();
  const size_t need = cache_attention_workspace(*cache, H, weights != AVITS_WEIGHTS_NONE, sms);
  if (need > 0 && (!workspace || !aligned16(workspace) || ws_bytes < need))
    return AVITS_ERR_INVALID_ARG;
  const CacheAttnCall call{*cache, q, H, q_sb, q_sh, softmax_scale, o, o_sb, o_sh, lse_opt,
                           weights, weight, workspace};
  return cuda_status(
      launch_cache_attention(call, sms, status_word(), static_cast<cudaStream_t>(stream)));
}

avits_status avits_cache_evict(const avits_kv_cache* src, const avits_kv_cache* dst, int keep,
                               int sinks, int recent, int32_t* keep_idx, void* stream) {
  AVITS_RANGE();
  if (!keep_idx || keep < 1 || sinks < 0 || recent < 0 || (int64_t)sinks + recent > keep)
    return AVITS_ERR_INVALID_ARG;
  for (const avits_kv_cache* c : {src, dst}) {
    const avits_status ok = check_cache(c);
    if (ok != AVITS_OK) return ok;
    if (!c->acc) return AVITS_ERR_INVALID_ARG;
  }
  if (src->dt != dst->dt || src->B != dst->B || src->Hkv != dst->Hkv || src->d != dst->d ||
      keep > dst->max_len || src->lens == dst->lens || src->acc == dst->acc)
    return AVITS_ERR_INVALID_ARG;
  if (!pages_apart(*dst) || !weights_apart(*dst)) return AVITS_ERR_INVALID_ARG;
  if ((int64_t)src->B * src->Hkv * ((int64_t)keep / 4 + 1) >= (1ll << 31))
    return AVITS_ERR_UNSUPPORTED;
  if (dst->k_pages == dst->v_pages) return AVITS_ERR_INVALID_ARG;
  return cuda_status(launch_cache_evict(*src, *dst, keep, sinks, recent, keep_idx, num_sms_current(),
                                        status_word(), static_cast<cudaStream_t>(stream)));
}

avits_status avits_cache_plan(const avits_kv_cache* cache, const int32_t* lens,
                              const int32_t* change, int32_t* free_pages,
                              const int32_t* free_count, int32_t* free_out, int T,
                              int32_t* cu_new, int64_t* slots, int32_t* seq, int32_t* place,
                              int32_t* pos_opt, const int32_t* pos_base_opt, void* stream) {
  AVITS_RANGE();
  if (T < 0 || !lens || !change || !free_pages || !free_count || !free_out || !cu_new ||
      (T > 0 && (!slots || !seq || !place)))
    return AVITS_ERR_INVALID_ARG;
  const avits_status ok = check_cache(cache);
  if (ok != AVITS_OK) return ok;
  if (cache->B > 1 && cache->table_sb < ((int64_t)cache->max_len - 1) / cache->page_size + 1)
    return AVITS_ERR_INVALID_ARG;
  if (T > (1 << 30)) return AVITS_ERR_UNSUPPORTED;
  const CachePlanCall call{*cache, lens, change, free_pages, free_count, free_out, T, cu_new,
                           slots, seq, place, pos_opt, pos_base_opt};
  return cuda_status(launch_cache_plan(call, status_word(), static_cast<cudaStream_t>(stream)));
}

avits_status avits_rotary_frequencies(int width, double base, int scaling, double factor,
                                      double original_len, double low, double high,
                                      uint64_t* freq) {
  if (!freq || width <= 0 || width % 2 || width > 256 || !(base > 0.0) || !std::isfinite(base))
    return AVITS_ERR_INVALID_ARG;
  if (scaling < AVITS_SCALE_NONE || scaling > AVITS_SCALE_PARTS) return AVITS_ERR_INVALID_ARG;
  if (scaling != AVITS_SCALE_NONE && (!(factor >= 1.0) || !std::isfinite(factor)))
    return AVITS_ERR_INVALID_ARG;
  if (scaling == AVITS_SCALE_PARTS &&
      (!(original_len > 0.0) || !std::isfinite(original_len) || !(low < high) ||
       !std::isfinite(low) || !std::isfinite(high)))
    return AVITS_ERR_INVALID_ARG;
  if (scaling == AVITS_SCALE_BASE && width > 2)
    base *= std::pow(factor, (double)width / (width - 2));
  constexpr double kTurn = 6.283185307179586476925286766559;
  uint64_t out[128];
  for (int i = 0; i < width / 2; ++i) {
    double f = std::pow(base, -2.0 * i / width) / kTurn;
    if (scaling == AVITS_SCALE_LINEAR) f /= factor;
    if (scaling == AVITS_SCALE_PARTS) {
      const double g = std::min(1.0, std::max(0.0, (original_len * f - low) / (high - low)));
      f = g * f + (1.0 - g) * f / factor;
    }
    if (!(f < 0.5)) return AVITS_ERR_INVALID_ARG;
    out[i] = (uint64_t)std::nearbyint(std::ldexp(f, 64));
  }
  std::copy(out, out + width / 2, freq);
  return AVITS_OK;
}

avits_status avits_norm_rotate(const avits_rotary* rot, avits_dtype dt, int B, int N, int d,
                               const int32_t* positions, int64_t pos_sb, int64_t pos_sn,
                               const void* q, int H, const int64_t* q_str, void* q_out,
                               const int64_t* qo_str, const void* k, int Hkv,
                               const int64_t* k_str, void* k_out, const int64_t* ko_str, int norm,
                               const void* q_weight, const void* k_weight, float eps,
                               void* stream) {
  AVITS_RANGE();
  if (!q || !q_out || !q_str || !qo_str || !valid_dtype(dt) || B <= 0 || N <= 0 || H <= 0 ||
      Hkv < 0 || d <= 0)
    return AVITS_ERR_INVALID_ARG;
  if ((Hkv > 0) != (k != nullptr) || (Hkv > 0 && (!k_out || !k_str || !ko_str)))
    return AVITS_ERR_INVALID_ARG;
  if (!rotary_ok(rot, d, positions) || pos_sb < 0 || pos_sn < 0) return AVITS_ERR_INVALID_ARG;
  if (!norm_ok(norm, q_weight, k_weight, eps)) return AVITS_ERR_INVALID_ARG;
  const int per16 = dt == AVITS_BF16 ? 8 : 4;
  if (d > 256 || d % per16 || (int64_t)B * N > (1 << 30) || H > (1 << 16) || Hkv > (1 << 16))
    return AVITS_ERR_UNSUPPORTED;
  const int64_t* in[2] = {q_str, k_str};
  const int64_t* out[2] = {qo_str, ko_str};
  const void* from[2] = {q, k};
  const void* to[2] = {q_out, k_out};
  for (int i = 0; i < (Hkv > 0 ? 2 : 1); ++i) {
    const int heads = i ? Hkv : H;
    for (int x = 0; x < 3; ++x) {
      if (in[i][x] < 0 || out[i][x] < 0) return AVITS_ERR_INVALID_ARG;
      if (in[i][x] % per16 || out[i][x] % per16) return AVITS_ERR_UNSUPPORTED;
    }
    if (!aligned16(from[i]) || !aligned16(to[i])) return AVITS_ERR_UNSUPPORTED;
    if (!rows_apart(d, {B, out[i][0]}, {N, out[i][1]}, {heads, out[i][2]}))
      return AVITS_ERR_INVALID_ARG;
    if (from[i] == to[i] && !same_strides(in[i], out[i], B, N, heads)) return AVITS_ERR_INVALID_ARG;
    if (to[i] == from[1 - i]) return AVITS_ERR_INVALID_ARG;
  }
  if (q_out == k_out) return AVITS_ERR_INVALID_ARG;
  if (!aligned16(q_weight) || !aligned16(k_weight)) return AVITS_ERR_UNSUPPORTED;
  RotateCall c{};
  c.rot = *rot;
  c.dt = dt;
  c.tokens = B * N;
  c.N = N; c.H = H; c.Hkv = Hkv; c.d = d;
  c.positions = positions;
  c.pos_sb = pos_sb; c.pos_sn = pos_sn;
  c.q = q; c.q_out = q_out; c.k = k; c.k_out = k_out;
  for (int x = 0; x < 3; ++x) {
    c.q_str[x] = q_str[x];
    c.qo_str[x] = qo_str[x];
    c.k_str[x] = Hkv > 0 ? k_str[x] : 0;
    c.ko_str[x] = Hkv > 0 ? ko_str[x] : 0;
  }
  c.norm = norm ? 1 : 0;
  c.q_weight = q_weight; c.k_weight = k_weight;
  c.eps = eps;
  return cuda_status(launch_norm_rotate(c, false, num_sms_current(), status_word(),
                                        static_cast<cudaStream_t>(stream)));
}

avits_status avits_cache_append_rotated(const avits_kv_cache* cache, const avits_rotary* rot, int T,
                                        const int32_t* positions, int64_t pos_st,
                                        const int64_t* slots, const int32_t* seq,
                                        const int32_t* place, const void* q, int H, int64_t q_st,
                                        int64_t q_sh, void* q_out, int64_t qo_st, int64_t qo_sh,
                                        const void* k_new, int64_t k_st, int64_t k_sh,
                                        const void* v_new, int64_t v_st, int64_t v_sh, int norm,
                                        const void* q_weight, const void* k_weight, float eps,
                                        void* stream) {
  AVITS_RANGE();
  if (T < 0 || H <= 0 || (T > 0 && (!slots || !q || !q_out || !k_new || !v_new)))
    return AVITS_ERR_INVALID_ARG;
  for (int64_t st : {q_st, q_sh, qo_st, qo_sh, k_st, k_sh, v_st, v_sh, pos_st})
    if (st < 0) return AVITS_ERR_INVALID_ARG;
  const avits_status ok = check_cache(cache);
  if (ok != AVITS_OK) return ok;
  if (!rotary_ok(rot, cache->d, T > 0 ? positions : cache->lens) ||
      !norm_ok(norm, q_weight, k_weight, eps))
    return AVITS_ERR_INVALID_ARG;
  if (cache->acc && T > 0 && (!seq || !place)) return AVITS_ERR_INVALID_ARG;
  if (T > (1 << 30) || H > (1 << 16)) return AVITS_ERR_UNSUPPORTED;
  if (T == 0) return AVITS_OK;
  if (!pages_apart(*cache) || (cache->acc && !weights_apart(*cache)) ||
      cache->k_pages == cache->v_pages)
    return AVITS_ERR_INVALID_ARG;
  const int per16 = cache->dt == AVITS_BF16 ? 8 : 4;
  for (const void* p : {q, static_cast<const void*>(q_out), k_new, v_new, q_weight, k_weight})
    if (!aligned16(p)) return AVITS_ERR_UNSUPPORTED;
  for (int64_t st : {q_st, q_sh, qo_st, qo_sh, k_st, k_sh, v_st, v_sh})
    if (st % per16) return AVITS_ERR_UNSUPPORTED;
  if (!rows_apart(cache->d, {T, qo_st}, {H, qo_sh})) return AVITS_ERR_INVALID_ARG;
  if (q == q_out && ((T > 1 && q_st != qo_st) || (H > 1 && q_sh != qo_sh)))
    return AVITS_ERR_INVALID_ARG;
  if (q_out == k_new || q_out == v_new || q_out == cache->k_pages || q_out == cache->v_pages)
    return AVITS_ERR_INVALID_ARG;
  RotateCall c{};
  c.rot = *rot;
  c.dt = static_cast<avits_dtype>(cache->dt);
  c.tokens = T;
  c.N = T; c.H = H; c.Hkv = cache->Hkv; c.d = cache->d;
  c.positions = positions;
  c.pos_sn = pos_st;
  c.q = q; c.q_out = q_out; c.k = k_new;
  c.q_str[1] = q_st; c.q_str[2] = q_sh; c.qo_str[1] = qo_st; c.qo_str[2] = qo_sh;
  c.k_str[1] = k_st; c.k_str[2] = k_sh;
  c.norm = norm ? 1 : 0;
  c.q_weight = q_weight; c.k_weight = k_weight;
  c.eps = eps;
  c.cache = *cache;
  c.slots = slots; c.seq = seq; c.place = place;
  c.v = v_new; c.v_st = v_st; c.v_sh = v_sh;
  return cuda_status(launch_norm_rotate(c, true, num_sms_current(), status_word(),
                                        static_cast<cudaStream_t>(stream)));
}

// Descriptions that avits_cache_attention_shared takes together, with H heads.
static avits_status check_shared(const avits_kv_cache* cache, const avits_kv_cache* prefix, int H,
                                 int sms) {
  for (const avits_kv_cache* c : {cache, prefix}) {
    const avits_status ok = check_cache(c);
    if (ok != AVITS_OK) return ok;
  }
  if (cache->dt != prefix->dt || cache->Hkv != prefix->Hkv || cache->d != prefix->d || H <= 0 ||
      H % cache->Hkv)
    return AVITS_ERR_INVALID_ARG;
  CacheSharedCall call{};
  call.cache = *cache;
  call.prefix = *prefix;
  call.H = H;
  return cache_shared_sizes_ok(call, sms) ? AVITS_OK : AVITS_ERR_UNSUPPORTED;
}

size_t avits_cache_attention_shared_workspace(const avits_kv_cache* cache,
                                              const avits_kv_cache* prefix, int H) {
  const int sms = std::max(1, num_sms_current());
  if (check_shared(cache, prefix, H, sms) != AVITS_OK) return 0;
  CacheSharedCall call{};
  call.cache = *cache;
  call.prefix = *prefix;
  call.H = H;
  return cache_shared_workspace(call, sms);
}

avits_status avits_cache_attention_shared(const avits_kv_cache* cache, const avits_kv_cache* prefix,
                                          const int32_t* group_start, const void* q, int H,
                                          int64_t q_sb, int64_t q_sh, float softmax_scale, void* o,
                                          int64_t o_sb, int64_t o_sh, float* lse_opt,
                                          void* workspace, size_t ws_bytes, void* stream) {
  AVITS_RANGE();
  if (!group_start || !q || !o || q_sb < 0 || q_sh < 0 || o_sb < 0 || o_sh < 0)
    return AVITS_ERR_INVALID_ARG;
  if (!(softmax_scale > 0.f) || !(softmax_scale < 3.0e38f)) return AVITS_ERR_INVALID_ARG;
  const int sms = std::max(1, num_sms_current());
  const avits_status ok = check_shared(cache, prefix, H, sms);
  if (ok != AVITS_OK) return ok;
  if (!rows_apart(cache->d, {cache->B, o_sb}, {H, o_sh})) return AVITS_ERR_INVALID_ARG;
  const CacheSharedCall call{*cache, *prefix, group_start, q, H, q_sb, q_sh, softmax_scale,
                             o, o_sb, o_sh, lse_opt, workspace};
  if (!workspace || !aligned16(workspace) || ws_bytes < cache_shared_workspace(call, sms))
    return AVITS_ERR_INVALID_ARG;
  return cuda_status(
      launch_cache_shared(call, sms, status_word(), static_cast<cudaStream_t>(stream)));
}

avits_status avits_call_packed(int call, const void* args) {
  if (!args) return AVITS_ERR_INVALID_ARG;
  Packed p{static_cast<const char*>(args)};
  // braces: initialised in the order they are written
  switch (call) {
    case AVITS_CALL_CACHE_PLAN: {
      struct {
        const avits_kv_cache* cache; const int32_t *lens, *change; int32_t* free_pages;
        const int32_t* free_count; int32_t* free_out; int T; int32_t* cu; int64_t* slots;
        int32_t *seq, *place, *pos; const int32_t* base; void* stream;
      } a{p.ptr<const avits_kv_cache>(), p.ptr<const int32_t>(), p.ptr<const int32_t>(),
          p.ptr<int32_t>(), p.ptr<const int32_t>(), p.ptr<int32_t>(), p.i32(), p.ptr<int32_t>(),
          p.ptr<int64_t>(), p.ptr<int32_t>(), p.ptr<int32_t>(), p.ptr<int32_t>(),
          p.ptr<const int32_t>(), p.ptr<void>()};
      if (!p.ok) return AVITS_ERR_INVALID_ARG;
      return avits_cache_plan(a.cache, a.lens, a.change, a.free_pages, a.free_count, a.free_out, a.T,
                              a.cu, a.slots, a.seq, a.place, a.pos, a.base, a.stream);
    }
    case AVITS_CALL_NORM_ROTATE: {
      struct {
        const avits_rotary* rot; int dt, B, N, d; const int32_t* positions; int64_t pos_sb, pos_sn;
        const void* q; int H; const int64_t* q_str; void* q_out; const int64_t* qo_str;
        const void* k; int Hkv; const int64_t* k_str; void* k_out; const int64_t* ko_str; int norm;
        const void *q_weight, *k_weight; float eps; void* stream;
      } a{p.ptr<const avits_rotary>(), p.i32(), p.i32(), p.i32(), p.i32(), p.ptr<const int32_t>(),
          p.i64(), p.i64(), p.ptr<const void>(), p.i32(), p.ptr<const int64_t>(), p.ptr<void>(),
          p.ptr<const int64_t>(), p.ptr<const void>(), p.i32(), p.ptr<const int64_t>(),
          p.ptr<void>(), p.ptr<const int64_t>(), p.i32(), p.ptr<const void>(),
          p.ptr<const void>(), p.f32(), p.ptr<void>()};
      if (!p.ok) return AVITS_ERR_INVALID_ARG;
      return avits_norm_rotate(a.rot, static_cast<avits_dtype>(a.dt), a.B, a.N, a.d, a.positions,
                               a.pos_sb, a.pos_sn, a.q, a.H, a.q_str, a.q_out, a.qo_str, a.k, a.Hkv,
                               a.k_str, a.k_out, a.ko_str, a.norm, a.q_weight, a.k_weight, a.eps,
                               a.stream);
    }
    case AVITS_CALL_CACHE_APPEND_ROTATED: {
      struct {
        const avits_kv_cache* cache; const avits_rotary* rot; int T; const int32_t* positions;
        int64_t pos_st; const int64_t* slots; const int32_t *seq, *place; const void* q; int H;
        int64_t q_st, q_sh; void* q_out; int64_t qo_st, qo_sh; const void* k; int64_t k_st, k_sh;
        const void* v; int64_t v_st, v_sh; int norm; const void *q_weight, *k_weight; float eps;
        void* stream;
      } a{p.ptr<const avits_kv_cache>(), p.ptr<const avits_rotary>(), p.i32(),
          p.ptr<const int32_t>(), p.i64(), p.ptr<const int64_t>(), p.ptr<const int32_t>(),
          p.ptr<const int32_t>(), p.ptr<const void>(), p.i32(), p.i64(), p.i64(), p.ptr<void>(),
          p.i64(), p.i64(), p.ptr<const void>(), p.i64(), p.i64(), p.ptr<const void>(), p.i64(),
          p.i64(), p.i32(), p.ptr<const void>(), p.ptr<const void>(), p.f32(), p.ptr<void>()};
      if (!p.ok) return AVITS_ERR_INVALID_ARG;
      return avits_cache_append_rotated(a.cache, a.rot, a.T, a.positions, a.pos_st, a.slots, a.seq,
                                        a.place, a.q, a.H, a.q_st, a.q_sh, a.q_out, a.qo_st,
                                        a.qo_sh, a.k, a.k_st, a.k_sh, a.v, a.v_st, a.v_sh, a.norm,
                                        a.q_weight, a.k_weight, a.eps, a.stream);
    }
    case AVITS_CALL_CACHE_ATTENTION_SHARED: {
      struct {
        const avits_kv_cache *cache, *prefix; const int32_t* start; const void* q; int H;
        int64_t q_sb, q_sh; float scale; void* o; int64_t o_sb, o_sh; float* lse; void* ws;
        int64_t ws_bytes; void* stream;
      } a{p.ptr<const avits_kv_cache>(), p.ptr<const avits_kv_cache>(), p.ptr<const int32_t>(),
          p.ptr<const void>(), p.i32(), p.i64(), p.i64(), p.f32(), p.ptr<void>(), p.i64(), p.i64(),
          p.ptr<float>(), p.ptr<void>(), p.i64(), p.ptr<void>()};
      if (!p.ok || a.ws_bytes < 0) return AVITS_ERR_INVALID_ARG;
      return avits_cache_attention_shared(a.cache, a.prefix, a.start, a.q, a.H, a.q_sb, a.q_sh,
                                          a.scale, a.o, a.o_sb, a.o_sh, a.lse, a.ws,
                                          (size_t)a.ws_bytes, a.stream);
    }
  }
  return AVITS_ERR_INVALID_ARG;
}

avits_status avits_selftest_bounded_wait(unsigned long long limit_ns, long long* result,
                                         void* stream) {
  AVITS_RANGE();
  if (!result || limit_ns < 1000ull || limit_ns > 100ull * 1000ull * 1000ull)
    return AVITS_ERR_INVALID_ARG;
  return cuda_status(launch_wait_selftest(limit_ns, result, status_word(),
                                          static_cast<cudaStream_t>(stream)));
}

avits_status avits_device_status(void* stream) {
  AVITS_RANGE();
  cudaError_t e = cudaStreamSynchronize(static_cast<cudaStream_t>(stream));
  if (e != cudaSuccess) return cuda_status(e);
  unsigned int w = 0, zero = 0;
  e = cudaMemcpyFromSymbol(&w, g_status, sizeof(w));
  if (e != cudaSuccess) return cuda_status(e);
  if (w) {
    e = cudaMemcpyToSymbol(g_status, &zero, sizeof(zero));
    if (e != cudaSuccess) return cuda_status(e);
  }
  for (int c = 1; c < 32; ++c)
    if (w & (1u << c)) return static_cast<avits_status>(c);
  return AVITS_OK;
}

}  // extern "C"
