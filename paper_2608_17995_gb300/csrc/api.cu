// api.cu — the C ABI of libavits (see include/avits.h): host-side argument
// checks, workspace sizing and dispatch to the kernels.  Nothing here
// allocates device memory or synchronises, except avits_device_status().
#include <algorithm>
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
