// Entry points of the head norm with rotation (declared in include/upipe.h):
// argument checks and the frequency table that travels with the launch.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <cmath>

#include "../../include/upipe.h"
#include "api_internal.h"
#include "kernels.h"

namespace upipe {

namespace {

constexpr int64_t kMaxNormRows = int64_t(1) << 31;    // tokens, exclusive

int check_norm(int64_t T, int Hq, int Hkv, int d) {
  if (T < 0 || Hq < 1 || Hkv < 1) return UPIPE_ERR_INVALID_ARG;
  if (d != HEAD_DIM || Hq > kMaxHeads || Hkv > kMaxHeads || T >= kMaxNormRows)
    return UPIPE_ERR_UNSUPPORTED;
  return UPIPE_OK;
}

bool positive(double x) { return x > 0.0 && std::isfinite(x); }

// What both directions check and hand on.
int norm_args(const upipe_heads& q, const upipe_heads& k, const void* wq, const void* wk,
              int w_fp32, const int64_t* positions, int64_t T, int Hq, int Hkv, double base,
              double eps, NormRopeArgs* a) {
  if ((w_fp32 != 0 && w_fp32 != 1) || !positive(base) || !positive(eps) ||
      !positive((float)eps) || !aligned16(wq) || !aligned16(wk) || !aligned16(positions))
    return UPIPE_ERR_INVALID_ARG;
  if (!heads_ok(q, T, Hq) || !heads_ok(k, T, Hkv)) return UPIPE_ERR_INVALID_ARG;
  *a = NormRopeArgs{};
  a->q.x = view_of(q);
  a->k.x = view_of(k);
  a->q.w = wq;
  a->k.w = wk;
  a->q.H = Hq;
  a->k.H = Hkv;
  const double log2_base = std::log2(base);
  for (int e = 0; e < HEAD_DIM / 2; ++e)
    a->freq.turns[e] = std::exp2(-(double)e * log2_base / 64.0) * 0.15915494309189535;
  a->positions = positions;
  a->T = T;
  a->eps = (float)eps;
  a->w_fp32 = w_fp32;
  return UPIPE_OK;
}

// Rows out may be written while the rows in are read: a row group reads its row of
// `same` before it writes it.
bool may_write(const upipe_heads& out, int64_t T, int H, const upipe_heads& in, int H_in,
               bool same) {
  return (same && heads_same(out, in)) || heads_apart(out, T, H, in, T, H_in);
}

size_t partial_bytes(int64_t T, int Hq, int Hkv) {
  return (size_t)norm_rope_bwd_partials(T, Hq, Hkv) * HEAD_DIM * sizeof(float);
}

}  // namespace

}  // namespace upipe

using namespace upipe;

extern "C" {

int upipe_qk_norm_rope(upipe_heads q, upipe_heads k, const void* wq, const void* wk, int w_fp32,
                       const int64_t* positions, upipe_heads q_out, upipe_heads k_out, int64_t T,
                       int Hq, int Hkv, int d, double base, double eps, hipStream_t stream) {
  try {
    int rc = check_norm(T, Hq, Hkv, d);
    if (rc != UPIPE_OK || T == 0) return rc;
    NormRopeArgs a;
    rc = norm_args(q, k, wq, wk, w_fp32, positions, T, Hq, Hkv, base, eps, &a);
    if (rc != UPIPE_OK) return rc;
    if (!heads_ok(q_out, T, Hq) || !heads_ok(k_out, T, Hkv) || !heads_distinct(q_out, T, Hq) ||
        !heads_distinct(k_out, T, Hkv))
      return UPIPE_ERR_INVALID_ARG;
    if (!may_write(q_out, T, Hq, q, Hq, true) || !may_write(q_out, T, Hq, k, Hkv, false) ||
        !may_write(k_out, T, Hkv, k, Hkv, true) || !may_write(k_out, T, Hkv, q, Hq, false) ||
        !may_write(q_out, T, Hq, k_out, Hkv, false))
      return UPIPE_ERR_INVALID_ARG;
    a.q.y = view_of(q_out);
    a.k.y = view_of(k_out);
    UPIPE_LAUNCH(kNormRope, stream, launch_norm_rope(a, stream));
    return UPIPE_OK;
  } catch (...) {
    return UPIPE_ERR_HIP;
  }
}

size_t upipe_qk_norm_rope_bwd_workspace_size(int64_t T, int Hq, int Hkv, int d) {
  if (check_norm(T, Hq, Hkv, d) != UPIPE_OK) return 0;
  return partial_bytes(T, Hq, Hkv) + 16;       // never 0: that says invalid
}

int upipe_qk_norm_rope_bwd(upipe_heads q, upipe_heads k, const void* wq, const void* wk, int w_fp32,
                           const int64_t* positions, upipe_heads dq_out, upipe_heads dk_out,
                           upipe_heads dq, upipe_heads dk, void* dwq, void* dwk, int64_t T, int Hq,
                           int Hkv, int d, double base, double eps, void* ws, size_t ws_bytes,
                           hipStream_t stream) {
  try {
    int rc = check_norm(T, Hq, Hkv, d);
    if (rc != UPIPE_OK) return rc;
    if (!aligned16(dwq) || !aligned16(dwk) || !aligned16(ws)) return UPIPE_ERR_INVALID_ARG;
    NormRopeArgs a{};
    if (T > 0) {
      rc = norm_args(q, k, wq, wk, w_fp32, positions, T, Hq, Hkv, base, eps, &a);
      if (rc != UPIPE_OK) return rc;
      const upipe_heads* out[2] = {&dq, &dk};
      const upipe_heads* x[2] = {&q, &k};
      const upipe_heads* dy[2] = {&dq_out, &dk_out};
      const int H[2] = {Hq, Hkv};
      for (int i = 0; i < 2; ++i) {
        if (!heads_ok(*dy[i], T, H[i]) || !heads_ok(*out[i], T, H[i]) ||
            !heads_distinct(*out[i], T, H[i]))
          return UPIPE_ERR_INVALID_ARG;
        for (int n = 0; n < 2; ++n)
          if (!may_write(*out[i], T, H[i], *x[n], H[n], i == n) ||
              !may_write(*out[i], T, H[i], *dy[n], H[n], i == n))
            return UPIPE_ERR_INVALID_ARG;
      }
      if (!may_write(dq, T, Hq, dk, Hkv, false)) return UPIPE_ERR_INVALID_ARG;
    } else if (w_fp32 != 0 && w_fp32 != 1) {
      return UPIPE_ERR_INVALID_ARG;
    }
    if (ws_bytes < upipe_qk_norm_rope_bwd_workspace_size(T, Hq, Hkv, d)) return UPIPE_ERR_WORKSPACE;
    if (T > 0) {
      a.q.dy = view_of(dq_out);
      a.k.dy = view_of(dk_out);
      a.q.y = view_of(dq);
      a.k.y = view_of(dk);
      UPIPE_LAUNCH(kNormRopeBwd, stream, launch_norm_rope_bwd(a, (float*)ws, stream));
    }
    UPIPE_LAUNCH(kNormDwFold, stream,
                 launch_norm_dw_fold((const float*)ws, T, Hq, Hkv, dwq, dwk, w_fp32, stream));
    return UPIPE_OK;
  } catch (...) {
    return UPIPE_ERR_HIP;
  }
}

}  // extern "C"
