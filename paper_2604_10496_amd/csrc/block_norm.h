// Shared by the two directions of the norms around a block (gfx950 only): arguments, checks and the rule for the row layout.
#ifndef CQ_BLOCK_NORM_H_
#define CQ_BLOCK_NORM_H_

#include <math.h>

#include "cq_rows.h"

namespace {

constexpr int kMaxNormWidth = 32768;

struct norm_args {
  int T, H, wf32, gate_kind, sigmoid;
  float eps, rho, beta;
  const void *w_pre, *w_post, *h, *y, *gate;
};

inline cq_status check_norm_spec(const cq_block_norm_spec* P, int T) {
  if (!P) return CQ_ERR_NULL;
  if (T < 0 || T > 1 << 30 || P->H <= 0 || P->H > kMaxNormWidth || !(P->eps > 0.f) || !isfinite(P->eps)) return CQ_ERR_SHAPE;
  if (!cq_row_kind(P->stream_kind)) return CQ_ERR_UNSUPPORTED;
  if (P->block_kind != P->stream_kind && P->block_kind != CQ_A_F32) return CQ_ERR_UNSUPPORTED;
  if (P->weight_kind != P->stream_kind && P->weight_kind != CQ_A_F32) return CQ_ERR_UNSUPPORTED;
  if (P->gate_kind != CQ_GATE_NONE && P->gate_kind != CQ_GATE_ROW && P->gate_kind != CQ_GATE_ELEM) return CQ_ERR_UNSUPPORTED;
  return CQ_OK;
}

inline norm_args make_norm_args(const cq_block_norm_spec* P, int T, const void* h, const void* y, const void* gate) {
  norm_args a;
  a.T = T;
  a.H = P->H;
  a.wf32 = P->weight_kind == CQ_A_F32;
  a.gate_kind = y ? P->gate_kind : CQ_GATE_NONE;
  a.sigmoid = P->gate_sigmoid != 0;
  a.eps = P->eps;
  a.rho = P->residual_scale;
  a.beta = P->branch_scale;
  a.w_pre = P->w_pre;
  a.w_post = y ? P->w_post : nullptr;
  a.h = h;
  a.y = y;
  a.gate = gate;
  return a;
}

template <int SK>
__device__ __forceinline__ void slot_weights(const void* w, int wf32, const row_slot& s, int H, float (&v)[8]) {
  if (SK == CQ_A_F32 || wf32)
    row_values<CQ_A_F32>(slot_fetch<CQ_A_F32>(w, 0, s, H, true), v);
  else
    row_values<SK>(slot_fetch<SK>(w, 0, s, H, true), v);
}

__device__ __forceinline__ float sigmoid_of(float z) { return 1.f / (1.f + expf(-z)); }

// The same with its slope s (1 - s) = s(z) s(-z) = e / (1 + e)^2, e = exp(-|z|): no difference, which would leave nothing of the slope
// of a gate that is nearly open (s - s^2: 1 % off at z = 12, 0 from z = 17).
__device__ __forceinline__ float sigmoid_of(float z, float& slope) {
  const float e = expf(-fabsf(z)), r = 1.f / (1.f + e), er = e * r;
  slope = er * r;
  return z >= 0.f ? r : er;
}

}  // namespace

// Runs LAUNCH(SK, BK, NT, C) for the kinds and the width of a call.  A row belongs to NT threads, each of which holds C groups
// of eight values.
#define CQ_NORM_WIDTHS(LAUNCH, SK, BK, H)            \
  do {                                               \
    if ((H) <= 512) LAUNCH(SK, BK, 64, 1);           \
    else if ((H) <= 2048) LAUNCH(SK, BK, 256, 1);    \
    else if ((H) <= 4096) LAUNCH(SK, BK, 512, 1);    \
    else if ((H) <= 8192) LAUNCH(SK, BK, 1024, 1);   \
    else if ((H) <= 16384) LAUNCH(SK, BK, 1024, 2);  \
    else LAUNCH(SK, BK, 1024, 4);                    \
  } while (0)
#define CQ_NORM_DISPATCH(LAUNCH, sk, bk, H)                                                       \
  do {                                                                                            \
    if ((sk) == CQ_A_F32) CQ_NORM_WIDTHS(LAUNCH, CQ_A_F32, CQ_A_F32, H);                          \
    else if ((sk) == CQ_A_F16 && (bk) == CQ_A_F16) CQ_NORM_WIDTHS(LAUNCH, CQ_A_F16, CQ_A_F16, H); \
    else if ((sk) == CQ_A_F16) CQ_NORM_WIDTHS(LAUNCH, CQ_A_F16, CQ_A_F32, H);                     \
    else if ((bk) == CQ_A_BF16) CQ_NORM_WIDTHS(LAUNCH, CQ_A_BF16, CQ_A_BF16, H);                  \
    else CQ_NORM_WIDTHS(LAUNCH, CQ_A_BF16, CQ_A_F32, H);                                          \
  } while (0)

#endif  // CQ_BLOCK_NORM_H_
