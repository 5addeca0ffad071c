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
  if (T < 0 || P->H <= 0 || P->H > kMaxNormWidth || !(P->eps > 0.f) || !isfinite(P->eps)) return CQ_ERR_SHAPE;
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

// Whether rows of width H may be moved 16 bytes at a time: every row starts on 16 bytes and is whole groups of eight values.
inline bool rows_aligned(int H, const void* const* p, int n) {
  uintptr_t all = 0;
  for (int i = 0; i < n; ++i) all |= reinterpret_cast<uintptr_t>(p[i]);
  return H % 8 == 0 && all % 16 == 0;
}

template <int SK, bool VEC>
__device__ __forceinline__ void weight_load8(const void* w, int wf32, int c, int left, float (&v)[8]) {
  if (SK == CQ_A_F32 || wf32)
    row_load8<CQ_A_F32, VEC>(w, c, left, v);
  else
    row_load8<SK, VEC>(w, c, left, v);
}

__device__ __forceinline__ float sigmoid_of(float z) { return 1.f / (1.f + expf(-z)); }

}  // namespace

// Runs LAUNCH(SK, BK, NT, C, VEC) for the kinds, the width and the alignment of a call.  A row belongs to one workgroup of NT
// threads, each of which holds C groups of eight values.
#define CQ_NORM_WIDTHS(LAUNCH, SK, BK, VEC, H)            \
  do {                                                    \
    if ((H) <= 512) LAUNCH(SK, BK, 64, 1, VEC);           \
    else if ((H) <= 2048) LAUNCH(SK, BK, 256, 1, VEC);    \
    else if ((H) <= 4096) LAUNCH(SK, BK, 512, 1, VEC);    \
    else if ((H) <= 8192) LAUNCH(SK, BK, 1024, 1, VEC);   \
    else if ((H) <= 16384) LAUNCH(SK, BK, 1024, 2, VEC);  \
    else LAUNCH(SK, BK, 1024, 4, VEC);                    \
  } while (0)
#define CQ_NORM_KINDS(LAUNCH, sk, bk, VEC, H)                                                          \
  do {                                                                                                 \
    if ((sk) == CQ_A_F32) CQ_NORM_WIDTHS(LAUNCH, CQ_A_F32, CQ_A_F32, VEC, H);                          \
    else if ((sk) == CQ_A_F16 && (bk) == CQ_A_F16) CQ_NORM_WIDTHS(LAUNCH, CQ_A_F16, CQ_A_F16, VEC, H); \
    else if ((sk) == CQ_A_F16) CQ_NORM_WIDTHS(LAUNCH, CQ_A_F16, CQ_A_F32, VEC, H);                     \
    else if ((bk) == CQ_A_BF16) CQ_NORM_WIDTHS(LAUNCH, CQ_A_BF16, CQ_A_BF16, VEC, H);                  \
    else CQ_NORM_WIDTHS(LAUNCH, CQ_A_BF16, CQ_A_F32, VEC, H);                                          \
  } while (0)
#define CQ_NORM_DISPATCH(LAUNCH, sk, bk, vec, H)               \
  do {                                                         \
    if (vec) CQ_NORM_KINDS(LAUNCH, sk, bk, true, H);           \
    else CQ_NORM_KINDS(LAUNCH, sk, bk, false, H);              \
  } while (0)

#endif  // CQ_BLOCK_NORM_H_
