// The norm behind a block, its gate, the residual sum and the norm before the next block, in one pass over the rows:
//   u = N(y) w_post (or y),  h' = rho h + beta a u,  x = N(h') w_pre,  N(v) = v / sqrt(mean v^2 + eps).
// Two row sums (y^2, then h'^2) stand between loads and stores; the row stays in registers in fp32 throughout, so that x comes
// from the unrounded h'.  Bound by HBM: y and h are read once, h' and x written once, about ten operations per value: 4096 x 4096 with
// norms on both sides and a gate per token, bf16 stream and fp32 block, 201 MB in 37.9 us = 5.3 TB/s (a copy: 5.16); a single
// token 2.6 us.
#include "block_norm.h"

namespace {

template <int SK, int BK, int NT, int C>
__global__ __launch_bounds__(NT) void block_norm_kernel(norm_args P, void* h_out, void* x_out) {
  __shared__ float lds[2][NT / 64];
  const size_t row = (size_t)blockIdx.x * P.H;
  const int H = P.H;
  auto slot = [&](int j) { return row_slot((threadIdx.x + j * NT) * 8, H); };
  row8<SK> h_raw[C];
  row8<BK> y_raw[C];
#pragma unroll
  for (int j = 0; j < C; ++j) {
    y_raw[j] = slot_fetch<BK>(P.y, row, slot(j), H, P.y != nullptr);
    h_raw[j] = slot_fetch<SK>(P.h, row, slot(j), H, true);
  }
  float q = P.beta;
  if (P.gate_kind == CQ_GATE_ROW) {
    const float z = elem_load<BK>(P.gate, blockIdx.x);
    q *= P.sigmoid ? sigmoid_of(z) : z;
  }
  float h[C][8];
  if (P.y) {
    float y[C][8];
#pragma unroll
    for (int j = 0; j < C; ++j) slot_values<BK>(y_raw[j], slot(j), H, y[j]);
    if (P.w_post) {
      float s[1] = {0.f};
#pragma unroll
      for (int j = 0; j < C; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) s[0] = fmaf(y[j][i], y[j][i], s[0]);
      group_sum<NT, 1>(s, lds[0]);
      q *= 1.f / sqrtf(s[0] / (float)H + P.eps);
    }
#pragma unroll
    for (int j = 0; j < C; ++j) {
      if (P.w_post) {
        float w[8];
        slot_weights<SK>(P.w_post, P.wf32, slot(j), H, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[j][i] *= w[i];
      }
      if (P.gate_kind == CQ_GATE_ELEM) {
        float z[8];
        row_values<BK>(slot_fetch<BK>(P.gate, row, slot(j), H, true), z);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[j][i] *= P.sigmoid ? sigmoid_of(z[i]) : z[i];
      }
      slot_values<SK>(h_raw[j], slot(j), H, h[j]);
#pragma unroll
      for (int i = 0; i < 8; ++i) h[j][i] = fmaf(q, y[j][i], P.rho * h[j][i]);
      slot_store<SK>(h_out, row, slot(j), H, true, h[j]);
    }
  } else {
#pragma unroll
    for (int j = 0; j < C; ++j) slot_values<SK>(h_raw[j], slot(j), H, h[j]);
  }
  if (!x_out) return;
  float s[1] = {0.f};
#pragma unroll
  for (int j = 0; j < C; ++j) {
    const int skip = slot(j).skip;
#pragma unroll
    for (int i = 0; i < 8; ++i) s[0] = H % 8 != 0 && i < skip ? s[0] : fmaf(h[j][i], h[j][i], s[0]);
  }
  group_sum<NT, 1>(s, lds[1]);
  const float r = 1.f / sqrtf(s[0] / (float)H + P.eps);
#pragma unroll
  for (int j = 0; j < C; ++j) {
    float w[8];
    slot_weights<SK>(P.w_pre, P.wf32, slot(j), H, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] *= h[j][i] * r;
    slot_store<BK>(x_out, row, slot(j), H, true, w);
  }
}

}  // namespace

extern "C" cq_status cq_block_norm(const cq_block_norm_spec* P, const void* h, const void* y, const void* gate, int T,
                                   void* h_out, void* x_out, cq_stream stream) {
  const cq_status st = check_norm_spec(P, T);
  if (st != CQ_OK) return st;
  if (T == 0) return CQ_OK;
  if (!h || (!y && !x_out) || (y && !h_out) || (x_out && !P->w_pre)) return CQ_ERR_NULL;
  if (y && P->gate_kind != CQ_GATE_NONE && !gate) return CQ_ERR_NULL;
  constexpr int kMostRows = (int)(kMostThreads / 1024);   // (of the widest rows' workgroups)
  for (int t = 0; t < T; t += kMostRows) {
    const int rows = T - t < kMostRows ? T - t : kMostRows;
    const size_t at = (size_t)t * P->H;
    const norm_args a = make_norm_args(P, rows, row_at(h, P->stream_kind, at), row_at(y, P->block_kind, at),
                                       row_at(gate, P->block_kind, P->gate_kind == CQ_GATE_ROW ? (size_t)t : at));
    void *const h_new = row_at(h_out, P->stream_kind, at), *const x = row_at(x_out, P->block_kind, at);
#define LAUNCH(SK, BK, NT, C) \
  hipLaunchKernelGGL((block_norm_kernel<SK, BK, NT, C>), dim3(rows), dim3(NT), 0, (hipStream_t)stream, a, h_new, x)
    CQ_NORM_DISPATCH(LAUNCH, P->stream_kind, P->block_kind, P->H);
#undef LAUNCH
    const cq_status launched = cq_check_launch();
    if (launched != CQ_OK) return launched;
  }
  return CQ_OK;
}
