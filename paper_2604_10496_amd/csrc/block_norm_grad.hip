// Gradients of the norms around a block, from h' as stored, y, the gate and the gradients of h' and x.  Per row, with
//   r = 1 / sqrt(mean h'^2 + eps), n = h' r, dn = dx w_pre:     D  = dh' + r (dn - n mean(dn n)),   dh = rho D,  dw_pre += dx n
//   q = 1 / sqrt(mean y^2 + eps),  m = y q,  u = m w_post, a:   du = beta a D,  da = beta u D,      dw_post += du m,
//                                                               dm = du w_post,  dy = q (dm - m mean(dm m)).
// The sums of squares are taken again, together with mean(dn h') in the first of two row sums and with the sum behind a row's
// gate in the second, so that the forward pass keeps no statistics.
// A workgroup takes rows b, b + parts, ...; its share of the weights' gradients stays in registers and goes to the workspace
// once, [parts][H] each; a second launch adds the parts in order.  No atomics: the results do not depend on timing.
#include "block_norm.h"

namespace {

constexpr int kMostParts = 512;

inline int grad_parts(int T) { return T < kMostParts ? T : kMostParts; }

struct norm_grad_args {
  norm_args f;
  int parts;
  const void *dh_out, *dx;
  void *dh, *dy, *dgate;
  float *part_pre, *part_post;
};

template <int SK, int BK, int NT, int C, bool VEC>
__global__ __launch_bounds__(NT) void block_norm_grad_kernel(norm_grad_args G) {
  const norm_args& P = G.f;
  // (two sets, used by rows in turn: a row's sums are read while the next row's may be written already)
  __shared__ float lds[2][2][3 * (NT / 64)];
  const int c0 = threadIdx.x * 8;
  const float inv_H = 1.f / (float)P.H;
  float acc_pre[C][8], acc_post[C][8];
#pragma unroll
  for (int j = 0; j < C; ++j)
#pragma unroll
    for (int i = 0; i < 8; ++i) acc_pre[j][i] = acc_post[j][i] = 0.f;
  int set = 0;
  for (int t = blockIdx.x; t < P.T; t += G.parts, set ^= 1) {
    const size_t row = (size_t)t * P.H;
    float d[C][8];   // gradient that reaches h'
#pragma unroll
    for (int j = 0; j < C; ++j) {
      const int c = c0 + j * NT * 8;
      if (G.dh_out) {
        row_load8<SK, VEC>(G.dh_out, row + c, P.H - c, d[j]);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) d[j][i] = 0.f;
      }
    }
    if (G.dx) {
      float h[C][8], dx[C][8];
      float s[2] = {0.f, 0.f};   // h'^2, dx w h'
#pragma unroll
      for (int j = 0; j < C; ++j) {
        const int c = c0 + j * NT * 8;
        float w[8];
        row_load8<SK, VEC>(P.h, row + c, P.H - c, h[j]);
        row_load8<BK, VEC>(G.dx, row + c, P.H - c, dx[j]);
        weight_load8<SK, VEC>(P.w_pre, P.wf32, c, P.H - c, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          s[0] = fmaf(h[j][i], h[j][i], s[0]);
          s[1] = fmaf(dx[j][i] * w[i], h[j][i], s[1]);
        }
      }
      group_sum<NT, 2>(s, lds[set][0]);
      const float r = 1.f / sqrtf(s[0] * inv_H + P.eps);
      const float back = r * r * s[1] * inv_H;   // D = dh' + r (dn - h' r^2 mean(dn h'))
#pragma unroll
      for (int j = 0; j < C; ++j) {
        const int c = c0 + j * NT * 8;
        float w[8];
        weight_load8<SK, VEC>(P.w_pre, P.wf32, c, P.H - c, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          d[j][i] = fmaf(r, fmaf(-back, h[j][i], dx[j][i] * w[i]), d[j][i]);
          acc_pre[j][i] = fmaf(dx[j][i], h[j][i] * r, acc_pre[j][i]);
        }
      }
    }
    const float rho = P.y ? P.rho : 1.f;
#pragma unroll
    for (int j = 0; j < C; ++j) {
      const int c = c0 + j * NT * 8;
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = rho * d[j][i];
      row_store8<SK, VEC>(G.dh, row + c, P.H - c, v);
    }
    if (P.y) {
      float y[C][8];
      float ga = 1.f;
      if (P.gate_kind == CQ_GATE_ROW) {
        const float z = elem_load<BK>(P.gate, t);
        ga = P.sigmoid ? sigmoid_of(z) : z;
      }
      // s: y^2, the sum behind mean(dm y) without beta, and behind the row's gate
      float s[3] = {0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < C; ++j) {
        const int c = c0 + j * NT * 8;
        float w[8];
        row_load8<BK, VEC>(P.y, row + c, P.H - c, y[j]);
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = 1.f;
        if (P.w_post) weight_load8<SK, VEC>(P.w_post, P.wf32, c, P.H - c, w);
        float z[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] = ga;
        if (P.gate_kind == CQ_GATE_ELEM) {
          row_load8<BK, VEC>(P.gate, row + c, P.H - c, z);
#pragma unroll
          for (int i = 0; i < 8; ++i) z[i] = P.sigmoid ? sigmoid_of(z[i]) : z[i];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float dw = d[j][i] * w[i];
          s[0] = fmaf(y[j][i], y[j][i], s[0]);
          s[1] = fmaf(dw * z[i], y[j][i], s[1]);
          s[2] = fmaf(dw, y[j][i], s[2]);
        }
      }
      float q = 1.f, back = 0.f;
      if (P.w_post || P.gate_kind == CQ_GATE_ROW) group_sum<NT, 3>(s, lds[set][1]);
      if (P.w_post) {
        q = 1.f / sqrtf(s[0] * inv_H + P.eps);
        back = q * q * s[1] * inv_H;
      }
      if (P.gate_kind == CQ_GATE_ROW && G.dgate && threadIdx.x == 0) {
        float da = P.beta * q * s[2];
        if (P.sigmoid) da *= ga * (1.f - ga);
        elem_store<BK>(G.dgate, t, da);
      }
#pragma unroll
      for (int j = 0; j < C; ++j) {
        const int c = c0 + j * NT * 8;
        float w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = 1.f;
        if (P.w_post) weight_load8<SK, VEC>(P.w_post, P.wf32, c, P.H - c, w);
        float z[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] = ga;
        if (P.gate_kind == CQ_GATE_ELEM) {
          float da[8];
          row_load8<BK, VEC>(P.gate, row + c, P.H - c, z);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            z[i] = P.sigmoid ? sigmoid_of(z[i]) : z[i];
            da[i] = P.beta * d[j][i] * y[j][i] * q * w[i];
            if (P.sigmoid) da[i] *= z[i] * (1.f - z[i]);
          }
          if (G.dgate) row_store8<BK, VEC>(G.dgate, row + c, P.H - c, da);
        }
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float du = P.beta * z[i] * d[j][i];
          acc_post[j][i] = fmaf(du, y[j][i] * q, acc_post[j][i]);
          v[i] = q * fmaf(-back * P.beta, y[j][i], du * w[i]);
        }
        row_store8<BK, VEC>(G.dy, row + c, P.H - c, v);
      }
    }
  }
  // (the workspace's rows are padded to whole groups of eight)
  const int Hp = (P.H + 7) & ~7;
#pragma unroll
  for (int j = 0; j < C; ++j) {
    const int c = c0 + j * NT * 8;
    if (G.part_pre) row_store8<CQ_A_F32, true>(G.part_pre, (size_t)blockIdx.x * Hp + c, P.H - c, acc_pre[j]);
    if (G.part_post) row_store8<CQ_A_F32, true>(G.part_post, (size_t)blockIdx.x * Hp + c, P.H - c, acc_post[j]);
  }
}

template <int WK>
__global__ __launch_bounds__(256) void weight_sum_kernel(const float* part_pre, const float* part_post, int parts, int H,
                                                         void* dw_pre, void* dw_post) {
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= H) return;
  const int Hp = (H + 7) & ~7;
  const float* p = blockIdx.y == 0 ? part_pre : part_post;
  void* out = blockIdx.y == 0 ? dw_pre : dw_post;
  if (!out) return;
  float s = 0.f;
  for (int b = 0; b < parts; ++b) s += p[(size_t)b * Hp + c];
  elem_store<WK>(out, c, s);
}

}  // namespace

extern "C" size_t cq_block_norm_grad_workspace_bytes(const cq_block_norm_spec* P, int T) {
  if (check_norm_spec(P, T) != CQ_OK) return 0;
  return 2 * cq_align_up((size_t)grad_parts(T) * ((P->H + 7) & ~7) * 4, 256);
}

extern "C" cq_status cq_block_norm_grad(const cq_block_norm_spec* P, const void* h, const void* y, const void* gate,
                                        const void* d_h_out, const void* d_x, int T, void* d_h, void* d_y, void* d_gate,
                                        void* d_w_pre, void* d_w_post, void* workspace, size_t workspace_bytes,
                                        cq_stream stream) {
  const cq_status st = check_norm_spec(P, T);
  if (st != CQ_OK) return st;
  if (T > 0) {
    if ((!d_h_out && !d_x) || !d_h || (y && !d_y)) return CQ_ERR_NULL;
    if (d_x && (!h || !P->w_pre)) return CQ_ERR_NULL;
    if (y && P->gate_kind != CQ_GATE_NONE && !gate) return CQ_ERR_NULL;
    if (!workspace && (d_w_pre || d_w_post)) return CQ_ERR_WORKSPACE;
  }
  if ((d_w_pre && !d_x && T > 0) || (d_w_post && (!P->w_post || (!y && T > 0)))) return CQ_ERR_NULL;
  if ((d_w_pre || d_w_post) && workspace_bytes < cq_block_norm_grad_workspace_bytes(P, T)) return CQ_ERR_WORKSPACE;
  if (T == 0 && !d_w_pre && !d_w_post) return CQ_OK;
  hipStream_t s = (hipStream_t)stream;
  norm_grad_args a;
  a.f = make_norm_args(P, T, h, y, gate);
  a.parts = grad_parts(T);
  a.dh_out = d_h_out;
  a.dx = d_x;
  a.dh = d_h;
  a.dy = d_y;
  a.dgate = d_gate;
  a.part_pre = d_w_pre ? (float*)workspace : nullptr;
  a.part_post = d_w_post ? (float*)((char*)workspace + cq_block_norm_grad_workspace_bytes(P, T) / 2) : nullptr;
  if (T > 0) {
    const bool elem = a.f.gate_kind == CQ_GATE_ELEM;
    const void* const rows[] = {d_x ? h : nullptr, y, elem ? gate : nullptr, d_h_out, d_x, d_h, y ? d_y : nullptr,
                                elem ? d_gate : nullptr, d_x ? P->w_pre : nullptr, a.f.w_post};
    const bool vec = rows_aligned(P->H, rows, 10);
#define LAUNCH(SK, BK, NT, C, VEC) \
  hipLaunchKernelGGL((block_norm_grad_kernel<SK, BK, NT, C, VEC>), dim3(a.parts), dim3(NT), 0, s, a)
    CQ_NORM_DISPATCH(LAUNCH, P->stream_kind, P->block_kind, vec, P->H);
#undef LAUNCH
  }
  if (d_w_pre || d_w_post) {
    const dim3 grid((P->H + 255) / 256, 2);
#define SUM(WK) \
  hipLaunchKernelGGL((weight_sum_kernel<WK>), grid, dim3(256), 0, s, a.part_pre, a.part_post, a.parts, P->H, d_w_pre, d_w_post)
    if (P->weight_kind == CQ_A_F32) SUM(CQ_A_F32);
    else if (P->weight_kind == CQ_A_F16) SUM(CQ_A_F16);
    else SUM(CQ_A_BF16);
#undef SUM
  }
  return cq_check_launch();
}
