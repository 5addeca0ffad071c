// Gradients of the norms around a block, from h' as stored, y, the gate and the gradients of h' and x.  Per row, with
//   r = 1 / sqrt(mean h'^2 + eps), n = h' r, dn = dx w_pre:     D  = dh' + r (dn - n mean(dn n)),   dh = rho D,  dw_pre += dx n
//   q = 1 / sqrt(mean y^2 + eps),  m = y q,  u = m w_post, a:   du = beta a D,  da = beta u D,      dw_post += du m,
//                                                               dm = du w_post,  dy = q (dm - m mean(dm m)).
// The sums of squares are taken again, together with mean(dn h') in the first of two row sums and with the sum behind a row's
// gate in the second, so that the forward pass keeps no statistics.
// Bound by HBM (five or six rows in, two or three out).  One workgroup of 1024 threads per compute unit takes 1024 / NT rows at
// a time and, where registers allow it (16-bit stream and block, up to 8192 values), asks for the next ones before it works on these, so
// that loads are in flight across the two barriers of a row sum.  A gate per token is waited for in front of its row's loads.
// The shares of the weights' gradients stay in registers, are added over a workgroup's rows in LDS and go to the workspace
// once, [parts][H] each; a second launch adds the parts in order.  No atomics: the results do not depend on timing.
// 8192 x 4096 in bf16 with a gate per value, 537 MB: 106 us = 5.1 TB/s, and 4.8 us for the sum of the parts; a sigmoid gate's
// exponentials and quotients make it 136 together.  Without the next rows in flight, one row per workgroup of 512 threads, 141 us.
// 2048 x 2048: 19.0 and 3.9 us (with a gate per token 1.4 more), two rounds of rows, in which the first loads, the weights and the
// shares at the end weigh as much as the rows.  4096 x 4096, bf16 stream, fp32 block, gate per token (no rows in flight), 302 MB: 69 us.
#include "block_norm.h"

namespace {

constexpr int kThreads = 1024;
constexpr int kMostParts = 256;   // one workgroup per compute unit

inline int grad_parts(int T) { return T < kMostParts ? T : kMostParts; }

struct norm_grad_args {
  norm_args f;
  int parts;
  const void *dh_out, *dx;
  void *dh, *dy, *dgate;
  float *part_pre, *part_post;
};

// what a thread reads of one row (ELEM: the gate has one value per value of the row)
template <int SK, int BK, int C, bool ELEM>
struct grad_row {
  row8<SK> dh[C], h[C];
  row8<BK> dx[C], y[C], gate[ELEM ? C : 1];
  float z;   // the row's own gate
};

template <int SK, int BK, int NT, int C, bool ELEM>
__device__ __forceinline__ void fetch_row(const norm_grad_args& G, int t, grad_row<SK, BK, C, ELEM>& R) {
  const norm_args& P = G.f;
  const bool in = t < P.T;
  const size_t row = (size_t)t * P.H;
  R.z = 1.f;
  if (P.gate_kind == CQ_GATE_ROW && in) R.z = elem_load<BK>(P.gate, t);
#pragma unroll
  for (int j = 0; j < C; ++j) {
    const row_slot s((threadIdx.x % NT + j * NT) * 8, P.H);
    R.h[j] = slot_fetch<SK>(P.h, row, s, P.H, in && G.dx);
    R.dx[j] = slot_fetch<BK>(G.dx, row, s, P.H, in && G.dx);
    R.dh[j] = slot_fetch<SK>(G.dh_out, row, s, P.H, in && G.dh_out);
    R.y[j] = slot_fetch<BK>(P.y, row, s, P.H, in && P.y);
    if constexpr (ELEM) R.gate[j] = slot_fetch<BK>(P.gate, row, s, P.H, in);
  }
}

template <int SK, int BK, int NT, int C, bool ELEM>
__global__ __launch_bounds__(kThreads) void block_norm_grad_kernel(norm_grad_args G) {
  constexpr int kGroups = kThreads / NT;
  // rows of 32 bits, of several groups of eight, and the widest of one group with a gate per value leave no registers for the next row
  constexpr bool kAhead = C == 1 && SK != CQ_A_F32 && BK != CQ_A_F32 && !(ELEM && NT == 1024);
  // Rows of several groups of eight are read again where they are used again (out of the caches) instead of held.  again(): the
  // compiler takes the pointer as a new one, so that it does not hold them, or the weights from row to row, after all.  The shares
  // of the weights' gradients and the row's own gradient still need more than the 128 registers of a lane: 116 to 188 bytes of a lane
  // spill up to 16384 values, 560 to 750 beyond (1024 x 16384, both norms: 125 us for a floor of 39).
  constexpr bool kHold = C == 1;
  auto again = [](const void* p) {
    asm volatile("" : "+s"(p));
    return p;
  };
  const norm_args& P = G.f;
  const int H = P.H;
  // (two sets, used by rows in turn: a row's sums are read while the next row's may be written already)
  __shared__ float sums[2][2][3 * (kThreads / 64)];
  // Both weights, where each thread has its own eight in its own place: loads of them from memory would wait for the next
  // rows', which were asked for before.  Later the rows' shares of the weights' gradients.
  __shared__ __align__(16) float lds[C > 1 ? 4 : (NT * 16 > kThreads * 8 || kGroups == 1 ? NT * 16 : kThreads * 8)];
  auto slot = [&](int j) { return row_slot((threadIdx.x % NT + j * NT) * 8, H); };
  auto weights = [&](const void* w, int which, int j, float (&v)[8]) {
    if constexpr (C == 1) {
      const cq_v4f* q = reinterpret_cast<const cq_v4f*>(&lds[(which * NT + threadIdx.x % NT) * 8]);
      const cq_v4f a = q[0], b = q[1];
#pragma unroll
      for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
    } else {
      slot_weights<SK>(again(w), P.wf32, slot(j), H, v);
    }
  };
  if constexpr (C == 1) {
    if (threadIdx.x < NT) {
      float w[2][8];
#pragma unroll
      for (int i = 0; i < 8; ++i) w[0][i] = w[1][i] = 1.f;
      if (G.dx) slot_weights<SK>(P.w_pre, P.wf32, slot(0), H, w[0]);
      if (P.w_post) slot_weights<SK>(P.w_post, P.wf32, slot(0), H, w[1]);
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int i = 0; i < 8; ++i) lds[(n * NT + threadIdx.x) * 8 + i] = w[n][i];
    }
    __syncthreads();
  }
  // rows part, part + parts, ...: first one row for every workgroup, then the second of each, so that few rows spread out
  int t = __builtin_amdgcn_readfirstlane((threadIdx.x / NT) * G.parts + blockIdx.x);   // (one row per wavefront)
  const float inv_H = 1.f / (float)H;
  float acc_pre[C][8], acc_post[C][8];
#pragma unroll
  for (int j = 0; j < C; ++j)
#pragma unroll
    for (int i = 0; i < 8; ++i) acc_pre[j][i] = acc_post[j][i] = 0.f;
  grad_row<SK, BK, C, ELEM> R, next;
  if constexpr (kAhead) fetch_row<SK, BK, NT, C, ELEM>(G, t, next);
  int set = 0;
  for (int first = blockIdx.x; first < P.T; first += kGroups * G.parts, t += kGroups * G.parts, set ^= 1) {
    if constexpr (kAhead) {
      R = next;
      if (first + kGroups * G.parts < P.T) fetch_row<SK, BK, NT, C, ELEM>(G, t + kGroups * G.parts, next);
    } else if constexpr (kHold) {
      fetch_row<SK, BK, NT, C, ELEM>(G, t, R);
    } else {
      R.z = P.gate_kind == CQ_GATE_ROW && t < P.T ? elem_load<BK>(P.gate, t) : 1.f;
    }
    const bool in = t < P.T;
    const size_t row = (size_t)t * H;
    float d[C][8];   // gradient that reaches h'
#pragma unroll
    for (int j = 0; j < C; ++j) {
      if constexpr (kHold)
        slot_values<SK>(R.dh[j], slot(j), H, d[j]);
      else
        slot_values<SK>(slot_fetch<SK>(G.dh_out, row, slot(j), H, in && G.dh_out), slot(j), H, d[j]);
    }
    auto stream_of = [&](int j, float (&h)[8], float (&dx)[8]) {
      if constexpr (kHold) {
        slot_values<SK>(R.h[j], slot(j), H, h);
        slot_values<BK>(R.dx[j], slot(j), H, dx);
      } else {
        slot_values<SK>(slot_fetch<SK>(again(P.h), row, slot(j), H, in), slot(j), H, h);
        slot_values<BK>(slot_fetch<BK>(again(G.dx), row, slot(j), H, in), slot(j), H, dx);
      }
    };
    if (G.dx) {
      float s[2] = {0.f, 0.f};   // h'^2, dx w h'
#pragma unroll
      for (int j = 0; j < C; ++j) {
        float w[8], h[8], dx[8];
        weights(P.w_pre, 0, j, w);
        stream_of(j, h, dx);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          s[0] = fmaf(h[i], h[i], s[0]);
          s[1] = fmaf(dx[i] * w[i], h[i], s[1]);
        }
      }
      group_sum<NT, 2>(s, sums[set][0]);
      const float r = 1.f / sqrtf(s[0] * inv_H + P.eps);
      const float back = r * r * s[1] * inv_H;   // D = dh' + r (dn - h' r^2 mean(dn h'))
#pragma unroll
      for (int j = 0; j < C; ++j) {
        if constexpr (kHold) {
          forget_values(R.h[j]);
          forget_values(R.dx[j]);
        }
        float w[8], h[8], dx[8];
        weights(P.w_pre, 0, j, w);
        stream_of(j, h, dx);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          d[j][i] = fmaf(r, fmaf(-back, h[i], dx[i] * w[i]), d[j][i]);
          acc_pre[j][i] = fmaf(dx[i], h[i] * r, acc_pre[j][i]);
        }
      }
    }
    const float rho = P.y ? P.rho : 1.f;
#pragma unroll
    for (int j = 0; j < C; ++j) {
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = rho * d[j][i];
      slot_store<SK>(G.dh, row, slot(j), H, in, v);
    }
    if (!P.y) continue;
    float row_slope = 1.f;
    const float ga = P.gate_kind == CQ_GATE_ROW && P.sigmoid ? sigmoid_of(R.z, row_slope) : R.z;
    // y, u's weight and the gate of eight values with its slope
    auto factors = [&](int j, float (&y)[8], float (&w)[8], float (&a)[8], float (&slope)[8]) {
      if constexpr (kHold)
        slot_values<BK>(R.y[j], slot(j), H, y);
      else
        slot_values<BK>(slot_fetch<BK>(again(P.y), row, slot(j), H, in), slot(j), H, y);
      if (C == 1 || P.w_post) {
        weights(P.w_post, 1, j, w);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = 1.f;
      }
      if constexpr (ELEM) {
        if constexpr (kHold)
          row_values<BK>(R.gate[j], a);
        else
          row_values<BK>(slot_fetch<BK>(again(P.gate), row, slot(j), H, in), a);
#pragma unroll
        for (int i = 0; i < 8; ++i) slope[i] = 1.f;
        if (P.sigmoid) {
#pragma unroll
          for (int i = 0; i < 8; ++i) a[i] = sigmoid_of(a[i], slope[i]);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) a[i] = ga;
      }
    };
    // y^2, the sum behind mean(dm y) without beta, and behind the row's gate
    float q = 1.f, back = 0.f;
    if (P.w_post || P.gate_kind == CQ_GATE_ROW) {
      float s[3] = {0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < C; ++j) {
        float y[8], w[8], a[8], slope[8];
        factors(j, y, w, a, slope);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float dw = d[j][i] * w[i];
          s[0] = fmaf(y[i], y[i], s[0]);
          s[1] = fmaf(dw * a[i], y[i], s[1]);
          s[2] = fmaf(dw, y[i], s[2]);
        }
      }
      group_sum<NT, 3>(s, sums[set][1]);
      if (P.w_post) {
        q = 1.f / sqrtf(s[0] * inv_H + P.eps);
        back = P.beta * q * q * s[1] * inv_H;
      }
      if (P.gate_kind == CQ_GATE_ROW && G.dgate && in && threadIdx.x % NT == 0) {
        const float da = P.beta * q * s[2];
        elem_store<BK>(G.dgate, t, da * row_slope);
      }
    }
#pragma unroll
    for (int j = 0; j < C; ++j) {
      if constexpr (kHold) {
        forget_values(R.y[j]);
        if constexpr (ELEM) forget_values(R.gate[j]);
      }
      float y[8], w[8], a[8], slope[8], v[8];
      factors(j, y, w, a, slope);
      if (ELEM && G.dgate) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = P.beta * d[j][i] * y[i] * q * w[i] * slope[i];
        slot_store<BK>(G.dgate, row, slot(j), H, in, v);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float du = P.beta * a[i] * d[j][i];
        acc_post[j][i] = fmaf(du, y[i] * q, acc_post[j][i]);
        v[i] = q * fmaf(-back, y[i], du * w[i]);
      }
      slot_store<BK>(G.dy, row, slot(j), H, in, v);
    }
  }
  // a workgroup's share: over its rows in LDS (one weight after the other), then to the workspace, rows of whole groups of eight
  const int Hp = (H + 7) & ~7;
  auto give = [&](float* part, float (&acc)[C][8]) {
    if (!part) return;
    if constexpr (kGroups == 1) {
#pragma unroll
      for (int j = 0; j < C; ++j) slot_store<CQ_A_F32>(part, (size_t)blockIdx.x * Hp, slot(j), H, true, acc[j]);
    } else {
      static_assert(C == 1, "several rows at a time are rows of one group of eight per thread");
      const row_slot s = slot(0);
      __syncthreads();
      if (s.on) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (i >= s.skip) lds[(threadIdx.x / NT * NT) * 8 + s.c + i] = acc[0][i];
      }
      __syncthreads();
      for (int c = threadIdx.x; c < H; c += kThreads) {
        float v = 0.f;
#pragma unroll
        for (int g = 0; g < kGroups; ++g) v += lds[g * NT * 8 + c];
        part[(size_t)blockIdx.x * Hp + c] = v;
      }
    }
  };
  give(G.part_pre, acc_pre);
  give(G.part_post, acc_post);
}

// d_w[c] = sum of the parts in order: 32 columns per workgroup, every eighth of 32 groups of threads takes four of them
template <int WK>
__global__ __launch_bounds__(256) void weight_sum_kernel(const float* part_pre, const float* part_post, int parts, int H,
                                                         void* dw_pre, void* dw_post) {
  __shared__ float lds[32][33];
  const float* p = blockIdx.y == 0 ? part_pre : part_post;
  void* out = blockIdx.y == 0 ? dw_pre : dw_post;
  if (!out) return;
  const int Hp = (H + 7) & ~7, c = blockIdx.x * 32 + (threadIdx.x & 7) * 4, g = threadIdx.x >> 3;
  cq_v4f s = {0.f, 0.f, 0.f, 0.f};
  if (c < Hp) {   // (what lies between H and Hp is read and not used)
#pragma unroll 8
    for (int b = g; b < parts; b += 32) s += *reinterpret_cast<const cq_v4f*>(p + (size_t)b * Hp + c);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) lds[g][(threadIdx.x & 7) * 4 + i] = s[i];
  __syncthreads();
  if (threadIdx.x < 32 && blockIdx.x * 32 + threadIdx.x < H) {
    float v = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) v += lds[i][threadIdx.x];
    elem_store<WK>(out, blockIdx.x * 32 + threadIdx.x, v);
  }
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
#define LAUNCH(SK, BK, NT, C)                                                                                            \
  do {                                                                                                                  \
    if (a.f.gate_kind == CQ_GATE_ELEM)                                                                                  \
      hipLaunchKernelGGL((block_norm_grad_kernel<SK, BK, NT, C, true>), dim3(a.parts), dim3(kThreads), 0, s, a);         \
    else                                                                                                                \
      hipLaunchKernelGGL((block_norm_grad_kernel<SK, BK, NT, C, false>), dim3(a.parts), dim3(kThreads), 0, s, a);        \
  } while (0)
    CQ_NORM_DISPATCH(LAUNCH, P->stream_kind, P->block_kind, P->H);
#undef LAUNCH
  }
  if (d_w_pre || d_w_post) {
    const dim3 grid((P->H + 31) / 32, 2);
#define SUM(WK) \
  hipLaunchKernelGGL((weight_sum_kernel<WK>), grid, dim3(256), 0, s, a.part_pre, a.part_post, a.parts, P->H, d_w_pre, d_w_post)
    if (P->weight_kind == CQ_A_F32) SUM(CQ_A_F32);
    else if (P->weight_kind == CQ_A_F16) SUM(CQ_A_F16);
    else SUM(CQ_A_BF16);
#undef SUM
  }
  return cq_check_launch();
}
