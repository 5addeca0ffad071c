// Norms of queries and keys for each head with the rotation by position, one pass.  Bound by HBM (a row in, a row out).
// A wavefront takes one token and some or all of its heads, so that the angles are computed once for all of them, and asks for the next two
// groups of rows before it works on these.
// 4096 tokens of 32 + 8 heads of 128, fp32 -> bf16 (126 MB): 24.5 us = 5.1 TB/s, a copy's rate (one group in flight 24.4, four 29.5; two
// wavefronts per token 32).  1 token in bf16: 4.2 us (four groups 5.0).
#include "heads.h"

namespace {

constexpr int kGroups = 2;   // groups of rows in flight

struct head_norm_args {
  head_layout L;
  int T, parts, per_part, groups_q, groups, wkind;
  float eps, rot_scale, inv_D;
  const double* freq;
  const void *w_q, *w_k;
  const int32_t* positions;
  head_rows q, k, q_out, k_out;
};

template <int XK, int OK, int LANES, int MODE, bool INTER>
__global__ __launch_bounds__(256) void head_norm_kernel(head_norm_args A) {
  constexpr int kAtOnce = 64 / LANES;
  const int unit = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
  const int t = unit / A.parts;
  if (t >= A.T) return;
  int group = (unit - t * A.parts) * A.per_part;
  const int end = min(A.groups, group + A.per_part);
  const int lane = threadIdx.x & 63, sub = lane / LANES;
  const head_slot s = make_slot<MODE>(A.L, lane % LANES);
  head_raw<XK> raw[kGroups];
  auto fetch = [&](int first) {
#pragma unroll
    for (int i = 0; i < kGroups; ++i) {
      const bool key = first + i >= A.groups_q;
      const head_rows& R = key ? A.k : A.q;
      const int h0 = (first + i - (key ? A.groups_q : 0)) * kAtOnce;
      raw[i] = head_fetch<XK, MODE, INTER>(R.p, t * R.token + h0 * R.head + sub * R.head, s, first + i < end && h0 + sub < R.n);
    }
  };
  fetch(group);
  const head_turn turn = turn_of(A.L, s, A.freq, A.rot_scale, A.L.rot ? A.positions[t] : 0);
  float w_q[8], w_k[8];
  head_weights<MODE, INTER>(A.w_q, A.wkind, s, w_q);
  head_weights<MODE, INTER>(A.w_k, A.wkind, s, w_k);
  for (; group < end; group += kGroups) {
    float v[kGroups][8];
#pragma unroll
    for (int i = 0; i < kGroups; ++i) {
      head_values<XK>(raw[i], v[i]);
      own_values<MODE>(s, v[i]);
    }
    if (group + kGroups < end) fetch(group + kGroups);
#pragma unroll
    for (int i = 0; i < kGroups; ++i) {
      const bool key = group + i >= A.groups_q;
      const head_rows& R = key ? A.k_out : A.q_out;
      const int h0 = (group + i - (key ? A.groups_q : 0)) * kAtOnce;
      if (key ? A.w_k : A.w_q) {
        if (key) head_normed<LANES>(v[i], w_k, A.inv_D, A.eps);
        else head_normed<LANES>(v[i], w_q, A.inv_D, A.eps);
      }
      turn_values<INTER, false>(s, turn, v[i]);
      if (group + i < end && h0 + sub < R.n)
        head_store<OK, MODE, INTER>(const_cast<void*>(R.p), t * R.token + h0 * R.head + sub * R.head, s, v[i]);
    }
  }
}

}  // namespace

extern "C" cq_status cq_head_norm(const cq_head_spec* P, const cq_heads* q, const cq_heads* k, const int32_t* positions, int T,
                                  const cq_heads* q_out, const cq_heads* k_out, cq_stream stream) {
  cq_status st = check_head_spec(P);
  if (st != CQ_OK) return st;
  if (T < 0 || T > 1 << 30) return CQ_ERR_SHAPE;
  if (!q && !k) return CQ_ERR_NULL;
  if ((st = check_heads(q, T)) != CQ_OK || (st = check_heads(k, T)) != CQ_OK) return st;
  if ((st = check_heads_out(q, q_out, T, P->D)) != CQ_OK || (st = check_heads_out(k, k_out, T, P->D)) != CQ_OK) return st;
  const int kind = q ? q->kind : k->kind, out = q ? q_out->kind : k_out->kind;
  if ((q && k && (k->kind != kind || k_out->kind != out)) || (out != kind && kind != CQ_A_F32)) return CQ_ERR_UNSUPPORTED;
  if (T == 0) return CQ_OK;
  if (P->rot > 0 && !positions) return CQ_ERR_NULL;
  head_norm_args a;
  a.L = make_head_layout(P->D, P->rot, P->interleaved != 0);
  a.wkind = P->weight_kind;
  a.eps = P->eps;
  a.rot_scale = P->rot_scale;
  a.inv_D = 1.f / (float)P->D;
  a.freq = P->freq;
  a.w_q = q ? P->w_q : nullptr;
  a.w_k = k ? P->w_k : nullptr;
  a.q = make_head_rows(q);
  a.k = make_head_rows(k);
  a.q_out = make_head_rows(q ? q_out : nullptr);
  a.k_out = make_head_rows(k ? k_out : nullptr);
  a.groups_q = head_groups(a.q.n, a.L);
  a.groups = a.groups_q + head_groups(a.k.n, a.L);
  share_groups(a.groups, T, 2048, a.per_part, a.parts);
  const long most = (kMostThreads / 64 / a.parts) & ~3l;
  for (long from = 0; from < T; from += most) {
    head_norm_args b = a;
    b.T = (int)(T - from < most ? T - from : most);
    b.positions = positions ? positions + from : nullptr;
    b.q = rows_from(a.q, kind, from);
    b.k = rows_from(a.k, kind, from);
    b.q_out = rows_from(a.q_out, out, from);
    b.k_out = rows_from(a.k_out, out, from);
    const dim3 grid((unsigned)(((long)b.T * b.parts + 3) / 4));
#define LAUNCH(XK, OK, LANES, MODE, INTER) \
  hipLaunchKernelGGL((head_norm_kernel<XK, OK, LANES, MODE, INTER>), grid, dim3(256), 0, (hipStream_t)stream, b)
    if (kind == CQ_A_F16) CQ_HEAD_LANES(LAUNCH, a.L, CQ_A_F16, CQ_A_F16);
    else if (kind == CQ_A_BF16) CQ_HEAD_LANES(LAUNCH, a.L, CQ_A_BF16, CQ_A_BF16);
    else if (out == CQ_A_F32) CQ_HEAD_LANES(LAUNCH, a.L, CQ_A_F32, CQ_A_F32);
    else if (out == CQ_A_F16) CQ_HEAD_LANES(LAUNCH, a.L, CQ_A_F32, CQ_A_F16);
    else CQ_HEAD_LANES(LAUNCH, a.L, CQ_A_F32, CQ_A_BF16);
#undef LAUNCH
  }
  return cq_check_launch();
}
