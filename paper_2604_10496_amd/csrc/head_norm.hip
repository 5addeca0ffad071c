// Norms of queries and keys for each head with the rotation by position, one pass.  Bound by HBM (a row in, a row out).
// A wavefront takes one token and some or all of its heads, so that the angles are computed once for all of them.
#include "heads.h"

namespace {

constexpr int kRows = 4;   // rows of a lane in flight

struct head_norm_args {
  head_layout L;
  int T, parts, rows_per_part, wkind;
  float eps, rot_scale, inv_D;
  const double* freq;
  const void *w_q, *w_k;
  const int32_t* positions;
  head_rows q, k, q_out, k_out;
};

template <int XK, int OK, int LANES>
__global__ __launch_bounds__(256) void head_norm_kernel(head_norm_args A) {
  constexpr int kAtOnce = 64 / LANES;
  const int unit = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
  const int t = unit / A.parts, part = unit - t * A.parts;
  if (t >= A.T) return;
  const int lane = threadIdx.x & 63;
  const head_slot s(A.L, lane % LANES);
  const int rows = A.q.n + A.k.n, end = min(rows, (part + 1) * A.rows_per_part);
  int row = part * A.rows_per_part + lane / LANES;
  head_raw<XK> raw[kRows];
  auto fetch = [&](int first) {
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      const int r = first + i * kAtOnce;
      const bool key = r >= A.q.n;
      const long at = key ? t * A.k.token + (r - A.q.n) * A.k.head : t * A.q.token + r * A.q.head;
      raw[i] = head_fetch<XK>(key ? A.k.p : A.q.p, at, s, r < end);
    }
  };
  fetch(row);
  const head_turn turn = turn_of(A.L, s, A.freq, A.rot_scale, A.L.rot ? A.positions[t] : 0);
  float w_q[8], w_k[8];
  head_weights(A.w_q, A.wkind, s, w_q);
  head_weights(A.w_k, A.wkind, s, w_k);
  // (the condition is the wavefront's, so that all lanes of a row sum are there)
  for (int first = part * A.rows_per_part; first < end; first += kRows * kAtOnce, row += kRows * kAtOnce) {
    float v[kRows][8];
#pragma unroll
    for (int i = 0; i < kRows; ++i) head_values<XK>(raw[i], v[i]);
    if (first + kRows * kAtOnce < end) fetch(row + kRows * kAtOnce);
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      const int r = row + i * kAtOnce;
      const bool key = r >= A.q.n;
      if (A.w_q || A.w_k) {
        float w[8], plain[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          w[e] = key ? w_k[e] : w_q[e];
          plain[e] = v[i][e];
        }
        head_normed<LANES>(v[i], w, A.inv_D, A.eps);
        if (!(key ? A.w_k : A.w_q)) {
#pragma unroll
          for (int e = 0; e < 8; ++e) v[i][e] = plain[e];
        }
      }
      turn_values<false>(A.L, s, turn, v[i]);
      if (r < end) {
        const long at = key ? t * A.k_out.token + (r - A.q.n) * A.k_out.head : t * A.q_out.token + r * A.q_out.head;
        head_store<OK>(const_cast<void*>(key ? A.k_out.p : A.q_out.p), at, s, v[i]);
      }
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
  // Few tokens: their heads on several wavefronts, one instruction's rows at a time.
  const int rows = a.q.n + a.k.n, at_once = 64 / a.L.lanes;
  int parts = 1;
  while (parts * 2 * at_once <= rows + at_once && (long)T * parts < 2048) parts *= 2;
  a.rows_per_part = (int)((cq_align_up((size_t)((rows + parts - 1) / parts), at_once)));
  a.parts = (rows + a.rows_per_part - 1) / a.rows_per_part;
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
#define LAUNCH(XK, OK, LANES) hipLaunchKernelGGL((head_norm_kernel<XK, OK, LANES>), grid, dim3(256), 0, (hipStream_t)stream, b)
    if (kind == CQ_A_F16) CQ_HEAD_LANES(LAUNCH, a.L.lanes, CQ_A_F16, CQ_A_F16);
    else if (kind == CQ_A_BF16) CQ_HEAD_LANES(LAUNCH, a.L.lanes, CQ_A_BF16, CQ_A_BF16);
    else if (out == CQ_A_F32) CQ_HEAD_LANES(LAUNCH, a.L.lanes, CQ_A_F32, CQ_A_F32);
    else if (out == CQ_A_F16) CQ_HEAD_LANES(LAUNCH, a.L.lanes, CQ_A_F32, CQ_A_F16);
    else CQ_HEAD_LANES(LAUNCH, a.L.lanes, CQ_A_F32, CQ_A_BF16);
#undef LAUNCH
  }
  return cq_check_launch();
}
