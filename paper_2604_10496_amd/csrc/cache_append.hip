// New tokens' keys and values into the pages of a cache, with the norm and the rotation of keys (and of the queries beside them) on
// the way.  Bound by HBM for prompts, by latency for single tokens: a wavefront asks for its rows first and finds the token's
// sequence, position and page while they are under way.  Every page number is checked before its page is touched.
// 9 prompts, 4096 tokens of 32 + 8 + 8 heads of 128 in f16 (101 MB): 22.6 us = 4.45 TB/s (three groups in flight 22.9, six 24.4; two wavefronts per
// token 24.6).  1 token in bf16: 5.5 us; 64 tokens, fp32 into e4m3: 6.4.
#include "cache.h"

namespace {

constexpr int kGroups = 2;   // groups of rows in flight

struct append_args {
  head_layout L;
  int T, first, parts, per_part, groups_q, groups_k, groups, wkind;   // tokens first .. first + T - 1
  float eps, rot_scale, inv_D;
  const double* freq;
  const void *w_q, *w_k;
  const int32_t *positions, *offsets;
  head_rows q, k, v, q_out;
  cache_args C;
};

// Sequence of token t: the last that begins at or before it.  64 offsets at a time: two rounds of loads for up to 4096 sequences.
__device__ __forceinline__ int sequence_of(const int32_t* offsets, int n_seqs, int t, int lane) {
  int lo = 0, hi = n_seqs;   // it is one of lo .. hi-1
  while (hi - lo > 1) {
    const int step = (hi - lo + 63) / 64;
    const int s = lo + lane * step;
    const bool before = s < hi && offsets[s] <= t;
    const int n = __popcll(__ballot(before));
    if (n == 0) return lo;
    lo += (n - 1) * step;
    hi = min(hi, lo + step);
  }
  return lo;
}

// where a token's key goes.  seq -1: the token is in no sequence or not in its table's row; page -1: its page is not there
struct place {
  int seq, position, page, slot;
};
__device__ __forceinline__ place place_of(const append_args& A, int t, int lane) {
  place p = {-1, 0, -1, 0};
  int seq = t, back = 1;   // back: how far the token is from the end of its sequence
  if (A.offsets) {
    seq = sequence_of(A.offsets, A.C.n_seqs, t, lane);
    const int begin = A.offsets[seq], end = A.offsets[seq + 1];
    if (t < begin || t >= end) return p;
    back = end - t;
  }
  p.position = A.C.lengths[seq] - back;
  if (p.position < 0) return p;
  const int column = p.position / A.C.page_size;
  if (column >= A.C.width) return p;
  p.seq = seq;
  const int page = A.C.table[seq * A.C.table_stride + column];
  p.slot = p.position - column * A.C.page_size;
  if (page >= 0 && page < A.C.pages) p.page = page;
  return p;
}

template <int XK, int CK, int LANES, int MODE, bool INTER>
__global__ __launch_bounds__(256) void cache_append_kernel(append_args A) {
  constexpr int kAtOnce = 64 / LANES;
  const int unit = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
  const int in_launch = unit / A.parts;
  if (in_launch >= A.T) return;
  const int t = A.first + in_launch;
  int group = (unit - in_launch * A.parts) * A.per_part;
  const int end = min(A.groups, group + A.per_part);
  const int lane = threadIdx.x & 63, sub = lane / LANES;
  const head_slot s = make_slot<MODE>(A.L, lane % LANES);
  // which rows a group holds: 0 queries, 1 keys, 2 values, from head h0 on
  auto what = [&](int g, int& h0) {
    const int which = g < A.groups_q ? 0 : g < A.groups_k ? 1 : 2;
    h0 = (g - (which == 0 ? 0 : which == 1 ? A.groups_q : A.groups_k)) * kAtOnce;
    return which;
  };
  head_raw<XK> raw[kGroups];
  auto fetch = [&](int first) {
#pragma unroll
    for (int i = 0; i < kGroups; ++i) {
      int h0;
      const int which = what(first + i, h0);
      const head_rows& R = which == 0 ? A.q : which == 1 ? A.k : A.v;
      raw[i] = head_fetch<XK, MODE, INTER>(R.p, t * R.token + h0 * R.head + sub * R.head, s, first + i < end && h0 + sub < R.n);
    }
  };
  fetch(group);
  const place to = place_of(A, t, lane);
  if (to.seq < 0) return;   // (nothing is written, the queries neither)
  const head_turn turn = turn_of(A.L, s, A.freq, A.rot_scale, A.positions ? A.positions[t] : to.position);
  float w_q[8], w_k[8];
  head_weights<MODE, INTER>(A.w_q, A.wkind, s, w_q);
  head_weights<MODE, INTER>(A.w_k, A.wkind, s, w_k);
  const long at = to.page * A.C.page + to.slot * A.C.slot;
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
      int h0;
      const int which = what(group + i, h0), h = h0 + sub;
      if (which == 0) {
        if (A.w_q) head_normed<LANES>(v[i], w_q, A.inv_D, A.eps);
      } else if (which == 1) {
        if (A.w_k) head_normed<LANES>(v[i], w_k, A.inv_D, A.eps);
      }
      if (which < 2) turn_values<INTER, false>(s, turn, v[i]);
      if (group + i >= end) break;
      if (which == 0) {
        if (h < A.q.n) head_store<XK, MODE, INTER>(const_cast<void*>(A.q_out.p), t * A.q_out.token + h * A.q_out.head, s, v[i]);
      } else if (to.page >= 0 && h < A.C.heads) {
        if constexpr (CK == CQ_C_E4M3) {
          const float* scale = which == 2 ? A.C.v_scale : A.C.k_scale;
          if (scale) {
            const float sc = scale[h];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] /= sc;
          }
        }
        head_store<CK, MODE, INTER>(which == 2 ? A.C.v : A.C.k, at + h * A.C.head, s, v[i]);
      }
    }
  }
}

}  // namespace

extern "C" cq_status cq_cache_append(const cq_cache* C, const cq_sequences* S, const cq_head_spec* P, const cq_heads* q,
                                     const cq_heads* k, const cq_heads* v, const int32_t* seq_offsets, const int32_t* positions, int T,
                                     const cq_heads* q_out, cq_stream stream) {
  cq_status st = check_cache(C);
  if (st != CQ_OK || (st = check_sequences(S, C)) != CQ_OK) return st;
  cq_head_spec none = {};
  none.D = C->D;
  none.rot_scale = 1.f;
  if (!P) P = &none;
  if ((st = check_head_spec(P)) != CQ_OK) return st;
  if (T < 0 || T > 1 << 30 || P->D != C->D) return CQ_ERR_SHAPE;
  if (!k || !v) return CQ_ERR_NULL;
  if ((st = check_heads(q, T)) != CQ_OK || (st = check_heads(k, T)) != CQ_OK || (st = check_heads(v, T)) != CQ_OK) return st;
  if ((st = check_heads_out(q, q_out, T, P->D)) != CQ_OK) return st;
  if (k->n != C->heads || v->n != C->heads) return CQ_ERR_SHAPE;
  if (v->kind != k->kind || (q && (q->kind != k->kind || q_out->kind != q->kind))) return CQ_ERR_UNSUPPORTED;
  if (!seq_offsets && T != S->n) return CQ_ERR_SHAPE;
  if (T == 0 || S->n == 0) return CQ_OK;
  append_args a;
  a.C = make_cache_args(C, S);
  a.L = make_head_layout(P->D, P->rot, P->interleaved != 0);
  a.wkind = P->weight_kind;
  a.eps = P->eps;
  a.rot_scale = P->rot_scale;
  a.inv_D = 1.f / (float)P->D;
  a.freq = P->freq;
  a.w_q = q ? P->w_q : nullptr;
  a.w_k = P->w_k;
  a.positions = positions;
  a.offsets = seq_offsets;
  a.q = make_head_rows(q);
  a.k = make_head_rows(k);
  a.v = make_head_rows(v);
  a.q_out = make_head_rows(q ? q_out : nullptr);
  a.groups_q = head_groups(a.q.n, a.L);
  a.groups_k = a.groups_q + head_groups(a.k.n, a.L);
  a.groups = a.groups_k + head_groups(a.v.n, a.L);
  share_groups(a.groups, T, 2048, a.per_part, a.parts);
  const long most = (kMostThreads / 64 / a.parts) & ~3l;
  for (long from = 0; from < T; from += most) {
    append_args b = a;
    b.first = (int)from;
    b.T = (int)(T - from < most ? T - from : most);
    const dim3 grid((unsigned)(((long)b.T * b.parts + 3) / 4));
#define LAUNCH(XK, CK, LANES, MODE, INTER) \
  hipLaunchKernelGGL((cache_append_kernel<XK, CK, LANES, MODE, INTER>), grid, dim3(256), 0, (hipStream_t)stream, b)
#define KINDS(XK)                                                              \
  do {                                                                         \
    if (C->kind == CQ_A_F16) CQ_HEAD_LANES(LAUNCH, a.L, XK, CQ_A_F16);   \
    else if (C->kind == CQ_A_BF16) CQ_HEAD_LANES(LAUNCH, a.L, XK, CQ_A_BF16); \
    else CQ_HEAD_LANES(LAUNCH, a.L, XK, CQ_C_E4M3);                      \
  } while (0)
    if (k->kind == CQ_A_F32) KINDS(CQ_A_F32);
    else if (k->kind == CQ_A_F16) KINDS(CQ_A_F16);
    else KINDS(CQ_A_BF16);
#undef KINDS
#undef LAUNCH
  }
  return cq_check_launch();
}
