// Load-balancing loss of a router over sequences, with per-expert counts, and its gradient:
//   p_t = softmax(z_t),  f_se = c_se / (k n_s),  P_se = mean of p_te over the n_s tokens of sequence s that count,
//   L = alpha / S' sum_s E sum_e f_se P_se (S' sequences with a token),   dz_te = g alpha E / (S' n_s) p_te (f_se - sum_j f_sj p_tj).
// Tokens are taken in tiles of kTile.  A tile's share of a sequence goes to slot  tile + sequence  of the workspace: from one
// pair to the next in order either the tile or the sequence grows by one at least, so the slots differ, and a second launch
// adds every sequence's slots in order.  Counts are integers added in LDS; no atomics on floats, no global atomics.
#include <math.h>

#include "cq_rows.h"

namespace {

constexpr int kTile = 64;
constexpr int kMaxExperts = 1024;

struct balance_args {
  const void* z;
  const int32_t *ids, *offsets;
  const uint8_t* mask;
  int T, E, k, S;
  float alpha;
};

__device__ __forceinline__ int offset_at(const balance_args& P, int s) {
  if (!P.offsets) return s == 0 ? 0 : P.T;
  const int o = P.offsets[s];
  return o < 0 ? 0 : (o > P.T ? P.T : o);
}

// the sequence that token t lies in: the last one that begins at or before it (-1: none does)
__device__ __forceinline__ int sequence_of(const balance_args& P, int t) {
  int lo = 0, hi = P.S;   // offsets[lo - 1] <= t < offsets[hi] in a non-decreasing list
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (offset_at(P, mid) <= t) lo = mid + 1;
    else hi = mid;
  }
  return lo - 1;
}

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
  return v;
}

// p_t of one token in a wavefront: lane l holds experts l, l + 64, ...  A row without a logit above -inf has p = 0.
template <int KIND, int C>
__device__ __forceinline__ void softmax_row(const balance_args& P, int t, int lane, float (&p)[C]) {
  float m = -INFINITY;
#pragma unroll
  for (int j = 0; j < C; ++j) {
    const int e = lane + j * 64;
    p[j] = e < P.E ? elem_load<KIND>(P.z, (size_t)t * P.E + e) : -INFINITY;
    m = fmaxf(m, p[j]);
  }
  m = wave_max(m);
  float sum = 0.f;
#pragma unroll
  for (int j = 0; j < C; ++j) {
    p[j] = m == -INFINITY && !(p[j] != p[j]) ? 0.f : expf(p[j] - m);
    sum += p[j];
  }
  sum = wave_sum(sum);
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
  for (int j = 0; j < C; ++j) p[j] *= inv;
}

// workspace: per slot probability sums [E] f32, counts [E] i32, tokens i32; per sequence its loss f32
struct balance_ws {
  float* probs;
  int32_t *counts, *tokens;
  float* loss;
};

template <int KIND, int C>
__global__ __launch_bounds__(256) void balance_tile_kernel(balance_args P, balance_ws W) {
  __shared__ float lds_p[4][kMaxExperts];
  __shared__ int lds_c[kMaxExperts];
  __shared__ int lds_n;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int t0 = blockIdx.x * kTile, t1 = min(P.T, t0 + kTile);
  int s = sequence_of(P, t0);
  if (s < 0) s = 0;
  for (; s < P.S; ++s) {
    const int a0 = offset_at(P, s), b0 = offset_at(P, s + 1);
    if (a0 >= t1) break;
    const int a = max(a0, t0), b = min(b0, t1);
    if (a >= b) continue;
    for (int e = threadIdx.x; e < P.E; e += 256) lds_c[e] = 0;
    if (threadIdx.x == 0) lds_n = 0;
    __syncthreads();
    float acc[C];
#pragma unroll
    for (int j = 0; j < C; ++j) acc[j] = 0.f;
    for (int t = a + wave; t < b; t += 4) {
      if (P.mask && !P.mask[t]) continue;
      if (lane == 0) atomicAdd(&lds_n, 1);
      if (lane < P.k) {
        const int id = P.ids[(size_t)t * P.k + lane];
        if (id >= 0 && id < P.E) atomicAdd(&lds_c[id], 1);
      }
      float p[C];
      softmax_row<KIND, C>(P, t, lane, p);
#pragma unroll
      for (int j = 0; j < C; ++j) acc[j] += p[j];
    }
#pragma unroll
    for (int j = 0; j < C; ++j)
      if (lane + j * 64 < P.E) lds_p[wave][lane + j * 64] = acc[j];
    __syncthreads();
    const size_t slot = (size_t)blockIdx.x + s;
    for (int e = threadIdx.x; e < P.E; e += 256) {
      W.probs[slot * P.E + e] = (lds_p[0][e] + lds_p[1][e]) + (lds_p[2][e] + lds_p[3][e]);
      W.counts[slot * P.E + e] = lds_c[e];
    }
    if (threadIdx.x == 0) W.tokens[slot] = lds_n;
    __syncthreads();
  }
}

__global__ __launch_bounds__(256) void balance_sequence_kernel(balance_args P, balance_ws W, int32_t* counts, float* probs,
                                                               int32_t* tokens) {
  __shared__ float lds[4];
  const int s = blockIdx.x;
  const int a = offset_at(P, s), b = offset_at(P, s + 1);
  const int i0 = a / kTile, i1 = b > a ? (b - 1) / kTile : i0 - 1;
  int n = 0;
  for (int i = i0; i <= i1; ++i) n += W.tokens[(size_t)i + s];
  float loss[1] = {0.f};
  for (int e = threadIdx.x; e < P.E; e += 256) {
    float p = 0.f;
    int c = 0;
    for (int i = i0; i <= i1; ++i) {
      p += W.probs[((size_t)i + s) * P.E + e];
      c += W.counts[((size_t)i + s) * P.E + e];
    }
    p = n > 0 ? p / (float)n : 0.f;
    probs[(size_t)s * P.E + e] = p;
    counts[(size_t)s * P.E + e] = c;
    if (n > 0) loss[0] = fmaf((float)c / ((float)P.k * (float)n), p, loss[0]);
  }
  group_sum<256, 1>(loss, lds);
  if (threadIdx.x == 0) {
    tokens[s] = n;
    W.loss[s] = loss[0];
  }
}

__global__ __launch_bounds__(256) void balance_total_kernel(balance_args P, balance_ws W, int32_t* tokens, float* loss) {
  __shared__ float lds[4];
  __shared__ int lds_used;
  if (threadIdx.x == 0) lds_used = 0;
  __syncthreads();
  float sum[1] = {0.f};
  int used = 0;
  for (int s = threadIdx.x; s < P.S; s += 256) {
    sum[0] += W.loss[s];
    used += tokens[s] > 0;
  }
  if (used) atomicAdd(&lds_used, used);
  group_sum<256, 1>(sum, lds);
  if (threadIdx.x == 0) {
    tokens[P.S] = lds_used;
    loss[0] = lds_used > 0 ? P.alpha * (float)P.E * sum[0] / (float)lds_used : 0.f;
  }
}

template <int KIND, int C>
__global__ __launch_bounds__(256) void balance_grad_kernel(balance_args P, const int32_t* counts, const int32_t* tokens,
                                                           const float* d_loss, void* dz) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int t = blockIdx.x * 4 + wave;
  if (t >= P.T) return;
  const int s = sequence_of(P, t);
  const bool counted = s >= 0 && t < offset_at(P, s + 1) && !(P.mask && !P.mask[t]);
  float p[C];
#pragma unroll
  for (int j = 0; j < C; ++j) p[j] = 0.f;
  if (counted) {
    softmax_row<KIND, C>(P, t, lane, p);
    const int n = tokens[s];
    const float per = n > 0 ? 1.f / ((float)P.k * (float)n) : 0.f;
    float f[C], dot = 0.f;
#pragma unroll
    for (int j = 0; j < C; ++j) {
      const int e = lane + j * 64;
      f[j] = e < P.E ? (float)counts[(size_t)s * P.E + e] * per : 0.f;
      dot = fmaf(f[j], p[j], dot);
    }
    dot = wave_sum(dot);
    const int used = tokens[P.S];
    const float w = (d_loss ? d_loss[0] : 1.f) * (n > 0 && used > 0 ? P.alpha * (float)P.E / ((float)used * (float)n) : 0.f);
#pragma unroll
    for (int j = 0; j < C; ++j) p[j] = w * p[j] * (f[j] - dot);
  }
#pragma unroll
  for (int j = 0; j < C; ++j)
    if (lane + j * 64 < P.E) elem_store<KIND>(dz, (size_t)t * P.E + lane + j * 64, p[j]);
}

cq_status check_balance(int logit_kind, const int32_t* offsets, int S, int T, int E, int k) {
  if (T < 0 || E <= 0 || E > kMaxExperts || k <= 0 || k > E || k > 64 || S <= 0) return CQ_ERR_SHAPE;
  if (!offsets && S != 1) return CQ_ERR_NULL;
  if (!cq_row_kind(logit_kind)) return CQ_ERR_UNSUPPORTED;
  return CQ_OK;
}

size_t slots_of(int T, int S) { return (size_t)(T + kTile - 1) / kTile + S; }

#define CQ_BALANCE_WIDTHS(LAUNCH, KIND, E)      \
  do {                                          \
    if ((E) <= 64) LAUNCH(KIND, 1);             \
    else if ((E) <= 128) LAUNCH(KIND, 2);       \
    else if ((E) <= 256) LAUNCH(KIND, 4);       \
    else LAUNCH(KIND, 16);                      \
  } while (0)
#define CQ_BALANCE_DISPATCH(LAUNCH, kind, E)                               \
  do {                                                                     \
    if ((kind) == CQ_A_F32) CQ_BALANCE_WIDTHS(LAUNCH, CQ_A_F32, E);        \
    else if ((kind) == CQ_A_F16) CQ_BALANCE_WIDTHS(LAUNCH, CQ_A_F16, E);   \
    else CQ_BALANCE_WIDTHS(LAUNCH, CQ_A_BF16, E);                          \
  } while (0)

}  // namespace

extern "C" size_t cq_balance_loss_workspace_bytes(int T, int E, int n_seqs) {
  if (T < 0 || E <= 0 || E > kMaxExperts || n_seqs <= 0) return 0;
  const size_t slots = slots_of(T, n_seqs);
  return 2 * cq_align_up(slots * E * 4, 256) + cq_align_up(slots * 4, 256) + cq_align_up((size_t)n_seqs * 4, 256);
}

extern "C" cq_status cq_balance_loss(const void* logits, int logit_kind, const int32_t* topk_ids, const int32_t* seq_offsets,
                                     int n_seqs, const uint8_t* token_mask, int T, int E, int top_k, float alpha, float* loss,
                                     int32_t* counts, float* probs, int32_t* tokens, void* workspace, size_t workspace_bytes,
                                     cq_stream stream) {
  const cq_status st = check_balance(logit_kind, seq_offsets, n_seqs, T, E, top_k);
  if (st != CQ_OK) return st;
  if ((T > 0 && (!logits || !topk_ids)) || !loss || !counts || !probs || !tokens) return CQ_ERR_NULL;
  if (!workspace || workspace_bytes < cq_balance_loss_workspace_bytes(T, E, n_seqs)) return CQ_ERR_WORKSPACE;
  hipStream_t s = (hipStream_t)stream;
  const balance_args P = {logits, topk_ids, seq_offsets, token_mask, T, E, top_k, n_seqs, alpha};
  const size_t slots = slots_of(T, n_seqs);
  balance_ws W;
  char* at = (char*)workspace;
  W.probs = (float*)at;
  at += cq_align_up(slots * E * 4, 256);
  W.counts = (int32_t*)at;
  at += cq_align_up(slots * E * 4, 256);
  W.tokens = (int32_t*)at;
  at += cq_align_up(slots * 4, 256);
  W.loss = (float*)at;
  if (T > 0) {
#define LAUNCH(KIND, C) \
  hipLaunchKernelGGL((balance_tile_kernel<KIND, C>), dim3((T + kTile - 1) / kTile), dim3(256), 0, s, P, W)
    CQ_BALANCE_DISPATCH(LAUNCH, logit_kind, E);
#undef LAUNCH
  }
  hipLaunchKernelGGL(balance_sequence_kernel, dim3(n_seqs), dim3(256), 0, s, P, W, counts, probs, tokens);
  hipLaunchKernelGGL(balance_total_kernel, dim3(1), dim3(256), 0, s, P, W, tokens, loss);
  return cq_check_launch();
}

extern "C" cq_status cq_balance_loss_grad(const void* logits, int logit_kind, const int32_t* counts, const int32_t* tokens,
                                          const int32_t* seq_offsets, int n_seqs, const uint8_t* token_mask, int T, int E,
                                          int top_k, float alpha, const float* d_loss, void* d_logits, cq_stream stream) {
  const cq_status st = check_balance(logit_kind, seq_offsets, n_seqs, T, E, top_k);
  if (st != CQ_OK) return st;
  if (T == 0) return CQ_OK;
  if (!logits || !counts || !tokens || !d_logits) return CQ_ERR_NULL;
  const balance_args P = {logits, nullptr, seq_offsets, token_mask, T, E, top_k, n_seqs, alpha};
#define LAUNCH(KIND, C)                                                                                                \
  hipLaunchKernelGGL((balance_grad_kernel<KIND, C>), dim3((T - 1) / 4 + 1), dim3(256), 0, (hipStream_t)stream, P, counts, \
                     tokens, d_loss, d_logits)
  CQ_BALANCE_DISPATCH(LAUNCH, logit_kind, E);
#undef LAUNCH
  return cq_check_launch();
}
