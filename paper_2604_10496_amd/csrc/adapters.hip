// Low-rank adapters of many requests beside a projection that they share:
//   out_t = base_t + scale_a B_a (A_a x_t),  a = ids[t];   a outside [0, adapters): out_t = base_t.
#include "cq_rows.h"

namespace {

constexpr int kMaxRank = 256;

struct adapter_args {
  const void *A, *B, *X, *base;
  const float* scale;
  const int32_t *ranks, *ids;
  void* out;
  float* low;   // [T][rank] A x
  int M, R, K, N, T;
  size_t ldx, ldb, ldo;
};

__device__ __forceinline__ int rank_of(const adapter_args& P, int a) {
  if (!P.ranks) return P.R;
  const int r = P.ranks[a];
  return r < 0 ? 0 : (r > P.R ? P.R : r);
}

__device__ __forceinline__ float kind_load(int kind, const void* p, size_t at) {
  if (kind == CQ_A_F32) return elem_load<CQ_A_F32>(p, at);
  if (kind == CQ_A_F16) return elem_load<CQ_A_F16>(p, at);
  return elem_load<CQ_A_BF16>(p, at);
}

// one wavefront per (token, row of A)
__global__ __launch_bounds__(64) void adapter_down_kernel(adapter_args P, int x_kind, int w_kind) {
  const int t = blockIdx.x, r = blockIdx.y;
  const int a = P.ids[t];
  if (a < 0 || a >= P.M || r >= rank_of(P, a)) return;
  float s = 0.f;
  const size_t row = ((size_t)a * P.R + r) * P.K;
  for (int k = threadIdx.x; k < P.K; k += 64)
    s = fmaf(kind_load(x_kind, P.X, t * P.ldx + k), kind_load(w_kind, P.A, row + k), s);
  s = wave_sum(s);
  if (threadIdx.x == 0) P.low[(size_t)t * P.R + r] = s;
}

// one thread per output
__global__ __launch_bounds__(256) void adapter_up_kernel(adapter_args P, int w_kind, int o_kind) {
  const int t = blockIdx.x, n = blockIdx.y * 256 + threadIdx.x;
  if (n >= P.N) return;
  float v = P.base ? kind_load(o_kind, P.base, t * P.ldb + n) : 0.f;
  const int a = P.ids[t];
  if (a >= 0 && a < P.M) {
    float s = 0.f;
    const int rank = rank_of(P, a);
    for (int r = 0; r < rank; ++r)
      s = fmaf(P.low[(size_t)t * P.R + r], kind_load(w_kind, P.B, ((size_t)a * P.N + n) * P.R + r), s);
    v = fmaf(P.scale ? P.scale[a] : 1.f, s, v);
  }
  if (o_kind == CQ_A_F32) elem_store<CQ_A_F32>(P.out, t * P.ldo + n, v);
  else if (o_kind == CQ_A_F16) elem_store<CQ_A_F16>(P.out, t * P.ldo + n, v);
  else elem_store<CQ_A_BF16>(P.out, t * P.ldo + n, v);
}

cq_status check_adapters(const cq_adapters* W, int T) {
  if (!W) return CQ_ERR_NULL;
  if (T < 0 || W->n <= 0 || W->rank <= 0 || W->rank > kMaxRank || W->K <= 0 || W->N <= 0) return CQ_ERR_SHAPE;
  if (W->N > 65535 * 256) return CQ_ERR_SHAPE;
  if (!cq_row_kind(W->kind)) return CQ_ERR_UNSUPPORTED;
  return CQ_OK;
}

}  // namespace

extern "C" size_t cq_adapter_workspace_bytes(const cq_adapters* W, int T) {
  if (check_adapters(W, T) != CQ_OK) return 0;
  return cq_align_up((size_t)T * W->rank * 4, 256);
}

extern "C" cq_status cq_adapter_apply(const cq_adapters* W, const void* X, int x_kind, long ldx, const int32_t* adapter_ids, int T,
                                      const void* base, long ld_base, void* out, int out_kind, long ld_out, void* workspace,
                                      size_t workspace_bytes, cq_stream stream) {
  const cq_status st = check_adapters(W, T);
  if (st != CQ_OK) return st;
  if (!cq_row_kind(x_kind) || !cq_row_kind(out_kind)) return CQ_ERR_UNSUPPORTED;
  if (T == 0) return CQ_OK;
  if (!W->A || !W->B || !X || !adapter_ids || !out) return CQ_ERR_NULL;
  if (ldx < W->K || ld_out < W->N || (base && ld_base < W->N)) return CQ_ERR_SHAPE;
  if (!workspace || workspace_bytes < cq_adapter_workspace_bytes(W, T)) return CQ_ERR_WORKSPACE;
  adapter_args P;
  P.A = W->A;
  P.B = W->B;
  P.X = X;
  P.base = base;
  P.scale = W->scale;
  P.ranks = W->ranks;
  P.ids = adapter_ids;
  P.out = out;
  P.low = (float*)workspace;
  P.M = W->n;
  P.R = W->rank;
  P.K = W->K;
  P.N = W->N;
  P.T = T;
  P.ldx = (size_t)ldx;
  P.ldb = (size_t)ld_base;
  P.ldo = (size_t)ld_out;
  hipStream_t s = (hipStream_t)stream;
  hipLaunchKernelGGL(adapter_down_kernel, dim3(T, W->rank), dim3(64), 0, s, P, x_kind, W->kind);
  hipLaunchKernelGGL(adapter_up_kernel, dim3(T, (W->N + 255) / 256), dim3(256), 0, s, P, W->kind, out_kind);
  return cq_check_launch();
}
