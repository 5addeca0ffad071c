// Load-balancing loss of a router over sequences, with per-expert counts, and its gradient:
//   p_t = softmax(z_t),  f_se = c_se / (k n_s),  P_se = mean of p_te over the n_s tokens of sequence s that count,
//   L = alpha / S' sum_s E sum_e f_se P_se (S' sequences with a token),   dz_te = g alpha E / (S' n_s) p_te (f_se - sum_j f_sj p_tj).
// One pass over the logits in either direction, bound by HBM for long batches and by latency for the others.  L lanes share a
// token (four neighbouring experts each), so that a wavefront reads 64 / L tokens in one contiguous load, and works on the logits of
// several loads at a time (asked for one behind the other without a mask; with one, each waits for its tokens' mask bytes).
// Forward: tokens are taken in tiles.  A tile's share of a sequence goes to slot  tile + sequence  of the workspace: from one
// pair to the next in order either the tile or the sequence grows by one at least, so the slots differ, and a second launch
// adds every sequence's slots in a fixed order; its last workgroup adds the sequences' losses.  Counts are integers added in LDS;
// no atomics on floats.  Few logits take one workgroup and one launch.
// 8192 x 64 in 13 sequences with padding 8.4 + 5.4 us (2.3 MB: latency), 64 x 4 5.9 us; the gradient of 65536 x 128 18.3 us for 67 MB =
// 3.7 TB/s.
#include <math.h>

#include "cq_rows.h"

namespace {

constexpr int kMaxExperts = 1024;
constexpr int kMostSequences = 1 << 26;   // (their workgroups of the second launch are counted in 32 bits)

struct balance_args {
  const void* z;
  const int32_t *ids, *offsets;
  const uint8_t* mask;
  int T, E, k, S, tile;
  int first;   // first workgroup of this launch (the gradient, the sums over sequences)
  float alpha;
};

// workspace: per slot probability sums [E] f32, counts [E] i32, tokens i32; per sequence and 32 experts a loss f32; a counter
struct balance_ws {
  float* probs;
  int32_t *counts, *tokens;
  float* loss;
  uint32_t* done;
};

__device__ __forceinline__ int offset_at(const balance_args& P, int s) {
  if (!P.offsets) return s == 0 ? 0 : P.T;
  const int o = P.offsets[s];
  return o < 0 ? 0 : (o > P.T ? P.T : o);
}

// The offsets around a token: sequence_of finds the last sequence that begins at or before token t (-1: none does; t is the same in
// the whole wavefront) and keeps the 64 offsets it has loaded for offset().
struct offset_window {
  const balance_args& P;
  int base, here;   // offsets base .. base+63, one per lane
  __device__ __forceinline__ explicit offset_window(const balance_args& args) : P(args) { load(0); }
  __device__ __forceinline__ void load(int first) {
    base = first;
    const int s = first + (int)(threadIdx.x & 63);
    here = s <= P.S ? offset_at(P, s) : 0x7fffffff;
  }
  __device__ __forceinline__ int sequence_of(int t) {
    int n = 0;
    for (;;) {
      const int found = __popcll(__ballot(base + (int)(threadIdx.x & 63) < P.S && here <= t));
      n += found;
      if (found < 64 || base + 64 >= P.S) return n - 1;
      load(base + 64);
    }
  }
  __device__ __forceinline__ int offset(int s) {   // 0 <= s <= S, the same in the whole wavefront
    if (s < base || s >= base + 64) load(s);
    return __builtin_amdgcn_readlane(here, s - base);
  }
};

// four consecutive values, the first `left` of which exist; the others read as -inf
template <int KIND>
__device__ __forceinline__ void load4(const void* p, size_t at, int left, float (&v)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = -INFINITY;
  if (left >= 4) {
    if constexpr (KIND == CQ_A_F32) {
      const cq_v4u w = *reinterpret_cast<const cq_v4u_any*>(reinterpret_cast<const float*>(p) + at);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(w[i]);
    } else {
      typedef __attribute__((__vector_size__(8))) uint16_t v4h;
      typedef v4h v4h_any __attribute__((aligned(2)));
      const v4h w = *reinterpret_cast<const v4h_any*>(reinterpret_cast<const uint16_t*>(p) + at);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        v[i] = KIND == CQ_A_BF16 ? __uint_as_float((uint32_t)w[i] << 16) : (float)__builtin_bit_cast(_Float16, (uint16_t)w[i]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 3; ++i)
      if (i < left) v[i] = elem_load<KIND>(p, at + i);
  }
}

template <int KIND>
__device__ __forceinline__ void store4(void* p, size_t at, int left, const float (&v)[4]) {
  if (left >= 4) {
    if constexpr (KIND == CQ_A_F32) {
      *reinterpret_cast<cq_v4u_any*>(reinterpret_cast<float*>(p) + at) =
          cq_v4u{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
    } else {
      typedef __attribute__((__vector_size__(8))) uint16_t v4h;
      typedef v4h v4h_any __attribute__((aligned(2)));
      v4h w;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        w[i] = KIND == CQ_A_BF16 ? __builtin_bit_cast(uint16_t, (__bf16)v[i]) : __builtin_bit_cast(uint16_t, (_Float16)v[i]);
      *reinterpret_cast<v4h_any*>(reinterpret_cast<uint16_t*>(p) + at) = w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 3; ++i)
      if (i < left) elem_store<KIND>(p, at + i, v[i]);
  }
}

// sum and maximum over the L lanes of a token
template <int L>
__device__ __forceinline__ float token_sum(float v) {
#pragma unroll
  for (int o = L / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}
template <int L>
__device__ __forceinline__ float token_max(float v) {
#pragma unroll
  for (int o = L / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
  return v;
}

// logits -> probabilities of a token; lane i of its L lanes holds experts 4 i + 4 L j ...  A token without a logit above -inf
// has no probabilities: zeros.
template <int L, int C>
__device__ __forceinline__ void softmax_token(float (&p)[C][4]) {
  float m = -INFINITY;
#pragma unroll
  for (int j = 0; j < C; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) m = fmaxf(m, p[j][i]);
  m = token_max<L>(m);
  const float from = m == -INFINITY ? 0.f : m;   // (exp(-inf) = 0; a NaN stays one)
  float sum = 0.f;
#pragma unroll
  for (int j = 0; j < C; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      p[j][i] = expf(p[j][i] - from);
      sum += p[j][i];
    }
  sum = token_sum<L>(sum);
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
  for (int j = 0; j < C; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) p[j][i] *= inv;
}

template <int NT, int L, int C>
struct segment_lds {
  float p[NT / 64][L * C * 4];   // per wavefront
  int c[kMaxExperts < L * C * 4 ? kMaxExperts : L * C * 4];
  int n;
};

// the sums over a workgroup of what its lanes hold for their experts, into S.p; no barrier
template <int NT, int L, int C>
__device__ __forceinline__ void give_probs(const float (&acc)[C][4], segment_lds<NT, L, C>& S) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, e0 = (lane % L) * 4;
#pragma unroll
  for (int j = 0; j < C; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float v = acc[j][i];
#pragma unroll
      for (int o = L; o < 64; o <<= 1) v += __shfl_xor(v, o, 64);
      if (lane < L) S.p[wave][e0 + j * L * 4 + i] = v;
    }
}

// Tokens [a, b) of one sequence: probability sums per wavefront, counts and the tokens that count, into LDS.  Ends with a barrier.
template <int KIND, int NT, int L, int C>
__device__ __forceinline__ void segment(const balance_args& P, int a, int b, segment_lds<NT, L, C>& S) {
  constexpr int U = C == 1 ? 4 : 1;   // loads in flight
  const int lane = threadIdx.x & 63, e0 = (lane % L) * 4;
  for (int e = threadIdx.x; e < P.E; e += NT) S.c[e] = 0;
  if (threadIdx.x == 0) S.n = P.mask ? 0 : b - a;
  __syncthreads();
  float acc[C][4];
#pragma unroll
  for (int j = 0; j < C; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[j][i] = 0.f;
  for (int t0 = a; t0 < b; t0 += U * (NT / L)) {
    float p[U][C][4];
    bool in[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int t = t0 + u * (NT / L) + threadIdx.x / L;
      in[u] = t < b && (!P.mask || P.mask[t]);
#pragma unroll
      for (int j = 0; j < C; ++j) {
        const int e = e0 + j * L * 4;
        load4<KIND>(P.z, (size_t)t * P.E + e, in[u] ? P.E - e : 0, p[u][j]);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      softmax_token<L, C>(p[u]);
#pragma unroll
      for (int j = 0; j < C; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[j][i] += p[u][j][i];
    }
    if (P.mask) {
      int n = 0;
#pragma unroll
      for (int u = 0; u < U; ++u) n += __popcll(__ballot(in[u] && lane % L == 0));
      if (lane == 0 && n) atomicAdd(&S.n, n);
    }
  }
  const int assignments = (b - a) * P.k;
  for (int i = threadIdx.x; i < assignments; i += NT) {
    if (P.mask && !P.mask[a + i / P.k]) continue;
    const int id = P.ids[(size_t)a * P.k + i];
    if (id >= 0 && id < P.E) atomicAdd(&S.c[id], 1);
  }
  give_probs<NT, L, C>(acc, S);
  __syncthreads();
}

template <int L, int C>
__device__ __forceinline__ void write_slot(const balance_args& P, const balance_ws& W, size_t slot, const segment_lds<256, L, C>& S) {
  for (int e = threadIdx.x; e < P.E; e += 256) {
    W.probs[slot * P.E + e] = (S.p[0][e] + S.p[1][e]) + (S.p[2][e] + S.p[3][e]);
    W.counts[slot * P.E + e] = S.c[e];
  }
  if (threadIdx.x == 0) W.tokens[slot] = S.n;
}

// Tiles of one round of loads: a tile's logits and ids are read once, in front of its sequences, which then take their tokens out of
// the registers.  Bound by latency, and by more of it than two dependent loads: the offsets, each of four mask bytes and each of four ids
// (and its token's mask byte) are tested inside a branch of their own, and waited for there.
template <int KIND, int L>
__global__ __launch_bounds__(256) void balance_tile_kernel(balance_args P, balance_ws W) {
  constexpr int U = 4, kTokens = U * (256 / L), kIds = 4;
  __shared__ segment_lds<256, L, 1> lds;
  if (blockIdx.x == 0 && threadIdx.x == 0) *W.done = 0;
  const int lane = threadIdx.x & 63, e0 = (lane % L) * 4;
  const int t0 = blockIdx.x * kTokens, t1 = min(P.T, t0 + kTokens);
  offset_window offsets(P);
  float p[U][1][4];
  bool in[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int t = t0 + u * (256 / L) + threadIdx.x / L;
    in[u] = t < t1 && (!P.mask || P.mask[t]);
    load4<KIND>(P.z, (size_t)t * P.E + e0, t < t1 ? P.E - e0 : 0, p[u][0]);
  }
  // the first ids of a thread (all of them for up to 1024 assignments), -1 where the token is left out
  const int assignments = (t1 - t0) * P.k;
  auto id_of = [&](int i) {
    const int id = P.ids[(size_t)t0 * P.k + i];
    return (!P.mask || P.mask[t0 + i / P.k]) && id >= 0 && id < P.E ? id : -1;
  };
  int ids[kIds];
#pragma unroll
  for (int n = 0; n < kIds; ++n) ids[n] = (int)threadIdx.x + n * 256 < assignments ? id_of(threadIdx.x + n * 256) : -1;
#pragma unroll
  for (int u = 0; u < U; ++u) softmax_token<L, 1>(p[u]);
  for (int s = max(offsets.sequence_of(t0), 0); s < P.S; ++s) {
    const int a0 = offsets.offset(s), b0 = offsets.offset(s + 1);
    if (a0 >= t1) break;
    const int a = max(a0, t0), b = min(b0, t1);
    if (a >= b) continue;
    for (int e = threadIdx.x; e < P.E; e += 256) lds.c[e] = 0;
    if (threadIdx.x == 0) lds.n = 0;
    __syncthreads();
    float acc[1][4] = {{0.f, 0.f, 0.f, 0.f}};
    int n = 0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int t = t0 + u * (256 / L) + threadIdx.x / L;
      const bool mine = in[u] && t >= a && t < b;
      n += __popcll(__ballot(mine && lane % L == 0));
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[0][i] += mine ? p[u][0][i] : 0.f;
    }
    if (lane == 0 && n) atomicAdd(&lds.n, n);
    const int from = (a - t0) * P.k, to = (b - t0) * P.k;
#pragma unroll
    for (int q = 0; q < kIds; ++q) {
      const int i = threadIdx.x + q * 256;
      if (ids[q] >= 0 && i >= from && i < to) atomicAdd(&lds.c[ids[q]], 1);
    }
    for (int i = threadIdx.x + kIds * 256; i < to; i += 256) {
      const int id = i >= from ? id_of(i) : -1;
      if (id >= 0) atomicAdd(&lds.c[id], 1);
    }
    give_probs<256, L, 1>(acc, lds);
    __syncthreads();
    write_slot<L, 1>(P, W, (size_t)blockIdx.x + s, lds);
    __syncthreads();
  }
}

// Tiles of any size, sequence after sequence.
template <int KIND, int L, int C>
__global__ __launch_bounds__(256) void balance_long_tile_kernel(balance_args P, balance_ws W) {
  __shared__ segment_lds<256, L, C> lds;
  if (blockIdx.x == 0 && threadIdx.x == 0) *W.done = 0;
  const int t0 = blockIdx.x * P.tile, t1 = min(P.T, t0 + P.tile);
  offset_window offsets(P);
  for (int s = max(offsets.sequence_of(t0), 0); s < P.S; ++s) {
    const int a0 = offsets.offset(s), b0 = offsets.offset(s + 1);
    if (a0 >= t1) break;
    const int a = max(a0, t0), b = min(b0, t1);
    if (a >= b) continue;
    segment<KIND, 256, L, C>(P, a, b, lds);
    write_slot<L, C>(P, W, (size_t)blockIdx.x + s, lds);
    __syncthreads();
  }
}

// Few logits: everything in one workgroup, sequence after sequence.
template <int KIND, int L, int C>
__global__ __launch_bounds__(1024) void balance_one_kernel(balance_args P, int32_t* counts, float* probs, int32_t* tokens, float* loss) {
  __shared__ segment_lds<1024, L, C> lds;
  __shared__ float sums[16];
  float total[1] = {0.f};
  int used = 0;
  for (int s = 0; s < P.S; ++s) {
    const int a = offset_at(P, s), b = max(a, offset_at(P, s + 1));
    segment<KIND, 1024, L, C>(P, a, b, lds);
    const int n = lds.n;
    used += n > 0;
    if (threadIdx.x < P.E) {
      const int e = threadIdx.x;
      float p = 0.f;
#pragma unroll
      for (int w = 0; w < 16; ++w) p += lds.p[w][e];
      p = n > 0 ? p / (float)n : 0.f;
      probs[(size_t)s * P.E + e] = p;
      counts[(size_t)s * P.E + e] = lds.c[e];
      if (n > 0) total[0] = fmaf((float)lds.c[e] / ((float)P.k * (float)n), p, total[0]);
    }
    if (threadIdx.x == 0) tokens[s] = n;
    __syncthreads();
  }
  group_sum<1024, 1>(total, sums);
  if (threadIdx.x == 0) {
    tokens[P.S] = used;
    loss[0] = used > 0 ? P.alpha * (float)P.E * total[0] / (float)used : 0.f;
  }
}

// One workgroup per sequence and 32 experts: 32 threads take its slots in turn for every expert.  The workgroup that ends last
// adds the losses.
__global__ __launch_bounds__(1024) void balance_sequence_kernel(balance_args P, balance_ws W, int32_t* counts, float* probs,
                                                                int32_t* tokens, float* loss) {
  __shared__ float lds_p[32][33];
  __shared__ int lds_c[32][33];
  __shared__ int lds_n;
  __shared__ bool last;
  __shared__ float sums[16];
  const int s = P.first + blockIdx.x, x = threadIdx.x & 31, y = threadIdx.x >> 5, e = blockIdx.y * 32 + x;
  const int a = offset_at(P, s), b = offset_at(P, s + 1);
  const int i0 = a / P.tile, i1 = b > a ? (b - 1) / P.tile : i0 - 1;
  if (threadIdx.x == 0) lds_n = 0;
  __syncthreads();
  int n = 0;
  for (int i = i0 + threadIdx.x; i <= i1; i += 1024) n += W.tokens[(size_t)i + s];
  if (n) atomicAdd(&lds_n, n);
  float p = 0.f;
  int c = 0;
  if (e < P.E) {
#pragma unroll 4
    for (int i = i0 + y; i <= i1; i += 32) {
      p += W.probs[((size_t)i + s) * P.E + e];
      c += W.counts[((size_t)i + s) * P.E + e];
    }
  }
  lds_p[y][x] = p;
  lds_c[y][x] = c;
  __syncthreads();
  n = lds_n;
  if (threadIdx.x < 32) {
    p = 0.f;
    c = 0;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      p += lds_p[i][x];
      c += lds_c[i][x];
    }
    float part = 0.f;
    if (e < P.E) {
      p = n > 0 ? p / (float)n : 0.f;
      probs[(size_t)s * P.E + e] = p;
      counts[(size_t)s * P.E + e] = c;
      if (n > 0) part = (float)c / ((float)P.k * (float)n) * p;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) part += __shfl_xor(part, o, 32);
    if (threadIdx.x == 0) {
      // (what the last workgroup reads goes through the caches that all compute units share)
      __hip_atomic_store(&W.loss[(size_t)s * gridDim.y + blockIdx.y], part, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      if (blockIdx.y == 0) __hip_atomic_store(&tokens[s], n, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      const uint32_t before = __hip_atomic_fetch_add(W.done, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT);
      last = before == (uint32_t)P.S * gridDim.y - 1;
    }
  }
  __syncthreads();
  if (!last) return;
  if (threadIdx.x == 0) lds_n = 0;
  __syncthreads();
  float total[1] = {0.f};
  for (size_t i = threadIdx.x; i < (size_t)P.S * gridDim.y; i += 1024)
    total[0] += __hip_atomic_load(&W.loss[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  int used = 0;
  for (int i = threadIdx.x; i < P.S; i += 1024) used += __hip_atomic_load(&tokens[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) > 0;
  if (used) atomicAdd(&lds_n, used);
  group_sum<1024, 1>(total, sums);
  if (threadIdx.x == 0) {
    tokens[P.S] = lds_n;
    loss[0] = lds_n > 0 ? P.alpha * (float)P.E * total[0] / (float)lds_n : 0.f;
  }
}

template <int KIND, int L, int C>
__global__ __launch_bounds__(256) void balance_grad_kernel(balance_args P, const int32_t* counts, const int32_t* tokens,
                                                           const float* d_loss, void* dz) {
  constexpr int U = C == 1 ? 4 : 1;
  const int e0 = (threadIdx.x % L) * 4, t0 = (P.first + blockIdx.x) * (U * (256 / L));
  offset_window offsets(P);
  float p[U][C][4];
  bool in[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int t = t0 + u * (256 / L) + threadIdx.x / L;
    in[u] = t < P.T && (!P.mask || P.mask[t]);
#pragma unroll
    for (int j = 0; j < C; ++j) {
      const int e = e0 + j * L * 4;
      load4<KIND>(P.z, (size_t)t * P.E + e, in[u] ? P.E - e : 0, p[u][j]);
    }
  }
  const int used = tokens[P.S];
  const float g = (d_loss ? d_loss[0] : 1.f) * P.alpha * (float)P.E;
  float f[C][4];
  float w = 0.f;
  int s = offsets.sequence_of(t0), have = -2;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int t = t0 + u * (256 / L) + threadIdx.x / L;
    softmax_token<L, C>(p[u]);
    if (P.offsets) {
      while (s + 1 < P.S && offset_at(P, s + 1) <= t) ++s;
      in[u] = in[u] && s >= 0 && t < offset_at(P, s + 1);
    }
    if (s != have) {
      have = s;
      const int n = s >= 0 ? tokens[s] : 0;
      const float per = n > 0 ? 1.f / ((float)P.k * (float)n) : 0.f;
      w = n > 0 && used > 0 ? g / ((float)used * (float)n) : 0.f;
#pragma unroll
      for (int j = 0; j < C; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int e = e0 + j * L * 4 + i;
          f[j][i] = e < P.E && s >= 0 ? (float)counts[(size_t)s * P.E + e] * per : 0.f;
        }
    }
    float dot = 0.f;
#pragma unroll
    for (int j = 0; j < C; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) dot = fmaf(f[j][i], p[u][j][i], dot);
    dot = token_sum<L>(dot);
#pragma unroll
    for (int j = 0; j < C; ++j) {
#pragma unroll
      for (int i = 0; i < 4; ++i) p[u][j][i] = in[u] ? w * p[u][j][i] * (f[j][i] - dot) : 0.f;
      const int e = e0 + j * L * 4;
      store4<KIND>(dz, (size_t)t * P.E + e, t < P.T ? P.E - e : 0, p[u][j]);
    }
  }
}

cq_status check_balance(int logit_kind, const int32_t* offsets, int S, int T, int E, int k) {
  if (T < 0 || T > 1 << 30 || E <= 0 || E > kMaxExperts || k <= 0 || k > E || k > 64 || S <= 0 || S > kMostSequences) return CQ_ERR_SHAPE;
  if ((long)T * k > 0x7fffffffL) return CQ_ERR_SHAPE;   // (counts are 32-bit)
  if (!offsets && S != 1) return CQ_ERR_NULL;
  if (!cq_row_kind(logit_kind)) return CQ_ERR_UNSUPPORTED;
  return CQ_OK;
}

// Tokens per workgroup.  One round of loads, about 4096 logits, where that makes no more tiles than the second launch, whose workgroups
// share out the sequences, adds quickly: 512 per sequence (65536 x 128 in one sequence 21.8 us, with 2048 tiles 27.3; 60000 x 100 in
// 64 sequences 36.1, with 1875 tiles 27.9).  Longer batches take as many tokens as make that many tiles.
constexpr int kMostExpertsInRound = 256;

long most_tiles(int S) { return 512 * (S < 4 ? S : 4); }

int round_tokens(int E) {
  int lanes = 1;
  while (lanes * 4 < E) lanes *= 2;
  return 4 * (256 / lanes);
}

bool in_rounds(int T, int E, int S) { return E <= kMostExpertsInRound && ((long)T + round_tokens(E) - 1) / round_tokens(E) <= most_tiles(S); }

int tile_of(int T, int E, int S) {
  if (in_rounds(T, E, S)) return round_tokens(E);
  const int tile = (int)((T + most_tiles(S) - 1) / most_tiles(S));
  return tile < 16 ? 16 : tile;
}

size_t slots_of(int T, int S) { return (size_t)(T < most_tiles(S) ? T : most_tiles(S)) + 1 + S; }   // (never falls as T grows)

// One workgroup and one launch: 64 x 4 6.2 us (two launches 8.7), 256 x 64 6.2 (10.2), 512 x 64 9.1 (10.2), 1024 x 64 15.0 (10.5); 512 x 64
// in four sequences, one after the other, 18.6 (10.5).
bool in_one(int T, int E, int S) { return (long)T * E * S <= 32768 && S <= 2 && E <= 256; }

#define CQ_BALANCE_WIDTHS(LAUNCH, KIND, E)      \
  do {                                          \
    if ((E) <= 4) LAUNCH(KIND, 1, 1);           \
    else if ((E) <= 8) LAUNCH(KIND, 2, 1);      \
    else if ((E) <= 16) LAUNCH(KIND, 4, 1);     \
    else if ((E) <= 32) LAUNCH(KIND, 8, 1);     \
    else if ((E) <= 64) LAUNCH(KIND, 16, 1);    \
    else if ((E) <= 128) LAUNCH(KIND, 32, 1);   \
    else if ((E) <= 256) LAUNCH(KIND, 64, 1);   \
    else LAUNCH(KIND, 64, 4);                   \
  } while (0)
#define CQ_BALANCE_DISPATCH(LAUNCH, kind, E)                               \
  do {                                                                     \
    if ((kind) == CQ_A_F32) CQ_BALANCE_WIDTHS(LAUNCH, CQ_A_F32, E);        \
    else if ((kind) == CQ_A_F16) CQ_BALANCE_WIDTHS(LAUNCH, CQ_A_F16, E);   \
    else CQ_BALANCE_WIDTHS(LAUNCH, CQ_A_BF16, E);                          \
  } while (0)

}  // namespace

extern "C" size_t cq_balance_loss_workspace_bytes(int T, int E, int n_seqs) {
  if (T < 0 || T > 1 << 30 || E <= 0 || E > kMaxExperts || n_seqs <= 0 || n_seqs > kMostSequences || in_one(T, E, n_seqs)) return 0;
  const size_t slots = slots_of(T, n_seqs);
  return 2 * cq_align_up(slots * E * 4, 256) + cq_align_up(slots * 4, 256) + cq_align_up((size_t)n_seqs * ((E + 31) / 32) * 4, 256) + 256;
}

extern "C" cq_status cq_balance_loss(const void* logits, int logit_kind, const int32_t* topk_ids, const int32_t* seq_offsets,
                                     int n_seqs, const uint8_t* token_mask, int T, int E, int top_k, float alpha, float* loss,
                                     int32_t* counts, float* probs, int32_t* tokens, void* workspace, size_t workspace_bytes,
                                     cq_stream stream) {
  const cq_status st = check_balance(logit_kind, seq_offsets, n_seqs, T, E, top_k);
  if (st != CQ_OK) return st;
  if ((T > 0 && (!logits || !topk_ids)) || !loss || !counts || !probs || !tokens) return CQ_ERR_NULL;
  const size_t need = cq_balance_loss_workspace_bytes(T, E, n_seqs);
  if (need > 0 && (!workspace || workspace_bytes < need)) return CQ_ERR_WORKSPACE;
  hipStream_t s = (hipStream_t)stream;
  balance_args P = {logits, topk_ids, seq_offsets, token_mask, T, E, top_k, n_seqs, tile_of(T, E, n_seqs), 0, alpha};
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
  W.done = (uint32_t*)(at + cq_align_up((size_t)n_seqs * ((E + 31) / 32) * 4, 256));
  if (in_one(T, E, n_seqs)) {
    // (in_one has no more than 256 experts)
#define LAUNCH(KIND, L, C)                                                                                                       \
  do {                                                                                                                           \
    if constexpr (C == 1)                                                                                                        \
      hipLaunchKernelGGL((balance_one_kernel<KIND, L, C>), dim3(1), dim3(1024), 0, s, P, counts, probs, tokens, loss);            \
  } while (0)
    CQ_BALANCE_DISPATCH(LAUNCH, logit_kind, E);
#undef LAUNCH
    return cq_check_launch();
  }
  const int tiles = T > 0 ? (T - 1) / P.tile + 1 : 1;
  const bool rounds = in_rounds(T, E, n_seqs);
#define LAUNCH(KIND, L, C)                                                                                             \
  do {                                                                                                                 \
    if (C == 1 && rounds) hipLaunchKernelGGL((balance_tile_kernel<KIND, L>), dim3(tiles), dim3(256), 0, s, P, W);      \
    else hipLaunchKernelGGL((balance_long_tile_kernel<KIND, L, C>), dim3(tiles), dim3(256), 0, s, P, W);               \
  } while (0)
  CQ_BALANCE_DISPATCH(LAUNCH, logit_kind, E);
#undef LAUNCH
  cq_status launched = cq_check_launch();
  constexpr int kMost = (int)(kMostThreads / 1024);
  for (; P.first < n_seqs && launched == CQ_OK; P.first += kMost) {
    const int seqs = n_seqs - P.first < kMost ? n_seqs - P.first : kMost;
    hipLaunchKernelGGL(balance_sequence_kernel, dim3(seqs, (E + 31) / 32), dim3(1024), 0, s, P, W, counts, probs, tokens, loss);
    launched = cq_check_launch();
  }
  return launched;
}

extern "C" cq_status cq_balance_loss_grad(const void* logits, int logit_kind, const int32_t* counts, const int32_t* tokens,
                                          const int32_t* seq_offsets, int n_seqs, const uint8_t* token_mask, int T, int E,
                                          int top_k, float alpha, const float* d_loss, void* d_logits, cq_stream stream) {
  const cq_status st = check_balance(logit_kind, seq_offsets, n_seqs, T, E, top_k);
  if (st != CQ_OK) return st;
  if (T == 0) return CQ_OK;
  if (!logits || !counts || !tokens || !d_logits) return CQ_ERR_NULL;
  balance_args P = {logits, nullptr, seq_offsets, token_mask, T, E, top_k, n_seqs, 0, 0, alpha};
  cq_status launched = CQ_OK;
#define LAUNCH(KIND, L, C)                                                                                                          \
  do {                                                                                                                              \
    constexpr int kMost = (int)(kMostThreads / 256), kTokens = (C == 1 ? 4 : 1) * (256 / L);                                        \
    const int groups = (T - 1) / kTokens + 1;                                                                                       \
    for (; P.first < groups && launched == CQ_OK; P.first += kMost) {                                                               \
      const int now = groups - P.first < kMost ? groups - P.first : kMost;                                                          \
      hipLaunchKernelGGL((balance_grad_kernel<KIND, L, C>), dim3(now), dim3(256), 0, (hipStream_t)stream, P, counts, tokens, d_loss, \
                         d_logits);                                                                                                 \
      launched = cq_check_launch();                                                                                                 \
    }                                                                                                                               \
  } while (0)
  CQ_BALANCE_DISPATCH(LAUNCH, logit_kind, E);
#undef LAUNCH
  return launched;
}
