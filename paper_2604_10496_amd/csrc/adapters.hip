// Low-rank adapters of many requests beside a projection that they share:
//   out_t = base_t + scale_a B_a (A_a x_t),  a = ids[t];   a outside [0, n): out_t = base_t.
//
// Two launches of matrix-core tiles, low = A_a x (fp32, kept in K parts in the workspace) and out = base + scale B_a low.
// Both hold tokens as the columns and rows of A or B as the rows of a 16 x 16 result, so that a lane owns four neighbouring
// rows of one token and stores them together.
//
// Tokens meet their adapters in one of two ways.  Batches of up to kLeaderTokens tokens (decode steps, in any order): a
// workgroup per token looks through the ids; the first of every kTile tokens of one adapter takes those tokens, the others'
// workgroups end.  Longer batches are prompts, whose neighbours share an adapter: tiles of neighbouring tokens, adapter by
// adapter within a tile.  Either way an adapter's weights are read once per tile, and nothing is sorted or kept.
//
// 16-bit rows against weights of the same type are multiplied as they are.  fp32 rows (and low itself) against bf16 weights are cut
// into three bf16 values of 8 bits each, which hold every bit of the fp32 value: three products, each exact in fp32.  The other pairs of
// types run on the fp32 matrix cores.  Either way A_a x and B_a low are fp32 sums of exact products.
#include "cq_rows.h"

namespace {

constexpr int kMaxRank = 256;
constexpr int kLeaderTokens = 1024;
constexpr int kDownTile = 16, kUpTile = 64;   // tokens per workgroup
constexpr int kDownWaves = 8, kUpWaves = 4;
constexpr int kRankBlock = 64;                // rows of A per workgroup

struct adapter_args {
  const void *A, *B, *X, *base;
  const float* scale;
  const int32_t *ranks, *ids;
  void* out;
  float* low;   // [parts][T][Rp]
  int n, R, Rp, K, N, T, parts, kpart;
  size_t ldx, ldb, ldo;
};

__device__ __forceinline__ int rank_of(const adapter_args& P, int a) {
  if (a < 0) return 0;
  if (!P.ranks) return P.R;
  const int r = P.ranks[a];
  return r < 0 ? 0 : (r > P.R ? P.R : r);
}

__device__ __forceinline__ int adapter_of(const adapter_args& P, int t) {
  const int a = P.ids[t];
  return a >= 0 && a < P.n ? a : -1;
}

// The tokens of this workgroup in LDS: rows[i] (-1: none) and their adapters.  False: nothing to do.  Ends with a barrier.
template <int TILE>
__device__ __forceinline__ bool find_rows(const adapter_args& P, int* rows, int* adapters, int* found) {
  const int lane = threadIdx.x & 63;
  if (threadIdx.x < 64) {
    if (P.T > kLeaderTokens) {
      const int t = blockIdx.x * TILE + lane;
      const bool ok = lane < TILE && t < P.T;
      if (lane < TILE) {
        rows[lane] = ok ? t : -1;
        adapters[lane] = ok ? adapter_of(P, t) : -1;
      }
      if (lane == 0) *found = min(TILE, P.T - (int)blockIdx.x * TILE);
    } else {
      const int me = blockIdx.x, mine = adapter_of(P, me);
      int before = 0, n = 0;
      bool lead = true;
      for (int c = 0; c < P.T; c += 64) {
        const int t = c + lane;
        const bool same = t < P.T && adapter_of(P, t) == mine;
        before += __popcll(__ballot(same && t < me));
        if (c + 64 > me) {
          if (c <= me) lead = before % TILE == 0;   // (all tokens in front of `me` have been counted)
          if (!lead) break;
          const unsigned long long m = __ballot(same && t >= me);
          const int at = n + __popcll(m & ((1ull << lane) - 1ull));
          if (same && t >= me && at < TILE) {
            rows[at] = t;
            adapters[at] = mine;
          }
          n += __popcll(m);
          if (n >= TILE) break;
        }
      }
      n = lead ? min(n, TILE) : 0;
      if (lane >= n && lane < TILE) {
        rows[lane] = -1;
        adapters[lane] = -1;
      }
      if (lane == 0) *found = n;
    }
  }
  __syncthreads();
  return *found > 0;
}

// An fp32 value as the sum of three values that bf16 holds (8 bits each, cut off, not rounded: no value overflows).
__device__ __forceinline__ void split3(float x, uint32_t& a, uint32_t& b, uint32_t& c) {
  a = __float_as_uint(x) & 0xffff0000u;
  float rest = x - __uint_as_float(a);
  if (__builtin_isinf(x)) rest = 0.f;
  b = __float_as_uint(rest) & 0xffff0000u;
  c = __float_as_uint(rest - __uint_as_float(b));
}

struct split_frag { cq_v8bf16 part[3]; };

__device__ __forceinline__ split_frag split_pack(const float (&v)[8]) {
  cq_v4u w[3];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t lo[3], hi[3];
    split3(v[2 * i], lo[0], lo[1], lo[2]);
    split3(v[2 * i + 1], hi[0], hi[1], hi[2]);
#pragma unroll
    for (int p = 0; p < 3; ++p) w[p][i] = __builtin_amdgcn_perm(hi[p], lo[p], 0x07060302u);
  }
  split_frag f;
#pragma unroll
  for (int p = 0; p < 3; ++p) f.part[p] = __builtin_bit_cast(cq_v8bf16, w[p]);
  return f;
}

// Eight consecutive 16-bit values as they are; the first `left` exist, the others are zero.
__device__ __forceinline__ cq_v4u raw_load8(const void* p, size_t at, int left) { return row_fetch<CQ_A_BF16>(p, at, left).w[0]; }

// How a pair of types is multiplied
enum { kSame16 = 0, kSplit = 1, kFloat = 2 };
template <int XK, int WK>
constexpr int product_path() {
  return XK == WK && XK != CQ_A_F32 ? kSame16 : (XK == CQ_A_F32 && WK == CQ_A_BF16 ? kSplit : kFloat);
}

// low[part][t][r] = sum over the part's k of A_a[r, k] x_t[k].  One workgroup: 16 tokens, RT tiles of 16 rows of A, one part of
// K, which its eight wavefronts share out in steps of 64 and add up in LDS.
template <int XK, int WK, int RT>
__global__ __launch_bounds__(64 * kDownWaves) void adapter_down_kernel(adapter_args P) {
  constexpr int RW = RT * 16, LD = RW + 4;
  __shared__ float lds[kDownWaves][16][LD];
  __shared__ int rows[kDownTile], adapters[kDownTile], found;
  if (!find_rows<kDownTile>(P, rows, adapters, &found)) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int col = lane & 15, g = lane >> 4;
  const int t = rows[col] >= 0 ? rows[col] : rows[0];
  const int mine = adapters[col];
  const int r0 = blockIdx.z * kRankBlock;
  const int k_end = min(P.K, (int)(blockIdx.y + 1) * P.kpart);
  unsigned todo = (unsigned)__ballot(rows[col] >= 0 && mine >= 0) & 0xffffu;
  while (todo) {
    const int a = adapters[__ffs(todo) - 1];
    const bool here = mine == a && rows[col] >= 0;
    todo &= ~((unsigned)__ballot(here) & 0xffffu);
    const int rank = rank_of(P, a);
    if (rank <= r0) continue;
    cq_v4f acc[RT];
#pragma unroll
    for (int i = 0; i < RT; ++i) acc[i] = cq_v4f{0.f, 0.f, 0.f, 0.f};
    const size_t w_row = ((size_t)a * P.R + r0 + col) * P.K;
    for (int k0 = blockIdx.y * P.kpart + wave * 64; k0 < k_end; k0 += 64 * kDownWaves) {
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int k = k0 + g * 16 + half * 8, left = k_end - k;   // this lane's eight of the 32 values of a product
        if constexpr (product_path<XK, WK>() == kSame16) {
          const cq_v4u x = raw_load8(P.X, (size_t)t * P.ldx + k, left);
#pragma unroll
          for (int i = 0; i < RT; ++i) {
            const bool in = r0 + i * 16 + col < rank;
            const cq_v4u w = raw_load8(P.A, w_row + (size_t)i * 16 * P.K + k, in ? left : 0);
            if constexpr (XK == CQ_A_BF16)
              acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(cq_v8bf16, w), __builtin_bit_cast(cq_v8bf16, x), acc[i], 0, 0, 0);
            else
              acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(cq_v8f16, w), __builtin_bit_cast(cq_v8f16, x), acc[i], 0, 0, 0);
          }
        } else {
          float x[8];
          row_load8<XK>(P.X, (size_t)t * P.ldx + k, left, x);
          if constexpr (product_path<XK, WK>() == kSplit) {
            const split_frag xs = split_pack(x);
#pragma unroll
            for (int i = 0; i < RT; ++i) {
              const bool in = r0 + i * 16 + col < rank;
              const cq_v8bf16 w = __builtin_bit_cast(cq_v8bf16, raw_load8(P.A, w_row + (size_t)i * 16 * P.K + k, in ? left : 0));
#pragma unroll
              for (int p = 0; p < 3; ++p) acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, xs.part[p], acc[i], 0, 0, 0);
            }
          } else {
#pragma unroll
            for (int i = 0; i < RT; ++i) {
              const bool in = r0 + i * 16 + col < rank;
              float w[8];
              row_load8<WK>(P.A, w_row + (size_t)i * 16 * P.K + k, in ? left : 0, w);
#pragma unroll
              for (int q = 0; q < 8; ++q) acc[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(w[q], x[q], acc[i], 0, 0, 0);
            }
          }
        }
      }
    }
#pragma unroll
    for (int i = 0; i < RT; ++i) *reinterpret_cast<cq_v4f*>(&lds[wave][col][i * 16 + g * 4]) = acc[i];
    __syncthreads();
    for (int e = threadIdx.x; e < 16 * RW; e += 64 * kDownWaves) {
      const int tok = e / RW, r = e % RW;
      if (rows[tok] < 0 || adapters[tok] != a || r0 + r >= P.Rp) continue;
      float s = 0.f;
#pragma unroll
      for (int w = 0; w < kDownWaves; ++w) s += lds[w][tok][r];
      P.low[((size_t)blockIdx.y * P.T + rows[tok]) * P.Rp + r0 + r] = s;
    }
    __syncthreads();
  }
}

// out = base + scale B_a low.  One workgroup: up to 64 tokens (16 at a time) and 256 outputs; a wavefront has 64 of them as
// four tiles of 16.  The rows of a tile are chosen so that a lane's outputs of one or (16 bits) two tiles are neighbours.
template <int OK>
__device__ __forceinline__ int out_row(int tile, int i) {
  if (OK == CQ_A_F32) return tile * 16 + i;
  return (tile >> 1) * 32 + (i >> 2) * 8 + (tile & 1) * 4 + (i & 3);
}

template <int WK, int OK>
__global__ __launch_bounds__(64 * kUpWaves) void adapter_up_kernel(adapter_args P) {
  __shared__ int rows[kUpTile], adapters[kUpTile], found;
  if (!find_rows<kUpTile>(P, rows, adapters, &found)) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int col = lane & 15, g = lane >> 4;
  const int n0 = (blockIdx.y * kUpWaves + wave) * 64;
  if (n0 >= P.N) return;
  for (int sub = 0; sub < found; sub += 16) {
    const int t = rows[sub + col], mine = adapters[sub + col];
    unsigned todo = (unsigned)__ballot(t >= 0) & 0xffffu;
    while (todo) {
      const int a = adapters[sub + __ffs(todo) - 1];
      const bool here = t >= 0 && mine == a;
      todo &= ~((unsigned)__ballot(here) & 0xffffu);
      const int rank = rank_of(P, a);
      cq_v4f acc[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[j] = cq_v4f{0.f, 0.f, 0.f, 0.f};
      for (int rb = 0; rb < rank; rb += 32) {
        const int r = rb + g * 8;
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0.f;
        if (here && r < rank) {
          for (int p = 0; p < P.parts; ++p) {
            float u[8];
            row_load8<CQ_A_F32>(P.low, ((size_t)p * P.T + t) * P.Rp + r, 8, u);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += u[i];
          }
#pragma unroll
          for (int i = 0; i < 8; ++i) v[i] = r + i < rank ? v[i] : 0.f;   // (0 times an infinite x is no 0)
        }
        if constexpr (WK == CQ_A_BF16) {
          const split_frag vs = split_pack(v);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int n = n0 + out_row<OK>(j, col);
            const cq_v4u b = raw_load8(P.B, ((size_t)a * P.N + n) * P.R + r, n < P.N ? rank - r : 0);
            const cq_v8bf16 w = __builtin_bit_cast(cq_v8bf16, b);
#pragma unroll
            for (int p = 0; p < 3; ++p) acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, vs.part[p], acc[j], 0, 0, 0);
          }
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int n = n0 + out_row<OK>(j, col);
            float w[8];
            row_load8<WK>(P.B, ((size_t)a * P.N + n) * P.R + r, n < P.N ? rank - r : 0, w);
#pragma unroll
            for (int q = 0; q < 8; ++q) acc[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(w[q], v[q], acc[j], 0, 0, 0);
          }
        }
      }
      if (!here) continue;
      const float scale = rank > 0 ? (P.scale ? P.scale[a] : 1.f) : 0.f;
      const size_t o = (size_t)t * P.ldo, b = (size_t)t * P.ldb;
      if constexpr (OK == CQ_A_F32) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int n = n0 + out_row<OK>(j, g * 4), left = P.N - n;
          if (left >= 4) {
            typedef cq_v4f cq_v4f_any __attribute__((aligned(4)));
            cq_v4f v = {0.f, 0.f, 0.f, 0.f};
            if (P.base) v = *reinterpret_cast<const cq_v4f_any*>(reinterpret_cast<const float*>(P.base) + b + n);
            if (rank > 0) v += scale * acc[j];
            *reinterpret_cast<cq_v4f_any*>(reinterpret_cast<float*>(P.out) + o + n) = v;
          } else {
#pragma unroll
            for (int q = 0; q < 3; ++q) {
              if (q >= left) continue;
              float v = P.base ? elem_load<OK>(P.base, b + n + q) : 0.f;
              if (rank > 0) v = fmaf(scale, acc[j][q], v);
              elem_store<OK>(P.out, o + n + q, v);
            }
          }
        }
      } else {
#pragma unroll
        for (int j = 0; j < 4; j += 2) {
          const int n = n0 + out_row<OK>(j, g * 4), left = P.N - n;
          float v[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) v[i] = 0.f;
          if (P.base) row_load8<OK>(P.base, b + n, left, v);
          if (rank > 0) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = fmaf(scale, acc[j + (i >> 2)][i & 3], v[i]);
          }
          row_store8<OK>(P.out, o + n, left, v);
        }
      }
    }
  }
}

cq_status check_adapters(const cq_adapters* W, int T) {
  if (!W) return CQ_ERR_NULL;
  if (T < 0 || W->n <= 0 || W->rank <= 0 || W->rank > kMaxRank || W->K <= 0 || W->N <= 0) return CQ_ERR_SHAPE;
  if (W->K > 1 << 23 || W->N > 1 << 23) return CQ_ERR_SHAPE;
  if (!cq_row_kind(W->kind)) return CQ_ERR_UNSUPPORTED;
  return CQ_OK;
}

int padded_rank(int R) { return (R + 15) / 16 * 16; }

// Parts of K: enough workgroups to fill the chip, each with one step of 64 values for every wavefront at least.
int parts_of(int T, int K) {
  const int tiles = (T + kDownTile - 1) / kDownTile, most = (K + 64 * kDownWaves - 1) / (64 * kDownWaves);
  const int want = tiles >= 512 ? 1 : 512 / tiles;
  const int parts = want < most ? want : most;
  return parts < 16 ? parts : 16;
}

}  // namespace

extern "C" size_t cq_adapter_workspace_bytes(const cq_adapters* W, int T) {
  if (check_adapters(W, T) != CQ_OK) return 0;
  // the most that any batch of up to T tokens takes: parts(T) T rises between the steps of parts
  size_t rows = (size_t)T * 1;
  for (int p = 2; p <= 16; ++p) {
    const long last = (long)(512 / p) * kDownTile;   // the longest batch with p parts
    const int t = T < last ? T : (int)last;
    if (t > 0) {
      const size_t need = (size_t)t * parts_of(t, W->K);
      rows = need > rows ? need : rows;
    }
  }
  return cq_align_up(rows * padded_rank(W->rank) * 4, 256);
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
  P.n = W->n;
  P.R = W->rank;
  P.Rp = padded_rank(W->rank);
  P.K = W->K;
  P.N = W->N;
  P.T = T;
  P.parts = parts_of(T, W->K);
  P.kpart = ((W->K + P.parts - 1) / P.parts + 63) / 64 * 64;
  P.ldx = (size_t)ldx;
  P.ldb = base ? (size_t)ld_base : 0;
  P.ldo = (size_t)ld_out;
  hipStream_t s = (hipStream_t)stream;
  const bool leaders = T <= kLeaderTokens;
  const dim3 down(leaders ? T : (T + kDownTile - 1) / kDownTile, P.parts, (W->rank + kRankBlock - 1) / kRankBlock);
  const dim3 up(leaders ? T : (T + kUpTile - 1) / kUpTile, (W->N + 64 * kUpWaves - 1) / (64 * kUpWaves));
#define DOWN2(XK, WK, RT) hipLaunchKernelGGL((adapter_down_kernel<XK, WK, RT>), down, dim3(64 * kDownWaves), 0, s, P)
#define DOWN1(XK, WK)                         \
  do {                                        \
    if (W->rank <= 16) DOWN2(XK, WK, 1);      \
    else if (W->rank <= 32) DOWN2(XK, WK, 2); \
    else DOWN2(XK, WK, 4);                    \
  } while (0)
#define DOWN(WK)                                      \
  do {                                                \
    if (x_kind == CQ_A_F32) DOWN1(CQ_A_F32, WK);      \
    else if (x_kind == CQ_A_F16) DOWN1(CQ_A_F16, WK); \
    else DOWN1(CQ_A_BF16, WK);                        \
  } while (0)
#define UP2(WK, OK) hipLaunchKernelGGL((adapter_up_kernel<WK, OK>), up, dim3(64 * kUpWaves), 0, s, P)
#define UP(WK)                                    \
  do {                                            \
    if (out_kind == CQ_A_F32) UP2(WK, CQ_A_F32);  \
    else if (out_kind == CQ_A_F16) UP2(WK, CQ_A_F16); \
    else UP2(WK, CQ_A_BF16);                      \
  } while (0)
  if (W->kind == CQ_A_F32) { DOWN(CQ_A_F32); UP(CQ_A_F32); }
  else if (W->kind == CQ_A_F16) { DOWN(CQ_A_F16); UP(CQ_A_F16); }
  else { DOWN(CQ_A_BF16); UP(CQ_A_BF16); }
  return cq_check_launch();
}
