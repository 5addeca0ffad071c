// Attention of one new token per sequence over a paged cache: for the queries of a key head, over the positions j of a sequence,
//     z_j = softcap(scale q.k_j),  out = sum_j e^(z_j) v_j / (sum_j e^(z_j) + e^sink),  lse = log of the denominator,
// in one pass with the running maximum and sum of the softmax.  Bound by the HBM reads of keys and values.
//
// A wavefront takes 32 positions at a time on 16 x 16 x 32 matrix products with the positions as rows and the queries of a key head
// as columns (16 of them; fewer leave columns idle, which costs nothing: the matrix cores have 20 times what the reads need).
//   S^T = K Q^T     lane (c, g) = (l % 16, l / 16) loads 16 bytes of row c at a time: what the product asks of it
//   O^T = V^T P^T   the product leaves lane (c, g) with query c's scores at positions 4g .. 4g+3 of both halves, which is the operand
//                   that the second product asks of it if its inner index runs over just these eight; lane (c, g) therefore loads
//                   dims 8c .. 8c+7 of those eight rows of V, whole lines, and turns the 8 x 8 block in registers
// so nothing passes through LDS, and every row of the softmax stays in its lane.
// Operands are of the cache's type (f16 for e4m3, which it holds exactly).  P, and queries of another type, are split into parts
// that add up to 16 bits at least, 22 where queries or results are fp32: rounded once to 8 bits, P alone would cost the result
// as much as its own rounding.
// The cache is cut along its length into parts, so that few sequences fill the chip; a second launch joins them in order.
#include "cache.h"

namespace {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr int kTile = 32;         // positions of a wavefront's step
constexpr int kMostSplits = 1024;

struct attention_args {
  cache_args C;
  int G, tiles;          // queries of a key head, groups of 16 of them
  int q_kind, out_kind, shift;   // shift: log2 of the page size, -1 where it is no power of two
  int splits, split_len, window, first_seq;
  float scale, softcap;
  const float* sinks;
  head_rows q, out;
  float *lse, *part, *stat;
};

__device__ __forceinline__ void span_of(const cache_args& C, int window, int s, int& begin, int& end) {
  const long most = (long)C.width * C.page_size;
  const int len = C.lengths[s];
  end = len < 0 ? 0 : len > most ? (int)most : len;
  begin = window > 0 && end > window ? end - window : 0;
}

// results of a row: maximum (base 2) and sum of its exponentials, with the sink
__device__ __forceinline__ void close_row(float m, float l, const float* sinks, int head, float& factor, float& lse) {
  float top = m, sum = l;
  if (sinks) {
    const float z = sinks[head] * kLog2e;
    top = fmaxf(m, z);
    const float base = top == -INFINITY ? 0.f : top;
    sum = l * __builtin_amdgcn_exp2f(m - base) + __builtin_amdgcn_exp2f(z - base);
    factor = sum == 0.f ? 0.f : __builtin_amdgcn_exp2f(m - base) / sum;
  } else {
    factor = sum == 0.f ? 0.f : 1.f / sum;
  }
  lse = sum == 0.f ? -INFINITY : (top + log2f(sum)) * kLn2;
}

__device__ __forceinline__ void store4(void* p, int kind, long at, const float (&v)[4]) {
  if (kind == CQ_A_F32) quad_store<CQ_A_F32>(p, at, 4, v);
  else if (kind == CQ_A_F16) quad_store<CQ_A_F16>(p, at, 4, v);
  else quad_store<CQ_A_BF16>(p, at, 4, v);
}

template <int CK>
struct operand;
template <>
struct operand<CQ_A_BF16> {
  static constexpr int kQuery = 3;
  static __device__ __forceinline__ uint16_t round(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }
  static __device__ __forceinline__ float value(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }
  static __device__ __forceinline__ cq_v4f mfma(cq_v4u a, cq_v4u b, cq_v4f c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(cq_v8bf16, a), __builtin_bit_cast(cq_v8bf16, b), c, 0, 0, 0);
  }
};
template <>
struct operand<CQ_A_F16> {
  static constexpr int kQuery = 2;
  static __device__ __forceinline__ uint16_t round(float v) { return __builtin_bit_cast(uint16_t, (_Float16)v); }
  static __device__ __forceinline__ float value(uint16_t b) { return (float)__builtin_bit_cast(_Float16, b); }
  static __device__ __forceinline__ cq_v4f mfma(cq_v4u a, cq_v4u b, cq_v4f c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(cq_v8f16, a), __builtin_bit_cast(cq_v8f16, b), c, 0, 0, 0);
  }
};
template <>
struct operand<CQ_C_E4M3> : operand<CQ_A_F16> {};

// eight values as PARTS operands that add up to them
template <int CK, int PARTS>
__device__ __forceinline__ void split8(const float (&v)[8], cq_v4u (&w)[PARTS]) {
  float rest[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) rest[i] = v[i];
#pragma unroll
  for (int n = 0; n < PARTS; ++n) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint16_t a = operand<CK>::round(rest[2 * i]), b = operand<CK>::round(rest[2 * i + 1]);
      rest[2 * i] -= operand<CK>::value(a);
      rest[2 * i + 1] -= operand<CK>::value(b);
      w[n][i] = (uint32_t)a | ((uint32_t)b << 16);
    }
  }
}

// two e4m3 codes (half HI of a word) as two f16
template <bool HI>
__device__ __forceinline__ uint32_t two_f16(uint32_t codes) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)codes, 1.f, HI));
}

template <int CK, int DPAD, int WAVES, bool HIGH>
__global__ __launch_bounds__(WAVES * 64) void cache_attention_kernel(attention_args A) {
  constexpr bool k8 = CK == CQ_C_E4M3;
  constexpr int kSize = k8 ? 1 : 2;
  constexpr int kSteps = DPAD / 32;                  // products over a row's dims
  constexpr int kE = DPAD >= 128 ? 8 : DPAD / 16;    // neighbouring dims of a lane in V
  constexpr int kChunks = DPAD / (16 * kE);
  constexpr int kQ = HIGH ? operand<CK>::kQuery : 1;
  constexpr int kP = HIGH ? operand<CK>::kQuery : 2;
  constexpr int kKWords = k8 ? DPAD / 64 : DPAD / 32;            // 16-byte pieces of a row of K per lane
  constexpr int kVWords = kE * kSize / 4;                        // words of a row of V per lane and chunk
  extern __shared__ __align__(16) float lds[];
  const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int unit = blockIdx.x;
  const int split = unit % A.splits;
  unit /= A.splits;
  const int h = unit % A.C.heads;
  unit /= A.C.heads;
  const int tile = unit % A.tiles, s = A.first_seq + unit / A.tiles;
  const int rows = min(16, A.G - tile * 16), first_head = h * A.G + tile * 16;
  int begin, end;
  span_of(A.C, A.window, s, begin, end);
  begin += split * A.split_len;   // (at most splits * split_len < 2^31: checked on the host)
  if (split + 1 < A.splits) end = min(end, begin + A.split_len);
  if (A.splits > 1 && begin >= end) return;
  const int D = A.C.D;

  // the queries: column c of the product's second operand
  cq_v4u Q[kSteps][kQ];
  float back = 1.f;   // what the queries were divided by
  {
    float v[kSteps][8], most = 0.f;
    const long row = (long)s * A.q.token + (long)(first_head + c) * A.q.head;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const int d = k8 ? (i >> 1) * 64 + g * 16 + (i & 1) * 8 : i * 32 + g * 8;
      const bool on = c < rows && d < D;
      if (A.q_kind == CQ_A_F32) row_values<CQ_A_F32>(row_fetch<CQ_A_F32>(A.q.p, row + d, on ? 8 : 0), v[i]);
      else if (A.q_kind == CQ_A_F16) row_values<CQ_A_F16>(row_fetch<CQ_A_F16>(A.q.p, row + d, on ? 8 : 0), v[i]);
      else row_values<CQ_A_BF16>(row_fetch<CQ_A_BF16>(A.q.p, row + d, on ? 8 : 0), v[i]);
#pragma unroll
      for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf(v[i][e]));
    }
    if constexpr (CK != CQ_A_BF16) {
      // f16 has less of a range than the other types: the row's largest value to 2^9 .. 2^10
      most = fmaxf(most, __shfl_xor(most, 16));
      most = fmaxf(most, __shfl_xor(most, 32));
      if (most > 0.f && most < INFINITY) {
        const int e = 10 - __builtin_amdgcn_frexp_expf(most);
        back = ldexpf(1.f, -e);
#pragma unroll
        for (int i = 0; i < kSteps; ++i)
#pragma unroll
          for (int j = 0; j < 8; ++j) v[i][j] = ldexpf(v[i][j], e);
      }
    }
#pragma unroll
    for (int i = 0; i < kSteps; ++i) split8<CK, kQ>(v[i], Q[i]);
  }
  const float factor = A.scale * back * (k8 && A.C.k_scale ? A.C.k_scale[h] : 1.f);

  const int32_t* table = A.C.table + (long)s * A.C.table_stride;
  const char* K = reinterpret_cast<const char*>(A.C.k) + (long)h * A.C.head * kSize;
  const char* V = reinterpret_cast<const char*>(A.C.v) + (long)h * A.C.head * kSize;
  // where the row of position from + lane % 32 lies, in bytes; -1: it has none
  auto row_at = [&](int from) -> long {
    const int p = from + (lane & 31);
    if (p >= end) return -1;
    const int column = A.shift >= 0 ? p >> A.shift : p / A.C.page_size;
    const int page = table[column];
    if (page < 0 || page >= A.C.pages) return -1;
    return (page * A.C.page + (p - column * A.C.page_size) * A.C.slot) * kSize;
  };

  cq_v4f O[kChunks][kE];
#pragma unroll
  for (int n = 0; n < kChunks; ++n)
#pragma unroll
    for (int d = 0; d < kE; ++d) O[n][d] = cq_v4f{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;   // of query c; l: this lane's share

  int from = begin + wave * kTile;
  long at = from < end ? row_at(from) : -1;
  for (; from < end; from += WAVES * kTile) {
    const uint32_t there = (uint32_t)__ballot(at >= 0);
    // K: rows c and 16 + c
    cq_v4u k[2][kKWords];
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      const long row = __shfl(at, n * 16 + c);
#pragma unroll
      for (int i = 0; i < kKWords; ++i) {
        const int d = k8 ? i * 64 + g * 16 : i * 32 + g * 8;
        k[n][i] = cq_v4u{0u, 0u, 0u, 0u};
        if (row >= 0 && d < D) k[n][i] = *reinterpret_cast<const cq_v4u*>(K + row + d * kSize);
      }
    }
    // V: dims kE c .. of rows 4g .. 4g+3 and 16 + 4g ..
    uint32_t v[kChunks][8][kVWords];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const long row = __shfl(at, (j >> 2) * 16 + g * 4 + (j & 3));
#pragma unroll
      for (int n = 0; n < kChunks; ++n) {
        const int d = n * 128 + c * kE;
#pragma unroll
        for (int w = 0; w < kVWords; ++w) v[n][j][w] = 0u;
        if (row >= 0 && d < D) {
          const char* p = V + row + d * kSize;
          if constexpr (kVWords == 4) {
            const cq_v4u x = *reinterpret_cast<const cq_v4u*>(p);
#pragma unroll
            for (int w = 0; w < 4; ++w) v[n][j][w] = x[w];
          } else if constexpr (kVWords == 2) {
            const cq_v2u x = *reinterpret_cast<const cq_v2u*>(p);
            v[n][j][0] = x[0];
            v[n][j][1] = x[1];
          } else {
            v[n][j][0] = *reinterpret_cast<const uint32_t*>(p);
          }
        }
      }
    }
    if (from + WAVES * kTile < end) at = row_at(from + WAVES * kTile);
    // scores of query c at positions 4g + r and 16 + 4g + r
    float z[8];
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      cq_v4f acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        cq_v4u a;
        if constexpr (k8) {
          const cq_v4u w = k[n][i >> 1];
          const uint32_t x = w[(i & 1) * 2], y = w[(i & 1) * 2 + 1];
          a = cq_v4u{two_f16<false>(x), two_f16<true>(x), two_f16<false>(y), two_f16<true>(y)};
        } else {
          a = k[n][i];
        }
#pragma unroll
        for (int q = kQ - 1; q >= 0; --q) acc = operand<CK>::mfma(a, Q[i][q], acc);
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) z[n * 4 + r] = acc[r] * factor;
    }
    if (A.softcap > 0.f) {
      const float inv = 1.f / A.softcap;
#pragma unroll
      for (int j = 0; j < 8; ++j) z[j] = A.softcap * tanhf(z[j] * inv);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      z[j] *= kLog2e;
      if (there != 0xffffffffu) z[j] = there >> ((j >> 2) * 16 + g * 4 + (j & 3)) & 1u ? z[j] : -INFINITY;
    }
    float top = m;
#pragma unroll
    for (int j = 0; j < 8; ++j) top = fmaxf(top, z[j]);
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    const float base = top == -INFINITY ? 0.f : top;
    if (__ballot(top > m)) {
      const float shrink = __builtin_amdgcn_exp2f(m - base);
      l *= shrink;
#pragma unroll
      for (int n = 0; n < kChunks; ++n)
#pragma unroll
        for (int d = 0; d < kE; ++d) O[n][d] *= shrink;
      m = top;
    }
    float p[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      p[j] = __builtin_amdgcn_exp2f(z[j] - base);
      l += p[j];
    }
    cq_v4u P[kP];
    split8<CK, kP>(p, P);
#pragma unroll
    for (int n = 0; n < kChunks; ++n) {
#pragma unroll
      for (int d = 0; d < kE; d += 2) {
        uint32_t two[8];   // dims d, d+1 of the eight rows
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if constexpr (k8)
            two[j] = d & 2 ? two_f16<true>(v[n][j][d >> 2]) : two_f16<false>(v[n][j][d >> 2]);
          else
            two[j] = v[n][j][d >> 1];
        }
        cq_v4u lo, hi;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          lo[w] = __builtin_amdgcn_perm(two[2 * w + 1], two[2 * w], 0x05040100u);
          hi[w] = __builtin_amdgcn_perm(two[2 * w + 1], two[2 * w], 0x07060302u);
        }
#pragma unroll
        for (int q = kP - 1; q >= 0; --q) {
          O[n][d] = operand<CK>::mfma(lo, P[q], O[n][d]);
          O[n][d + 1] = operand<CK>::mfma(hi, P[q], O[n][d + 1]);
        }
      }
    }
  }
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);

  // the wavefronts' shares, [WAVES][rows][DPAD + 4], and their maxima and sums behind them
  constexpr int kPitch = DPAD + 4;
  float* stats = lds + WAVES * rows * kPitch;   // [rows][WAVES][2]
  if (c < rows) {
    float* o = lds + (wave * rows + c) * kPitch;
#pragma unroll
    for (int n = 0; n < kChunks; ++n)
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int d = 0; d < kE; d += 4)
          *reinterpret_cast<cq_v4f*>(o + n * 128 + (g * 4 + r) * kE + d) = cq_v4f{O[n][d][r], O[n][d + 1][r], O[n][d + 2][r], O[n][d + 3][r]};
    if (g == 0) {
      stats[(c * WAVES + wave) * 2] = m;
      stats[(c * WAVES + wave) * 2 + 1] = l;
    }
  }
  __syncthreads();
  const int quads = D >> 2;
  for (int i = threadIdx.x; i < rows * quads; i += WAVES * 64) {
    const int row = i / quads, d = (i - row * quads) * 4;
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) top = fmaxf(top, stats[(row * WAVES + w) * 2]);
    const float base = top == -INFINITY ? 0.f : top;
    float sum = 0.f;
    cq_v4f o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      const float f = __builtin_amdgcn_exp2f(stats[(row * WAVES + w) * 2] - base);
      sum = fmaf(stats[(row * WAVES + w) * 2 + 1], f, sum);
      o += *reinterpret_cast<const cq_v4f*>(lds + (w * rows + row) * kPitch + d) * f;
    }
    const int head = first_head + row;
    const size_t line = (size_t)s * A.G * A.C.heads + head;
    if (A.splits > 1) {
      *reinterpret_cast<cq_v4f*>(A.part + (line * A.splits + split) * D + d) = o;
      if (d == 0) {
        A.stat[(line * A.splits + split) * 2] = top;
        A.stat[(line * A.splits + split) * 2 + 1] = sum;
      }
    } else {
      float f, lse;
      close_row(top, sum, A.sinks, head, f, lse);
      if (k8 && A.C.v_scale) f *= A.C.v_scale[h];
      const float r[4] = {o[0] * f, o[1] * f, o[2] * f, o[3] * f};
      store4(const_cast<void*>(A.out.p), A.out_kind, (long)s * A.out.token + (long)head * A.out.head + d, r);
      if (d == 0 && A.lse) A.lse[line] = lse;
    }
  }
}

// joins the parts of a row in order: thread (quad of dims, every n-th part)
__global__ __launch_bounds__(256) void attention_join_kernel(attention_args A) {
  __shared__ float weight[kMostSplits];
  __shared__ float red[8];
  __shared__ cq_v4f sums[256];
  const int heads = A.G * A.C.heads, s = A.first_seq + blockIdx.x / heads, head = blockIdx.x % heads, tid = threadIdx.x;
  const size_t line = (size_t)s * heads + head;
  int begin, end;
  span_of(A.C, A.window, s, begin, end);
  const int parts = min(A.splits, (end - begin + A.split_len - 1) / A.split_len);
  const float* stat = A.stat + line * A.splits * 2;
  float top = -INFINITY;
  for (int i = tid; i < parts; i += 256) top = fmaxf(top, stat[2 * i]);
#pragma unroll
  for (int d = 1; d < 64; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
  if ((tid & 63) == 0) red[tid >> 6] = top;
  __syncthreads();
  top = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
  const float base = top == -INFINITY ? 0.f : top;
  float sum = 0.f;
  for (int i = tid; i < parts; i += 256) {
    const float f = __builtin_amdgcn_exp2f(stat[2 * i] - base);
    weight[i] = f;
    sum = fmaf(stat[2 * i + 1], f, sum);
  }
  sum = wave_sum(sum);
  if ((tid & 63) == 0) red[4 + (tid >> 6)] = sum;
  __syncthreads();
  sum = red[4] + red[5] + red[6] + red[7];
  const int D = A.C.D, quads = D >> 2, groups = 256 / quads, group = tid / quads, d = (tid - group * quads) * 4;
  cq_v4f o = {0.f, 0.f, 0.f, 0.f};
  if (group < groups) {
    const float* part = A.part + line * A.splits * D + d;
#pragma unroll 4
    for (int i = group; i < parts; i += groups) o += *reinterpret_cast<const cq_v4f*>(part + (size_t)i * D) * weight[i];
  }
  sums[tid] = o;
  __syncthreads();
  if (group > 0) return;
  for (int n = 1; n < groups; ++n) o += sums[n * quads + tid];
  float f, lse;
  close_row(top, sum, A.sinks, head, f, lse);
  if (A.C.v_scale) f *= A.C.v_scale[head / A.G];
  const float r[4] = {o[0] * f, o[1] * f, o[2] * f, o[3] * f};
  store4(const_cast<void*>(A.out.p), A.out_kind, (long)s * A.out.token + (long)head * A.out.head + d, r);
  if (tid == 0 && A.lse) A.lse[line] = lse;
}

struct plan {
  int waves, splits, split_len;
};

// How many parts the sequences are cut into: about as many workgroups as the chip holds at once.
inline plan plan_of(const cq_cache* C, int n_seqs, int Hq, int max_length, int window) {
  plan p;
  const int G = Hq / C->heads;
  const long units = (long)n_seqs * C->heads * ((G + 15) / 16);
  const long span = window > 0 && window < max_length ? window : max_length;
  p.waves = 4;
  const long quantum = p.waves * kTile;
  long splits = units > 0 ? (1024 + units - 1) / units : 1;
  if (splits > (span + quantum - 1) / quantum) splits = (span + quantum - 1) / quantum;
  if (splits > kMostSplits) splits = kMostSplits;
  if (splits < 1) splits = 1;
  p.split_len = (int)(((span + splits - 1) / splits + quantum - 1) / quantum * quantum);
  if (p.split_len < quantum) p.split_len = (int)quantum;
  p.splits = (int)((span + p.split_len - 1) / p.split_len);
  if (p.splits < 1) p.splits = 1;
  return p;
}

inline cq_status check_attention(const cq_cache* C, int n_seqs, int Hq, int max_length) {
  const cq_status st = check_cache(C);
  if (st != CQ_OK) return st;
  if (n_seqs < 0 || max_length < 0 || max_length > 1 << 30 || Hq <= 0 || Hq > kMaxHeads || Hq % C->heads != 0) return CQ_ERR_SHAPE;
  return CQ_OK;
}

}  // namespace

extern "C" size_t cq_cache_attention_workspace_bytes(const cq_cache* C, int n_seqs, int Hq, int max_length, int window) {
  if (check_attention(C, n_seqs, Hq, max_length) != CQ_OK) return 0;
  const plan p = plan_of(C, n_seqs, Hq, max_length, window);
  if (p.splits == 1) return 0;
  return (size_t)n_seqs * Hq * p.splits * (C->D + 2) * 4;
}

extern "C" cq_status cq_cache_attention(const cq_cache* C, const cq_sequences* S, const cq_attention_spec* P, const cq_heads* q,
                                        const cq_heads* out, float* lse, void* workspace, size_t workspace_bytes, cq_stream stream) {
  cq_status st = check_cache(C);
  if (st != CQ_OK || (st = check_sequences(S, C)) != CQ_OK) return st;
  if (!P || !q) return CQ_ERR_NULL;
  if ((st = check_heads(q, S->n)) != CQ_OK || (st = check_heads_out(q, out, S->n, C->D)) != CQ_OK) return st;
  if ((st = check_attention(C, S->n, q->n, P->max_length)) != CQ_OK) return st;
  if (!isfinite(P->scale) || !(P->softcap >= 0.f) || !isfinite(P->softcap) || P->window < 0) return CQ_ERR_SHAPE;
  if (S->n == 0) return CQ_OK;
  const plan p = plan_of(C, S->n, q->n, P->max_length, P->window);
  const size_t need = cq_cache_attention_workspace_bytes(C, S->n, q->n, P->max_length, P->window);
  if (need && (!workspace || workspace_bytes < need)) return CQ_ERR_WORKSPACE;
  attention_args a;
  a.C = make_cache_args(C, S);
  a.G = q->n / C->heads;
  a.tiles = (a.G + 15) / 16;
  a.q_kind = q->kind;
  a.out_kind = out->kind;
  a.shift = -1;
  for (int i = 0; i < 31; ++i)
    if (C->page_size == 1 << i) a.shift = i;
  a.splits = p.splits;
  a.split_len = p.split_len;
  a.window = P->window;
  a.scale = P->scale;
  a.softcap = P->softcap;
  a.sinks = P->sinks;
  a.q = make_head_rows(q);
  a.out = make_head_rows(out);
  a.lse = lse;
  a.part = (float*)workspace;
  a.stat = a.part + (size_t)S->n * q->n * p.splits * C->D;
  const bool high = q->kind == CQ_A_F32 || out->kind == CQ_A_F32 || (C->kind == CQ_A_BF16 && q->kind == CQ_A_F16);
  const int dpad = C->D <= 64 ? 64 : C->D <= 128 ? 128 : 256;
  const int rows = a.G < 16 ? a.G : 16;
  const int lds = (p.waves * rows * (dpad + 4) + rows * p.waves * 2) * 4;
  // sequences of a launch: its threads are counted in 32 bits
  const long per_seq = (long)p.splits * C->heads * a.tiles;
  const long most = (1l << 22) / (per_seq > q->n ? per_seq : q->n) > 0 ? (1l << 22) / (per_seq > q->n ? per_seq : q->n) : 1;
  for (long from = 0; from < S->n; from += most) {
    const long n = S->n - from < most ? S->n - from : most;
    a.first_seq = (int)from;
    const dim3 grid((unsigned)(n * per_seq));
#define LAUNCH(CK, DPAD, HIGH)                                                                                              \
  do {                                                                                                                      \
    static std::atomic<bool> done{false};                                                                                   \
    if (lds > 64 * 1024 - 1024 &&                                                                                           \
        cq_configure_lds(cache_attention_kernel<CK, DPAD, 4, HIGH>, 4 * (16 * (DPAD + 4) + 32) * 4, done, false) != CQ_OK)  \
      return CQ_ERR_HIP;                                                                                                    \
    hipLaunchKernelGGL((cache_attention_kernel<CK, DPAD, 4, HIGH>), grid, dim3(256), lds, (hipStream_t)stream, a);          \
  } while (0)
#define WIDTHS(CK, HIGH)                      \
  do {                                        \
    if (dpad == 64) LAUNCH(CK, 64, HIGH);     \
    else if (dpad == 128) LAUNCH(CK, 128, HIGH); \
    else LAUNCH(CK, 256, HIGH);               \
  } while (0)
#define KINDS(CK)                \
  do {                           \
    if (high) WIDTHS(CK, true);  \
    else WIDTHS(CK, false);      \
  } while (0)
    if (C->kind == CQ_A_F16) KINDS(CQ_A_F16);
    else if (C->kind == CQ_A_BF16) KINDS(CQ_A_BF16);
    else KINDS(CQ_C_E4M3);
#undef KINDS
#undef WIDTHS
#undef LAUNCH
    if (p.splits > 1) hipLaunchKernelGGL(attention_join_kernel, dim3((unsigned)(n * q->n)), dim3(256), 0, (hipStream_t)stream, a);
  }
  return cq_check_launch();
}
