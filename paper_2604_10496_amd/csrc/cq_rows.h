// Rows of fp32, f16 or bf16 values as the operators around the layer read and write them (gfx950 only): eight consecutive
// values per lane, arithmetic in fp32, one rounding (to nearest, ties to even; no saturation) where a value is stored.
#ifndef CQ_ROWS_H_
#define CQ_ROWS_H_

#include "cq_internal.h"

namespace {

// element kinds are the activation kinds of cq.h: CQ_A_F16, CQ_A_F32, CQ_A_BF16
inline bool cq_row_kind(int kind) { return kind == CQ_A_F16 || kind == CQ_A_F32 || kind == CQ_A_BF16; }

// The threads along a dimension of a launch are counted in 32 bits, and what does not fit is cut off without an error (2^26 + 3 rows of
// 64 threads: 3 rows were worked on): larger batches take several launches.
constexpr long kMostThreads = 1l << 31;

// p moved on by `values` elements (a null pointer stays one)
template <typename P>
inline P* row_at(P* p, int kind, size_t values) {
  return p ? (P*)((uintptr_t)p + values * (kind == CQ_A_F32 ? 4 : 2)) : nullptr;
}

template <int KIND>
__device__ __forceinline__ float elem_load(const void* p, size_t at) {
  if constexpr (KIND == CQ_A_F32) return reinterpret_cast<const float*>(p)[at];
  if constexpr (KIND == CQ_A_F16) return (float)reinterpret_cast<const _Float16*>(p)[at];
  if constexpr (KIND == CQ_A_BF16) return __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(p)[at] << 16);
}

template <int KIND>
__device__ __forceinline__ void elem_store(void* p, size_t at, float v) {
  if constexpr (KIND == CQ_A_F32) reinterpret_cast<float*>(p)[at] = v;
  if constexpr (KIND == CQ_A_F16) reinterpret_cast<_Float16*>(p)[at] = (_Float16)v;
  if constexpr (KIND == CQ_A_BF16) reinterpret_cast<__bf16*>(p)[at] = (__bf16)v;
}

// Eight consecutive values as they lie in memory.  Rows may start on any element: the loads and stores ask for the alignment of
// one, which global memory instructions of any width work with (a row of odd width costs a few more cache lines per
// instruction, not eight instructions).  Values that do not exist read as zero and are not stored.
typedef cq_v4u cq_v4u_any __attribute__((aligned(2)));

template <int KIND>
struct row8 {
  static constexpr int N = KIND == CQ_A_F32 ? 2 : 1;
  cq_v4u w[N];
};

template <int KIND>
__device__ __forceinline__ row8<KIND> row_fetch(const void* p, size_t at, int left) {
  row8<KIND> r;
#pragma unroll
  for (int n = 0; n < row8<KIND>::N; ++n) r.w[n] = cq_v4u{0u, 0u, 0u, 0u};
  if (left >= 8) {
    const cq_v4u_any* q = reinterpret_cast<const cq_v4u_any*>(reinterpret_cast<const char*>(p) + at * (KIND == CQ_A_F32 ? 4 : 2));
#pragma unroll
    for (int n = 0; n < row8<KIND>::N; ++n) r.w[n] = q[n];
  } else if (left > 0) {
#pragma unroll
    for (int i = 0; i < 7; ++i) {
      if (i < left) {
        if constexpr (KIND == CQ_A_F32)
          r.w[i >> 2][i & 3] = reinterpret_cast<const uint32_t*>(p)[at + i];
        else
          r.w[0][i >> 1] |= (uint32_t)reinterpret_cast<const uint16_t*>(p)[at + i] << (16 * (i & 1));
      }
    }
  }
  return r;
}

template <int KIND>
__device__ __forceinline__ void row_values(const row8<KIND>& r, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if constexpr (KIND == CQ_A_F32) {
      v[i] = __uint_as_float(r.w[i >> 2][i & 3]);
    } else {
      const uint32_t w = r.w[0][i >> 1];
      if constexpr (KIND == CQ_A_BF16)
        v[i] = __uint_as_float(i & 1 ? w & 0xffff0000u : w << 16);
      else
        v[i] = (float)__builtin_bit_cast(_Float16, (uint16_t)(i & 1 ? w >> 16 : w & 0xffffu));
    }
  }
}

template <int KIND>
__device__ __forceinline__ void row_store8(void* p, size_t at, int left, const float (&v)[8]) {
  if (left >= 8) {
    row8<KIND> r;
    if constexpr (KIND == CQ_A_F32) {
#pragma unroll
      for (int i = 0; i < 8; ++i) r.w[i >> 2][i & 3] = __float_as_uint(v[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint16_t lo, hi;
        if constexpr (KIND == CQ_A_BF16) {
          lo = __builtin_bit_cast(uint16_t, (__bf16)v[2 * i]);
          hi = __builtin_bit_cast(uint16_t, (__bf16)v[2 * i + 1]);
        } else {
          lo = __builtin_bit_cast(uint16_t, (_Float16)v[2 * i]);
          hi = __builtin_bit_cast(uint16_t, (_Float16)v[2 * i + 1]);
        }
        r.w[0][i] = (uint32_t)lo | ((uint32_t)hi << 16);
      }
    }
    cq_v4u_any* q = reinterpret_cast<cq_v4u_any*>(reinterpret_cast<char*>(p) + at * (KIND == CQ_A_F32 ? 4 : 2));
#pragma unroll
    for (int n = 0; n < row8<KIND>::N; ++n) q[n] = r.w[n];
  } else if (left > 0) {
#pragma unroll
    for (int i = 0; i < 7; ++i)
      if (i < left) elem_store<KIND>(p, at + i, v[i]);
  }
}

// Where a thread's eight values of a row lie: columns c .. c+7, of which the first `skip` belong to its neighbour (the last
// thread of a row that is no whole number of groups takes the row's last eight values, so that no load needs a loop over single
// values); on: the thread has any.
struct row_slot {
  int c, skip;
  bool on;
  __device__ __forceinline__ row_slot(int c0, int H) : c(H >= 8 && c0 > H - 8 ? H - 8 : c0), skip(c0 - c), on(c0 < H) {}
};

// Eight values at `at` + `lane_at` of p (uniform and per lane), zero where `on` is false.
template <int KIND>
__device__ __forceinline__ row8<KIND> fetch8(const void* p, size_t at, uint32_t lane_at, bool on) {
  constexpr uint32_t kSize = KIND == CQ_A_F32 ? 4 : 2;
  row8<KIND> r;
#pragma unroll
  for (int n = 0; n < row8<KIND>::N; ++n) r.w[n] = cq_v4u{0u, 0u, 0u, 0u};
  if (on) {
    const cq_v4u_any* q = reinterpret_cast<const cq_v4u_any*>(reinterpret_cast<const char*>(p) + at * kSize + lane_at * kSize);
#pragma unroll
    for (int n = 0; n < row8<KIND>::N; ++n) r.w[n] = q[n];
  }
  return r;
}

template <int KIND>
__device__ __forceinline__ row8<KIND> slot_fetch(const void* p, size_t row, const row_slot& s, int H, bool wanted) {
  if (H < 8) return row_fetch<KIND>(p, row, s.on && wanted ? H : 0);
  row8<KIND> r;
#pragma unroll
  for (int n = 0; n < row8<KIND>::N; ++n) r.w[n] = cq_v4u{0u, 0u, 0u, 0u};
  if (s.on && wanted) {
    const cq_v4u_any* q = reinterpret_cast<const cq_v4u_any*>(reinterpret_cast<const char*>(p) + (row + s.c) * (KIND == CQ_A_F32 ? 4 : 2));
#pragma unroll
    for (int n = 0; n < row8<KIND>::N; ++n) r.w[n] = q[n];
  }
  return r;
}

// raw values from .. to-1 of eight, the others as zero
template <int KIND>
__device__ __forceinline__ void keep_values(row8<KIND>& r, int from, int to) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const bool keep = i >= from && i < to;
    if constexpr (KIND == CQ_A_F32)
      r.w[i >> 2][i & 3] = keep ? r.w[i >> 2][i & 3] : 0u;
    else
      r.w[0][i >> 1] &= keep ? 0xffffffffu : (i & 1 ? 0x0000ffffu : 0xffff0000u);
  }
}

// Makes the compiler take the raw values as new, so that it converts them again instead of keeping the converted ones, twice
// as many registers, from one use to the next.
template <int KIND>
__device__ __forceinline__ void forget_values(row8<KIND>& r) {
#pragma unroll
  for (int n = 0; n < row8<KIND>::N; ++n) asm volatile("" : "+v"(r.w[n]));
}

// the values, the neighbour's as zero
template <int KIND>
__device__ __forceinline__ void slot_values(const row8<KIND>& r, const row_slot& s, int H, float (&v)[8]) {
  row_values<KIND>(r, v);
  if (H % 8 != 0) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < s.skip ? 0.f : v[i];
  }
}

template <int KIND>
__device__ __forceinline__ void slot_store(void* p, size_t row, const row_slot& s, int H, bool wanted, const float (&v)[8]) {
  if (!s.on || !wanted) return;
  if (s.skip == 0 && H >= 8) {
    row_store8<KIND>(p, row + s.c, 8, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i >= s.skip && s.c + i < H) elem_store<KIND>(p, row + s.c + i, v[i]);
  }
}

// Sum over a wavefront, the same in every lane: four exchanges within rows of 16 lanes, two from row to row.
template <int CTRL, int ROWS>
__device__ __forceinline__ float add_dpp(float v) {
  return v + __uint_as_float(__builtin_amdgcn_update_dpp(0u, __float_as_uint(v), CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ float wave_sum(float v) {
  v = add_dpp<0xb1, 0xf>(v);    // quad_perm 1 0 3 2
  v = add_dpp<0x4e, 0xf>(v);    // quad_perm 2 3 0 1
  v = add_dpp<0x141, 0xf>(v);   // row_half_mirror
  v = add_dpp<0x140, 0xf>(v);   // row_mirror
  v = add_dpp<0x142, 0xa>(v);   // row_bcast:15 into rows 1 and 3
  v = add_dpp<0x143, 0xc>(v);   // row_bcast:31 into rows 2 and 3
  return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), 63));
}

// Sums of N values over groups of NT threads of a workgroup, the same in every thread of a group, added in a fixed order.  `lds`
// holds N * NT / 64 floats per group; two calls in a row use different arrays.  All threads of the workgroup make the call.
template <int NT, int N>
__device__ __forceinline__ void group_sum(float (&v)[N], float* lds) {
#pragma unroll
  for (int n = 0; n < N; ++n) v[n] = wave_sum(v[n]);
  if constexpr (NT > 64) {
    constexpr int W = NT / 64;
    const int wave = threadIdx.x >> 6, group = wave / W * W * N;
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int n = 0; n < N; ++n) lds[group + n * W + wave % W] = v[n];
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < N; ++n) {
      float s = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) s += lds[group + n * W + w];
      v[n] = s;
    }
  }
}

}  // namespace

#endif  // CQ_ROWS_H_
