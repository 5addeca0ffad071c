// Rows of fp32, f16 or bf16 values as the operators around the layer read and write them (gfx950 only): eight consecutive
// values per lane, arithmetic in fp32, one rounding (to nearest, ties to even; no saturation) where a value is stored.
#ifndef CQ_ROWS_H_
#define CQ_ROWS_H_

#include "cq_internal.h"

namespace {

// element kinds are the activation kinds of cq.h: CQ_A_F16, CQ_A_F32, CQ_A_BF16
inline bool cq_row_kind(int kind) { return kind == CQ_A_F16 || kind == CQ_A_F32 || kind == CQ_A_BF16; }
inline int cq_row_bytes(int kind) { return kind == CQ_A_F32 ? 4 : 2; }

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

// Values at .. at+7 of p.  VEC: p + at is 16-byte aligned and all eight exist or none does (left > 0 decides); otherwise the
// first `left` of them exist.  Values that do not exist read as zero and are not stored.
template <int KIND, bool VEC>
__device__ __forceinline__ void row_load8(const void* p, size_t at, int left, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = 0.f;
  if constexpr (VEC) {
    if (left <= 0) return;
    if constexpr (KIND == CQ_A_F32) {
      const cq_v4f* q = reinterpret_cast<const cq_v4f*>(reinterpret_cast<const float*>(p) + at);
      const cq_v4f a = q[0], b = q[1];
#pragma unroll
      for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
    } else {
      const cq_v4u w = *reinterpret_cast<const cq_v4u*>(reinterpret_cast<const uint16_t*>(p) + at);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (KIND == CQ_A_BF16) {
          v[2 * i] = __uint_as_float(w[i] << 16);
          v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        } else {
          v[2 * i] = (float)__builtin_bit_cast(_Float16, (uint16_t)(w[i] & 0xffffu));
          v[2 * i + 1] = (float)__builtin_bit_cast(_Float16, (uint16_t)(w[i] >> 16));
        }
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < left) v[i] = elem_load<KIND>(p, at + i);
  }
}

template <int KIND, bool VEC>
__device__ __forceinline__ void row_store8(void* p, size_t at, int left, const float (&v)[8]) {
  if constexpr (VEC) {
    if (left <= 0) return;
    if constexpr (KIND == CQ_A_F32) {
      cq_v4f* q = reinterpret_cast<cq_v4f*>(reinterpret_cast<float*>(p) + at);
      q[0] = cq_v4f{v[0], v[1], v[2], v[3]};
      q[1] = cq_v4f{v[4], v[5], v[6], v[7]};
    } else {
      cq_v4u w;
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
        w[i] = (uint32_t)lo | ((uint32_t)hi << 16);
      }
      *reinterpret_cast<cq_v4u*>(reinterpret_cast<uint16_t*>(p) + at) = w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < left) elem_store<KIND>(p, at + i, v[i]);
  }
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// Sums of N values over a workgroup of NT threads, the same in every thread, added in a fixed order.  `lds` holds
// N * NT / 64 floats; two calls in a row use different arrays, or a barrier stands between them.
template <int NT, int N>
__device__ __forceinline__ void group_sum(float (&v)[N], float* lds) {
#pragma unroll
  for (int n = 0; n < N; ++n) v[n] = wave_sum(v[n]);
  if constexpr (NT > 64) {
    constexpr int W = NT / 64;
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int n = 0; n < N; ++n) lds[n * W + wave] = v[n];
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < N; ++n) {
      float s = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) s += lds[n * W + w];
      v[n] = s;
    }
  }
}

}  // namespace

#endif  // CQ_ROWS_H_
