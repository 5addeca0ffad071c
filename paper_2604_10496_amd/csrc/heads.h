// Heads of queries, keys and values as the operators behind the Q/K/V projection see them (gfx950 only): rows of D values, one per
// token and head, with a norm and a rotation by the token's position:
//     r = 1 / sqrt(mean x^2 + eps),  n = x r w,   pairs (a, b) of the first `rot` values:  a' = n_a c - n_b s,  b' = n_b c + n_a s,
//     (c, s) = m (cos, sin)(position freq_i)
// A row belongs to 8, 16, 32 or 64 neighbouring lanes, each of which holds eight values in two quads that are chosen so that both
// values of a pair lie in the same lane: four values and their partners half a rotation further, or eight neighbours.  What is not
// rotated follows in lanes of eight neighbours.  The angle is taken modulo one revolution in 64 bits: in 32 bits a position of 10^5
// would leave it 2^-8 radians off.
#ifndef CQ_HEADS_H_
#define CQ_HEADS_H_

#include <math.h>

#include "cq_rows.h"

namespace {

constexpr int kMaxHeadWidth = 256;
constexpr int kMaxHeads = 1 << 14;
constexpr float kMostE4M3 = 448.f;

// ---- host side --------------------------------------------------------------------------------

// how the lanes of a row share its values
struct head_layout {
  int D, rot, inter;
  int turned;   // lanes that hold rotated values
  int used;     // lanes that hold any
  int lanes;    // 8, 16, 32 or 64
  int mode;
};

// whole: the used lanes hold eight values each.  shifted: the last of the rotated ones and the last of all are moved back to the last values
// there are, of which their neighbours own the first (few rotated values are followed by others), so that no load or sum needs a loop
// over single values: 4096 tokens of 40 heads of 80, 20 rotated, 29 us with such loops, 21 without.  general: rows of fewer than eight.  Each
// is a kernel of its own: the code for single values is ten times as long, and what single tokens wait for is instructions (1 token of
// 40 heads in 4.2 us; 6.6 with it).
constexpr int kGeneral = 0, kShifted = 1, kWhole = 2;

inline head_layout make_head_layout(int D, int rot, int inter) {
  head_layout L;
  L.D = D;
  L.rot = rot;
  L.inter = inter || rot == 0;
  L.turned = inter ? (rot + 7) / 8 : (rot / 2 + 3) / 4;
  L.used = L.turned + (D - rot + 7) / 8;
  L.mode = L.used * 8 == D ? kWhole : D >= 8 ? kShifted : kGeneral;
  L.lanes = L.used <= 8 ? 8 : L.used <= 16 ? 16 : L.used <= 32 ? 32 : 64;
  return L;
}

inline cq_status check_head_spec(const cq_head_spec* P) {
  if (!P) return CQ_ERR_NULL;
  if (P->D <= 0 || P->D > kMaxHeadWidth || P->rot < 0 || P->rot > P->D || P->rot % 2 != 0) return CQ_ERR_SHAPE;
  if (!isfinite(P->rot_scale)) return CQ_ERR_SHAPE;
  if ((P->w_q || P->w_k) && (!(P->eps > 0.f) || !isfinite(P->eps))) return CQ_ERR_SHAPE;
  if (P->rot > 0 && !P->freq) return CQ_ERR_NULL;
  if ((P->w_q || P->w_k) && !cq_row_kind(P->weight_kind)) return CQ_ERR_UNSUPPORTED;
  return CQ_OK;
}

// rows that a call reads (NULL: there are none)
inline cq_status check_heads(const cq_heads* h, int T) {
  if (!h) return CQ_OK;
  if (h->n <= 0 || h->n > kMaxHeads) return CQ_ERR_SHAPE;
  if (!cq_row_kind(h->kind)) return CQ_ERR_UNSUPPORTED;
  if (T > 0 && !h->p) return CQ_ERR_NULL;
  return CQ_OK;
}

// rows that a call writes: as many heads, none on another's place
inline cq_status check_heads_out(const cq_heads* in, const cq_heads* out, int T, int D) {
  if (!in) return CQ_OK;
  if (!out) return CQ_ERR_NULL;
  const cq_status st = check_heads(out, T);
  if (st != CQ_OK) return st;
  if (out->n != in->n || (out->n > 1 && out->head_stride < D) || (T > 1 && out->token_stride < D)) return CQ_ERR_SHAPE;
  // (one of the steps over all rows of the other)
  if (out->n > 1 && T > 1 && out->head_stride < (T - 1) * (double)out->token_stride + D &&
      out->token_stride < (out->n - 1) * (double)out->head_stride + D)
    return CQ_ERR_SHAPE;
  return CQ_OK;
}

struct head_rows {
  const void* p;
  long token, head;   // values between tokens and between heads
  int n;
};

inline head_rows make_head_rows(const cq_heads* h) {
  head_rows r = {nullptr, 0, 0, 0};
  if (h) r = {h->p, h->token_stride, h->head_stride, h->n};
  return r;
}

// the groups of rows that a wavefront takes in one instruction: heads of one kind, so that what depends on the kind is the same in every lane
inline int head_groups(int n, const head_layout& L) { return (n + 64 / L.lanes - 1) / (64 / L.lanes); }

// Groups per wavefront and wavefronts per token: one, or several where there are few tokens (at most `most` wavefronts come of that).
inline void share_groups(int groups, long T, long most, int& per_part, int& parts) {
  parts = 1;
  while (parts * 2 <= groups && T * parts * 2 <= most) parts *= 2;
  per_part = (groups + parts - 1) / parts;
  parts = (groups + per_part - 1) / per_part;
}

inline head_rows rows_from(head_rows r, int kind, long token) {
  r.p = row_at(r.p, kind, (size_t)(token * r.token));
  return r;
}

// ---- device side ------------------------------------------------------------------------------

// four consecutive values as they lie in memory, on any element
typedef __attribute__((__vector_size__(2 * sizeof(uint32_t)))) uint32_t cq_v2u;
typedef cq_v2u cq_v2u_any __attribute__((aligned(2)));

template <int KIND>
struct quad {
  static constexpr int N = 2;
  cq_v2u w;
};
template <>
struct quad<CQ_A_F32> {
  static constexpr int N = 4;
  cq_v4u w;
};

template <int KIND, int MODE>
__device__ __forceinline__ quad<KIND> quad_fetch(const void* p, long at, int n) {
  quad<KIND> q;
  q.w = decltype(q.w){};
  const char* b = reinterpret_cast<const char*>(p) + at * (KIND == CQ_A_F32 ? 4 : 2);
  if (n == 4) {
    if constexpr (KIND == CQ_A_F32)
      q.w = *reinterpret_cast<const cq_v4u_any*>(b);
    else
      q.w = *reinterpret_cast<const cq_v2u_any*>(b);
  } else if constexpr (MODE == kGeneral) {
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      if (i < n) {
        if constexpr (KIND == CQ_A_F32)
          q.w[i] = reinterpret_cast<const uint32_t*>(b)[i];
        else
          q.w[i >> 1] |= (uint32_t)reinterpret_cast<const uint16_t*>(b)[i] << (16 * (i & 1));
      }
    }
  }
  return q;
}

template <int KIND>
__device__ __forceinline__ float quad_value(const quad<KIND>& q, int i) {
  if constexpr (KIND == CQ_A_F32) return __uint_as_float(q.w[i]);
  const uint32_t w = q.w[KIND == CQ_A_F32 ? 0 : i >> 1];
  if constexpr (KIND == CQ_A_BF16) return __uint_as_float(i & 1 ? w & 0xffff0000u : w << 16);
  return (float)__builtin_bit_cast(_Float16, (uint16_t)(i & 1 ? w >> 16 : w & 0xffffu));
}

template <int KIND>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  uint16_t a, b;
  if constexpr (KIND == CQ_A_BF16) {
    a = __builtin_bit_cast(uint16_t, (__bf16)lo);
    b = __builtin_bit_cast(uint16_t, (__bf16)hi);
  } else {
    a = __builtin_bit_cast(uint16_t, (_Float16)lo);
    b = __builtin_bit_cast(uint16_t, (_Float16)hi);
  }
  return (uint32_t)a | ((uint32_t)b << 16);
}

// The four e4m3 codes of four values, rounded to nearest, ties to even; beyond +-448 saturated (NaN stays NaN).
__device__ __forceinline__ uint32_t pack_e4m3(const float (&v)[4]) {
  float c[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) c[i] = v[i] != v[i] ? v[i] : fminf(fmaxf(v[i], -kMostE4M3), kMostE4M3);
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(c[0], c[1], 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c[2], c[3], w, true);
}

template <int KIND>
__device__ __forceinline__ void quad_store(void* p, long at, int n, const float (&v)[4]) {
  char* b = reinterpret_cast<char*>(p) + at * (KIND == CQ_A_F32 ? 4 : KIND == CQ_C_E4M3 ? 1 : 2);
  if constexpr (KIND == CQ_C_E4M3) {
    typedef uint32_t word_any __attribute__((aligned(1)));
    const uint32_t w = pack_e4m3(v);
    if (n == 4) {
      *reinterpret_cast<word_any*>(b) = w;
    } else {
#pragma unroll
      for (int i = 0; i < 3; ++i)
        if (i < n) reinterpret_cast<uint8_t*>(b)[i] = (uint8_t)(w >> (8 * i));
    }
  } else if (n == 4) {
    if constexpr (KIND == CQ_A_F32)
      *reinterpret_cast<cq_v4u_any*>(b) =
          cq_v4u{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
    else
      *reinterpret_cast<cq_v2u_any*>(b) = cq_v2u{pack2<KIND>(v[0], v[1]), pack2<KIND>(v[2], v[3])};
  } else {
#pragma unroll
    for (int i = 0; i < 3; ++i)
      if (i < n) elem_store<KIND>(b, i, v[i]);
  }
}

// Which values a lane holds: the sa-th to na-th of four from column a, the sb-th to nb-th from column b; turned: they are rotated, as pairs
// first .. first+3.
struct head_slot {
  int a, b, na, nb, sa, sb, first;
  bool turned;
};

template <int MODE>
__device__ __forceinline__ head_slot make_slot(const head_layout& L, int j) {
  head_slot s;
  const int half = L.rot >> 1;
  s.turned = j < L.turned;
  const bool apart = s.turned && !L.inter;
  int from = apart ? 4 * j : s.turned ? 8 * j : L.rot + 8 * (j - L.turned);
  const int left = (apart ? half : s.turned ? L.rot : L.D) - from;   // of which there are
  const int more = apart ? left : left - 4;
  s.na = left < 0 ? 0 : left < 4 ? left : 4;
  s.nb = more < 0 ? 0 : more < 4 ? more : 4;
  s.sa = s.sb = 0;
  if constexpr (MODE == kShifted) {
    const int width = apart ? 4 : 8, back = left > 0 && left < width && from >= width - left ? width - left : 0;
    from -= back;
    if (back) s.na = s.nb = 4;
    s.sa = back < 4 ? back : 4;
    s.sb = apart ? back : back - s.sa;
  }
  s.first = apart ? from : from >> 1;
  s.a = from;
  s.b = apart ? half + from : from + 4;
  return s;
}

template <int KIND>
struct head_raw {
  quad<KIND> a, b;
};

// SIDE: a lane's quads lie side by side (all but pairs apart).
template <int KIND, int MODE, bool SIDE>
__device__ __forceinline__ head_raw<KIND> head_fetch(const void* p, long at, const head_slot& s, bool on) {
  head_raw<KIND> r;
  if constexpr (MODE != kGeneral) {
    const bool there = on && s.na;   // (all eight values are)
    if constexpr (SIDE && KIND != CQ_A_F32) {
      cq_v4u w = {0u, 0u, 0u, 0u};
      if (there) w = *reinterpret_cast<const cq_v4u_any*>(reinterpret_cast<const char*>(p) + (at + s.a) * 2);
      r.a.w = cq_v2u{w[0], w[1]};
      r.b.w = cq_v2u{w[2], w[3]};
      return r;
    }
    r.a = quad_fetch<KIND, MODE>(p, at + s.a, there ? 4 : 0);
    r.b = quad_fetch<KIND, MODE>(p, at + s.b, there ? 4 : 0);
  } else {
    r.a = quad_fetch<KIND, MODE>(p, at + s.a, on ? s.na : 0);
    r.b = quad_fetch<KIND, MODE>(p, at + s.b, on ? s.nb : 0);
  }
  return r;
}

template <int KIND>
__device__ __forceinline__ void head_values(const head_raw<KIND>& r, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[i] = quad_value<KIND>(r.a, i);
    v[4 + i] = quad_value<KIND>(r.b, i);
  }
}

// the values for the row's sums: a neighbour's as zeros
template <int MODE>
__device__ __forceinline__ void own_values(const head_slot& s, float (&v)[8]) {
  if constexpr (MODE == kShifted) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (i & 3) < (i < 4 ? s.sa : s.sb) || (i & 3) >= (i < 4 ? s.na : s.nb) ? 0.f : v[i];
  }
}

// the values from the from-th to the end-th
template <int KIND>
__device__ __forceinline__ void quad_store_some(void* p, long at, int from, int end, const float (&v)[4]) {
  if (from == 0 && end == 4) {
    quad_store<KIND>(p, at, 4, v);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float one[4] = {v[i], 0.f, 0.f, 0.f};
      if (i >= from && i < end) quad_store<KIND>(p, at + i, 1, one);
    }
  }
}

template <int KIND, int MODE, bool SIDE>
__device__ __forceinline__ void head_store(void* p, long at, const head_slot& s, const float (&v)[8]) {
  const float a[4] = {v[0], v[1], v[2], v[3]}, b[4] = {v[4], v[5], v[6], v[7]};
  if constexpr (MODE == kGeneral) {
    quad_store<KIND>(p, at + s.a, s.na, a);
    quad_store<KIND>(p, at + s.b, s.nb, b);
  } else if (s.na) {
    if constexpr (SIDE && MODE == kWhole && (KIND == CQ_A_F16 || KIND == CQ_A_BF16)) {
      row_store8<KIND>(p, (size_t)(at + s.a), 8, v);
    } else if constexpr (MODE == kWhole) {
      quad_store<KIND>(p, at + s.a, 4, a);
      quad_store<KIND>(p, at + s.b, 4, b);
    } else {
      quad_store_some<KIND>(p, at + s.a, s.sa, s.na, a);
      quad_store_some<KIND>(p, at + s.b, s.sb, s.nb, b);
    }
  }
}

// a lane's share of a norm's weights (ones without a norm)
template <int MODE, bool SIDE>
__device__ __forceinline__ void head_weights(const void* w, int kind, const head_slot& s, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = 1.f;
  if (!w) return;
  if (kind == CQ_A_F32)
    head_values<CQ_A_F32>(head_fetch<CQ_A_F32, MODE, SIDE>(w, 0, s, true), v);
  else if (kind == CQ_A_F16)
    head_values<CQ_A_F16>(head_fetch<CQ_A_F16, MODE, SIDE>(w, 0, s, true), v);
  else
    head_values<CQ_A_BF16>(head_fetch<CQ_A_BF16, MODE, SIDE>(w, 0, s, true), v);
}

// cosines and sines of a lane's four pairs
struct head_turn {
  float c[4], s[4];
};

// position freq / (2 pi) modulo 1, in -1/2 .. 1/2.  The product and the quotient keep what their roundings leave over: at position 2^31
// these are 2^-22 radians each, more than fp32 sines and cosines are off by.
__device__ __forceinline__ float revolutions(int position, double freq) {
  constexpr double kHi = 0.15915494309189533577, kLo = -9.839338337591243e-18;   // 1 / (2 pi), and what 64 bits leave of it
  const double t = (double)position * freq, dt = fma((double)position, freq, -t);
  const double rev = t * kHi, rest = fma(t, kHi, -rev) + fma(t, kLo, dt * kHi);
  return (float)((rev - rint(rev)) + rest);
}

// Cosine and sine of x revolutions, |x| <= 1/2 and a little: by quarters, of which the rest is at most pi/4, with the series of both to
// where the next term is under 2^-29 (sine) and 2^-33 (cosine).  (The library's function for this keeps its results in scratch memory.)
__device__ __forceinline__ void turn_by(float x, float& c, float& s) {
  const float quarter = rintf(4.f * x);
  const float t = 6.28318530717958647693f * fmaf(-0.25f, quarter, x), t2 = t * t;
  const float sn = fmaf(t * t2, fmaf(t2, fmaf(t2, fmaf(t2, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), t);
  const float cs = fmaf(t2, fmaf(t2, fmaf(t2, fmaf(t2, fmaf(t2, -1.f / 3628800.f, 1.f / 40320.f), -1.f / 720.f), 1.f / 24.f), -0.5f), 1.f);
  const int n = (int)quarter;
  const float a = n & 1 ? sn : cs, b = n & 1 ? cs : sn;
  c = (n + 1) & 2 ? -a : a;
  s = n & 2 ? -b : b;
}

__device__ __forceinline__ head_turn turn_of(const head_layout& L, const head_slot& s, const double* freq, float rot_scale, int position) {
  head_turn t;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    t.c[i] = 1.f;
    t.s[i] = 0.f;
    if (s.turned && s.first + i < (L.rot >> 1)) {
      turn_by(revolutions(position, freq[s.first + i]), t.c[i], t.s[i]);
      t.c[i] *= rot_scale;
      t.s[i] *= rot_scale;
    }
  }
  return t;
}

// a' = a c - b s, b' = b c + a s; back: by the angle's negative
template <bool INTER, bool BACK>
__device__ __forceinline__ void turn_values(const head_slot& s, const head_turn& t, float (&v)[8]) {
  if (!s.turned) return;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float sn = BACK ? -t.s[i] : t.s[i];
    if constexpr (INTER) {
      const float a = v[2 * i], b = v[2 * i + 1];
      v[2 * i] = fmaf(a, t.c[i], -(b * sn));
      v[2 * i + 1] = fmaf(b, t.c[i], a * sn);
    } else {
      const float a = v[i], b = v[4 + i];
      v[i] = fmaf(a, t.c[i], -(b * sn));
      v[4 + i] = fmaf(b, t.c[i], a * sn);
    }
  }
}

// sum over the LANES neighbouring lanes of a row, the same in each, in a fixed order
template <int LANES>
__device__ __forceinline__ float row_sum(float v) {
  v = add_dpp<0xb1, 0xf>(v);     // quad_perm 1 0 3 2
  v = add_dpp<0x4e, 0xf>(v);     // quad_perm 2 3 0 1
  v = add_dpp<0x141, 0xf>(v);    // row_half_mirror
  if constexpr (LANES >= 16) v = add_dpp<0x140, 0xf>(v);   // row_mirror
  if constexpr (LANES >= 32) v += __shfl_xor(v, 16);
  if constexpr (LANES >= 64) v += __shfl_xor(v, 32);
  return v;
}

template <int LANES>
__device__ __forceinline__ void head_normed(float (&v)[8], const float (&w)[8], float inv_D, float eps) {
  float ss = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) ss = fmaf(v[i], v[i], ss);
  const float r = 1.f / sqrtf(row_sum<LANES>(ss) * inv_D + eps);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = v[i] * r * w[i];
}

}  // namespace

// Runs LAUNCH(..., LANES, MODE, INTER) for a layout (64 lanes are never all whole: that would take 512 values).  Pairs of neighbours (or
// none) and pairs apart are two kernels: in one the compiler reads a row's values by index, from scratch memory.
#define CQ_HEAD_WIDTHS(LAUNCH, L, INTER, ...)                                                        \
  do {                                                                                               \
    if ((L).mode == kWhole && (L).lanes == 8) LAUNCH(__VA_ARGS__, 8, kWhole, INTER);                 \
    else if ((L).mode == kWhole && (L).lanes == 16) LAUNCH(__VA_ARGS__, 16, kWhole, INTER);          \
    else if ((L).mode == kWhole) LAUNCH(__VA_ARGS__, 32, kWhole, INTER);                             \
    else if ((L).mode == kShifted && (L).lanes == 8) LAUNCH(__VA_ARGS__, 8, kShifted, INTER);        \
    else if ((L).mode == kShifted && (L).lanes == 16) LAUNCH(__VA_ARGS__, 16, kShifted, INTER);      \
    else if ((L).mode == kShifted && (L).lanes == 32) LAUNCH(__VA_ARGS__, 32, kShifted, INTER);      \
    else if ((L).mode == kShifted) LAUNCH(__VA_ARGS__, 64, kShifted, INTER);                         \
    else LAUNCH(__VA_ARGS__, 8, kGeneral, INTER);                                                    \
  } while (0)
#define CQ_HEAD_LANES(LAUNCH, L, ...)                              \
  do {                                                             \
    if ((L).inter) CQ_HEAD_WIDTHS(LAUNCH, L, true, __VA_ARGS__);   \
    else CQ_HEAD_WIDTHS(LAUNCH, L, false, __VA_ARGS__);            \
  } while (0)

#endif  // CQ_HEADS_H_
