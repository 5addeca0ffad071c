// Low-rank adapters of many requests beside a projection that they share:
//   out_t = base_t + scale_a B_a (A_a x_t),  a = ids[t];   a outside [0, n): out_t = base_t.
//
// Two launches of matrix-core tiles, low = A_a x (fp32, kept in K parts in the workspace) and out = base + scale B_a low; one launch
// for few tokens of low rank.  They hold tokens as the columns and rows of A or B as the rows of a 16 x 16 result, so that a lane
// owns four neighbouring rows of one token and stores them together.
//
// Tokens meet their adapters in one of two ways.  Batches of up to kLeaderTokens tokens (decode steps, in any order): a
// workgroup per token looks through the ids; the first of every 16 tokens of one adapter takes those tokens, the others'
// workgroups end.  Longer batches are prompts, whose neighbours share an adapter: tiles of neighbouring tokens, adapter by
// adapter within a tile.  Either way an adapter's weights are read once per tile, and nothing is sorted or kept.
//
// 16-bit rows against weights of the same type are multiplied as they are.  fp32 rows (and low itself) against bf16 weights are cut
// into three bf16 values of 8 bits each, which hold every bit of the fp32 value: three products, each exact in fp32.  The other pairs of
// types run on the fp32 matrix cores.  Either way A_a x and B_a low are fp32 sums of exact products.
//
// 4096 tokens of 9 prompts, K = N = 4096, rank 32, bf16: 18.4 + 18.2 us for 104 MB (2.8 TB/s); 64 requests with adapters of ranks 16 to
// 64, K = 2048, N = 2816: 7.6 + 10.2 us for 22 MB; one token of fp32 rows at rank 16: 11.5 us in one launch.
#include <type_traits>

#include "cq_rows.h"

namespace {

constexpr int kMaxRank = 256;
// Both ways at K = N = 4096, rank 32 (us; 8 adapters in order / in turn, 32 adapters in order / in turn): 257 tokens singly 20 / 22, 22 / 20,
// as prompts 21 / 72, 31 / 143; 400 tokens 27 / 31, 31 / 25 and 21 / 73, 30 / 142; 512 tokens 36 / 37, 37 / 31 and 14 / 74, 16 / 143.  Decode
// batches stay below, the usual pieces of prompts above.
constexpr int kLeaderTokens = 384;
// Workgroups of a launch for single tokens, most of which end at once: they are started at about 250 per us (1024 tokens of 16 adapters
// taken singly: 96.6 us with 8192 and 16384 workgroups, 55.4 with at most 4096).
constexpr int kMostGroups = 4096;
constexpr int kTile = 16;         // tokens of a matrix-core tile
constexpr int kPromptTiles = 2;   // tiles that a wavefront of the second launch takes, of prompts
constexpr int kDownWaves = 4, kPromptDownWaves = 8, kFewWaves = 8, kUpWaves = 4;
constexpr int kRankBlock = 64;                // rows of A per workgroup

struct adapter_args {
  const void *A, *B, *X, *base;
  const float* scale;
  const int32_t *ranks, *ids;
  void* out;
  float* low;   // [parts][tiles of 16 tokens][Rp], see low_at
  int n, R, Rp, K, N, T, tiles, parts, kpart;
  int up_blocks;   // blocks of 256 outputs that a workgroup of the second launch takes, of single tokens
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

// The tile of a group of workgroups.  Single tokens: which ones have work depends on the ids (every 16th where neighbours share an
// adapter, the first ones where they take turns); workgroups go to the eight XCDs in turn, and either pattern is spread over them.
// (1024 tokens in order, taken singly: 97 us where every 16th workgroup is on the same XCD, 55 spread.)
__device__ __forceinline__ int tile_of_group(const adapter_args& P, int group) {
  return P.T > kLeaderTokens ? group : group ^ (group >> 4 & 7);
}

// The tokens of a tile: lane i < TILE gets the i-th one's row (-1: none) and adapter.  Every wavefront finds them by itself, the
// same ones.  False: another tile has them.
template <int TILE>
__device__ __forceinline__ bool find_rows(const adapter_args& P, int tile, int& row, int& id) {
  const int lane = threadIdx.x & 63;
  if (P.T > kLeaderTokens) {
    const int t = tile * TILE + lane;
    const bool in = lane < TILE && t < P.T;
    row = in ? t : -1;
    id = in ? adapter_of(P, t) : -1;
    return true;
  }
  if (tile >= P.T) return false;
  const int me = tile, mine = adapter_of(P, me);
  int before = 0, n = 0;
  row = -1;
  for (int c = 0; c < P.T; c += 64) {
    const int t = c + lane;
    const bool same = t < P.T && adapter_of(P, t) == mine;
    before += __popcll(__ballot(same && t < me));
    if (c + 64 <= me) continue;
    if (c <= me && before % TILE != 0) return false;   // (all tokens in front of `me` have been counted)
    const unsigned long long m = __ballot(same && t >= me);
    const int at = n + __popcll(m & ((1ull << lane) - 1ull));
    // lane `at` gets t; those without a place send theirs to the last lane, which no tile uses
    const int got = __builtin_amdgcn_ds_permute((same && t >= me && at < TILE ? at : 63) * 4, t);
    if (lane >= n && lane < min(n + __popcll(m), TILE)) row = got;
    n += __popcll(m);
    if (n >= TILE) break;
  }
  id = row >= 0 ? mine : -1;
  return true;
}

// An fp32 value as the sum of three values that bf16 holds (8 bits each, cut off, not rounded: no value overflows; what is below
// bf16's smallest, 2^-133, is lost).  An infinity is its own first part.
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

// The second and third parts of a value are often 0, and 0 times an infinite weight makes a NaN of what should be an infinite product.
// Sums that come out as NaN are therefore taken again (FINITE below) with those parts against finite_weights: infinities and NaN as the
// largest finite value of their sign.  The first part, which has the value's sign and is 0 only with it (from 2^-133 on), meets the weight
// itself, and what a finite weight adds to that has the same sign.  4096 tokens of fp32 rows at rank 64: 59.8 us without either, 60.1 with
// the second look at NaN, 64.2 with finite weights at all times.
__device__ __forceinline__ cq_v8bf16 finite_weights(const cq_v4u& w) {
  typedef __attribute__((__vector_size__(16))) uint16_t v8u;
  typedef __attribute__((__vector_size__(16))) int16_t v8i;
  const v8u bits = __builtin_elementwise_min(__builtin_bit_cast(v8u, w), (v8u)(v8u{} + (uint16_t)0xff7f));   // negative ones
  const v8i both = __builtin_elementwise_min(__builtin_bit_cast(v8i, bits), (v8i)(v8i{} + (int16_t)0x7f7f));
  return __builtin_bit_cast(cq_v8bf16, both);
}

template <int N>
__device__ __forceinline__ bool any_nan(const cq_v4f (&acc)[N]) {   // in the wavefront; true at times where infinities of both signs meet
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) s += (acc[i][0] + acc[i][1]) + (acc[i][2] + acc[i][3]);
  return __ballot(s != s) != 0;
}

// How a pair of types is multiplied
enum { kSame16 = 0, kSplit = 1, kFloat = 2 };
template <int XK, int WK>
constexpr int product_path() {
  return XK == WK && XK != CQ_A_F32 ? kSame16 : (XK == CQ_A_F32 && WK == CQ_A_BF16 ? kSplit : kFloat);
}

// Eight values of a row of K from k on, zero where k >= k_end (the last part's k_end is K, the others' a multiple of 64).  The last
// eight of a row that is no whole number of eights overlap their neighbours, whose values they hold as zero.
template <int KIND>
__device__ __forceinline__ row8<KIND> fetch_k(const void* p, size_t row, int k, int k_end, int K) {
  if (K < 8) return row_fetch<KIND>(p, row, k == 0 ? K : 0);
  const int at = min(k, K - 8);
  row8<KIND> r = fetch8<KIND>(p, row + at, 0, k < k_end);
  if (K % 8 != 0) keep_values(r, k - at, 8);
  return r;
}

// Units of a round that a kernel has registers for (256 per lane: one workgroup of eight wavefronts per compute unit, or two of four).
template <int XK, int WK, int RT>
constexpr int most_units() {
  return product_path<XK, WK>() == kSame16 ? (RT == 1 ? 4 : 2) : product_path<XK, WK>() == kSplit && RT == 1 ? 2 : 1;
}

// Four neighbouring lanes hand each other their registers: lane q of the four gets, as its value c, value q of lane c.
__device__ __forceinline__ void quad_transpose(cq_v4u (&r)[4]) {
  const bool odd = threadIdx.x & 1, high = threadIdx.x & 2;
#pragma unroll
  for (int d = 0; d < 4; ++d) {
#pragma unroll
    for (int n = 0; n < 4; n += 2) {
      const uint32_t a = r[n][d], b = r[n + 1][d];
      const uint32_t from_b = __builtin_amdgcn_update_dpp(0u, b, 0xb1, 0xf, 0xf, false);   // quad_perm 1 0 3 2
      const uint32_t from_a = __builtin_amdgcn_update_dpp(0u, a, 0xb1, 0xf, 0xf, false);
      r[n][d] = odd ? from_b : a;
      r[n + 1][d] = odd ? b : from_a;
    }
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      const uint32_t a = r[n][d], b = r[n + 2][d];
      const uint32_t from_b = __builtin_amdgcn_update_dpp(0u, b, 0x4e, 0xf, 0xf, false);   // quad_perm 2 3 0 1
      const uint32_t from_a = __builtin_amdgcn_update_dpp(0u, a, 0x4e, 0xf, 0xf, false);
      r[n][d] = high ? from_b : a;
      r[n + 2][d] = high ? b : from_a;
    }
  }
}

// 128 values of K of 16 rows, as operands of four products: a lane of row l % 16 has values (l / 16) * 32 + c * 8 .. +7 as its c-th.
// The four lanes of rows 4 i .. 4 i + 3 read 64 contiguous bytes of one row after the other and exchange them: lanes that
// each read their own row take the cache three times as long (out of L2 15 instead of 42 bytes per clock and compute unit).
// OWN: each lane reads its own row all the same, and exchanges nothing (fp32 rows of few tokens, whose exchange costs more than their
// loads: one token at rank 16, K = N = 4096 in one launch 10.9 instead of 13.5 us).
template <int KIND, bool OWN = false>
struct k_unit {
  static constexpr int kSize = KIND == CQ_A_F32 ? 4 : 2, kSets = KIND == CQ_A_F32 ? 2 : 1;
  cq_v4u raw[kSets][4];
  // row[n]: first value of row 4 i + n, k: first value of the unit
  __device__ __forceinline__ void fetch(const void* p, const size_t (&row)[4], int k) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const size_t from = OWN ? row[0] : row[n];
      const char* q = reinterpret_cast<const char*>(p) + (from + k + (lane >> 4) * 32) * kSize + (OWN ? n : lane & 3) * 16;
#pragma unroll
      for (int h = 0; h < kSets; ++h) raw[h][n] = reinterpret_cast<const cq_v4u_any*>(q + h * 64)[0];
    }
  }
  __device__ __forceinline__ void exchange() {
    if constexpr (!OWN) {
#pragma unroll
      for (int h = 0; h < kSets; ++h) quad_transpose(raw[h]);
    }
  }
  __device__ __forceinline__ row8<KIND> operand(int c) const {
    row8<KIND> r;
    if constexpr (KIND == CQ_A_F32) {
      r.w[0] = raw[c >> 1][2 * (c & 1)];
      r.w[1] = raw[c >> 1][2 * (c & 1) + 1];
    } else {
      r.w[0] = raw[0][c];
    }
    return r;
  }
};

// acc += 16 rows of A times 16 tokens over 32 values of K
template <int XK, int WK, bool FINITE>
__device__ __forceinline__ void down_product(const row8<WK>& w, const row8<XK>& x, cq_v4f& acc) {
  if constexpr (product_path<XK, WK>() == kSame16) {
    if constexpr (XK == CQ_A_BF16)
      acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(cq_v8bf16, w.w[0]), __builtin_bit_cast(cq_v8bf16, x.w[0]), acc, 0, 0, 0);
    else
      acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(cq_v8f16, w.w[0]), __builtin_bit_cast(cq_v8f16, x.w[0]), acc, 0, 0, 0);
  } else {
    float v[8];
    row_values<XK>(x, v);
    if constexpr (product_path<XK, WK>() == kSplit) {
      const split_frag xs = split_pack(v);
      const cq_v8bf16 rest = FINITE ? finite_weights(w.w[0]) : __builtin_bit_cast(cq_v8bf16, w.w[0]);
      acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(cq_v8bf16, w.w[0]), xs.part[0], acc, 0, 0, 0);
      acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(rest, xs.part[1], acc, 0, 0, 0);
      acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(rest, xs.part[2], acc, 0, 0, 0);
    } else {
      float u[8];
      row_values<WK>(w, u);
#pragma unroll
      for (int q = 0; q < 8; ++q) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(u[q], v[q], acc, 0, 0, 0);
    }
  }
}

// A wavefront's share of the sums over k .. k_end-1 for one adapter's rows r0 .. and 16 tokens: rounds of UNITS units per wavefront,
// then of half as many, down to one; the values that make no whole unit come last, with bounds.  `x` holds the first round's units of
// the tokens where `fetched`.
struct down_place {
  int a, rank, r0;
  size_t own_row, x_row[4];   // X of the lane's own token, and of the four tokens that its quad reads
};

template <int XK, int WK, int RT, int UNITS, int WAVES, bool FINITE, bool OWN>
__device__ __forceinline__ void down_rounds(const adapter_args& P, const down_place& at, int k, int k_end, bool fetched,
                                            k_unit<XK, OWN> (&x)[UNITS], cq_v4f (&acc)[RT]) {
  constexpr int kRound = 128 * WAVES * UNITS;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, g = lane >> 4;
  // (rows beyond the adapter's rank repeat its last one: their sums are not used)
  auto w_row = [&](int r) { return ((size_t)at.a * P.R + min(at.r0 + r, at.rank - 1)) * P.K; };
  auto fetch_rows = [&](int i, int kk, k_unit<WK>& w) {
    const size_t row[4] = {w_row(i * 16 + (col & 12)), w_row(i * 16 + (col & 12) + 1), w_row(i * 16 + (col & 12) + 2), w_row(i * 16 + (col & 12) + 3)};
    w.fetch(P.A, row, kk);
  };
#pragma unroll 1
  for (; k_end - k >= kRound; k += kRound) {
    const int kk = k + wave * 128 * UNITS;
    if (!fetched) {
#pragma unroll
      for (int u = 0; u < UNITS; ++u) x[u].fetch(P.X, at.x_row, kk + u * 128);
    }
    // (two tiles of rows at a time, all their loads before the first product: the scheduler would hold the second's back)
    constexpr int kPair = RT < 2 ? 1 : 2;
#pragma unroll
    for (int i = 0; i < RT; i += kPair) {
      k_unit<WK> w[kPair][UNITS];
#pragma unroll
      for (int j = 0; j < kPair; ++j)
#pragma unroll
        for (int u = 0; u < UNITS; ++u) fetch_rows(i + j, kk + u * 128, w[j][u]);
      __builtin_amdgcn_sched_barrier(0);
      if (i == 0 && !fetched) {
#pragma unroll
        for (int u = 0; u < UNITS; ++u) x[u].exchange();
      }
#pragma unroll
      for (int j = 0; j < kPair; ++j)
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
          w[j][u].exchange();
#pragma unroll
          for (int c = 0; c < 4; ++c) down_product<XK, WK, FINITE>(w[j][u].operand(c), x[u].operand(c), acc[i + j]);
        }
    }
    fetched = false;
  }
  if constexpr (UNITS > 1) {
    k_unit<XK, OWN> fewer[UNITS / 2];
    down_rounds<XK, WK, RT, UNITS / 2, WAVES, FINITE, OWN>(P, at, k, k_end, false, fewer, acc);
  } else {
    const int kk = k + wave * 128;
    if (kk + 128 <= k_end) {
      k_unit<XK, OWN> last;   // (x may be wanted again)
      last.fetch(P.X, at.x_row, kk);
      last.exchange();
#pragma unroll
      for (int i = 0; i < RT; ++i) {
        k_unit<WK> w;
        fetch_rows(i, kk, w);
        w.exchange();
#pragma unroll
        for (int c = 0; c < 4; ++c) down_product<XK, WK, FINITE>(w.operand(c), last.operand(c), acc[i]);
      }
    } else {
#pragma unroll 1
      for (int from = kk; from < k_end; from += 32) {
        const row8<XK> rest = fetch_k<XK>(P.X, at.own_row, from + g * 8, k_end, P.K);
#pragma unroll
        for (int i = 0; i < RT; ++i) down_product<XK, WK, FINITE>(fetch_k<WK>(P.A, w_row(i * 16 + col), from + g * 8, k_end, P.K), rest, acc[i]);
      }
    }
  }
}

// acc again, where it holds a NaN that finite_weights may spare (x then holds the first round of these tokens, as before)
template <int XK, int WK, int RT, int UNITS, int WAVES, bool OWN>
__device__ __forceinline__ void down_again(const adapter_args& P, const down_place& at, int k, int k_end, k_unit<XK, OWN> (&x)[UNITS],
                                           cq_v4f (&acc)[RT]) {
  if constexpr (product_path<XK, WK>() == kSplit) {
    if (__builtin_expect(!any_nan(acc), 1)) return;
#pragma unroll
    for (int i = 0; i < RT; ++i) acc[i] = cq_v4f{0.f, 0.f, 0.f, 0.f};
    down_rounds<XK, WK, RT, UNITS, WAVES, true, OWN>(P, at, k, k_end, false, x, acc);
  }
}

// the rows of X that the quad of a lane reads, and the lane's own (lanes without a token: the first lane's, which has one; readlane
// does not depend on which lanes are active)
__device__ __forceinline__ void place_tokens(const adapter_args& P, int row, down_place& at) {
  const int col = threadIdx.x & 15, some = __builtin_amdgcn_readlane(row, 0);
  auto token = [&](int of) {
    const int t = __shfl(row, of);
    return (size_t)(t < 0 ? some : t) * P.ldx;
  };
  at.own_row = token(col);
#pragma unroll
  for (int n = 0; n < 4; ++n) at.x_row[n] = token((col & 12) + n);
}

// Where low holds value r of token t: blocks of 16 tokens x 8 values, so that what the four lanes of neighbouring tokens read of
// it is contiguous.
__device__ __forceinline__ size_t low_at(const adapter_args& P, int part, int t, int r) {
  return (((size_t)part * P.tiles + (t >> 4)) * (P.Rp / 8) + (r >> 3)) * 128 + (t & 15) * 8 + (r & 7);
}

// low[part][t][r] = sum over the part's k of A_a[r, k] x_t[k].  One workgroup: 16 tokens, RT tiles of 16 rows of A, one part of K,
// which its wavefronts share out and add up in LDS.  Bound by latency and by the traffic out of L2 (every tile reads its adapter's
// A): the loads of a round are all asked for before the first product, those of prompts' tokens before the ids are known.
template <int XK, int WK, int RT, int UNITS, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void adapter_down_kernel(adapter_args P) {
  constexpr int RW = RT * 16, LD = RW + 4, kRound = 128 * WAVES * UNITS;
  __shared__ float lds[WAVES][16][LD];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int col = lane & 15, g = lane >> 4;
  const int k_first = blockIdx.y * P.kpart, k_end = min(P.K, k_first + P.kpart);
  const int rounds = (k_end - k_first) / kRound;
  // Workgroups go to the eight XCDs in turn.  Prompts: an XCD takes neighbouring tiles, which share an adapter in its L2.
  int tile = tile_of_group(P, blockIdx.x);
  if (P.T > kLeaderTokens) {
    const int each = gridDim.x / 8;   // (the grid is a multiple of 8 then)
    tile = blockIdx.x % 8 * each + blockIdx.x / 8;
    if (tile * kTile >= P.T) return;
  }
  down_place at;
  k_unit<XK> x[UNITS];
  bool fetched = P.T > kLeaderTokens && rounds > 0;   // x holds the first round of this workgroup's tokens
  if (fetched) {
#pragma unroll
    for (int n = 0; n < 4; ++n) at.x_row[n] = (size_t)min(tile * kTile + (col & 12) + n, P.T - 1) * P.ldx;
#pragma unroll
    for (int u = 0; u < UNITS; ++u) x[u].fetch(P.X, at.x_row, k_first + (wave * UNITS + u) * 128);
  }
  int row, id;
  if (!find_rows<kTile>(P, tile, row, id)) return;
  place_tokens(P, row, at);
  if (fetched) {
#pragma unroll
    for (int u = 0; u < UNITS; ++u) x[u].exchange();
  }
  at.r0 = blockIdx.z * kRankBlock;
  unsigned todo = (unsigned)__ballot(id >= 0) & 0xffffu;
  while (todo) {
    at.a = __builtin_amdgcn_readlane(id, __ffs(todo) - 1);
    const unsigned match = (unsigned)__ballot(id == at.a) & 0xffffu;
    todo &= ~match;
    at.rank = rank_of(P, at.a);
    if (at.rank > at.r0) {
      cq_v4f acc[RT];
#pragma unroll
      for (int i = 0; i < RT; ++i) acc[i] = cq_v4f{0.f, 0.f, 0.f, 0.f};
      down_rounds<XK, WK, RT, UNITS, WAVES, false, false>(P, at, k_first, k_end, fetched, x, acc);
      down_again<XK, WK, RT, UNITS, WAVES, false>(P, at, k_first, k_end, x, acc);
      fetched = rounds == 1;   // x serves the next adapter's tokens as well
#pragma unroll
      for (int i = 0; i < RT; ++i) *reinterpret_cast<cq_v4f*>(&lds[wave][col][i * 16 + g * 4]) = acc[i];
      __syncthreads();
      for (int e = threadIdx.x; e < 16 * RW; e += 64 * WAVES) {
        const int tok = e / RW, r = at.r0 + e % RW;
        const int to = __shfl(row, tok);
        if (!(match >> tok & 1u) || r >= P.Rp) continue;
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) s += lds[w][tok][e % RW];
        P.low[low_at(P, blockIdx.y, to, r)] = r < at.rank ? s : 0.f;
      }
      __syncthreads();
    }
  }
}

// out = base + scale B_a low.  A workgroup has 256 outputs of its tokens, a wavefront 64 of them as four tiles of 16, whose rows are
// chosen so that a lane's 16 outputs are neighbours.
__device__ __forceinline__ int out_row(int tile, int i) { return (i >> 2) * 16 + tile * 4 + (i & 3); }

// A lane's outputs as kOuts pieces of 16 bytes.  kOuts neighbouring lanes read and write one token after the other, a piece each, and
// exchange the pieces (k_unit has the reason).
template <int OK>
struct out_pieces {
  static constexpr int kOuts = OK == CQ_A_F32 ? 4 : 2, kOut = OK == CQ_A_F32 ? 4 : 8, kSize = OK == CQ_A_F32 ? 4 : 2;
  cq_v4u w[kOuts];
  // the first output of the piece that this lane moves for its neighbours
  static __device__ __forceinline__ int moved(int n0, int g) { return n0 + g * 16 + (int)(threadIdx.x & (kOuts - 1)) * kOut; }
  // token[n]: of the n-th of the neighbouring lanes, -1: none
  __device__ __forceinline__ void fetch(const adapter_args& P, const int (&token)[kOuts], int n0, int g) {
    const int at = moved(n0, g);
#pragma unroll
    for (int n = 0; n < kOuts; ++n) {
      w[n] = cq_v4u{0u, 0u, 0u, 0u};
      if (P.base && token[n] >= 0 && at + kOut <= P.N)
        w[n] = *reinterpret_cast<const cq_v4u_any*>(reinterpret_cast<const char*>(P.base) + ((size_t)token[n] * P.ldb + at) * kSize);
    }
  }
  __device__ __forceinline__ void store(const adapter_args& P, const int (&token)[kOuts], int n0, int g) const {
    const int at = moved(n0, g);
#pragma unroll
    for (int n = 0; n < kOuts; ++n)
      if (token[n] >= 0 && at + kOut <= P.N)
        *reinterpret_cast<cq_v4u_any*>(reinterpret_cast<char*>(P.out) + ((size_t)token[n] * P.ldo + at) * kSize) = w[n];
  }
  __device__ __forceinline__ void exchange() {
    if constexpr (kOuts == 4) {
      quad_transpose(w);
    } else {
      const bool odd = threadIdx.x & 1;
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        const uint32_t a = w[0][d], b = w[1][d];
        const uint32_t from_b = __builtin_amdgcn_update_dpp(0u, b, 0xb1, 0xf, 0xf, false);
        const uint32_t from_a = __builtin_amdgcn_update_dpp(0u, a, 0xb1, 0xf, 0xf, false);
        w[0][d] = odd ? from_b : a;
        w[1][d] = odd ? b : from_a;
      }
    }
  }
};

// raw values from, from + 1, ... of eight, zeros behind them
template <int KIND>
__device__ __forceinline__ void drop_values(row8<KIND>& r, int from) {
#pragma unroll
  for (int bit = 1; bit < 8; bit *= 2) {
    const bool move = from & bit;
    if constexpr (KIND == CQ_A_F32) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t next = i + bit < 8 ? r.w[(i + bit) >> 2][(i + bit) & 3] : 0u;
        r.w[i >> 2][i & 3] = move ? next : r.w[i >> 2][i & 3];
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t up = i < 3 ? r.w[0][i + 1 < 4 ? i + 1 : 3] : 0u, far = i < 2 ? r.w[0][i + 2 < 4 ? i + 2 : 3] : 0u;
        const uint32_t next = bit == 1 ? (r.w[0][i] >> 16 | up << 16) : bit == 2 ? up : far;
        r.w[0][i] = move ? next : r.w[0][i];
      }
    }
  }
}

// Columns r .. r+7 of B's rows n0 .. n0+63 (four tiles) where r < most, zeros beyond the row.  A row that is no whole number of
// eights: its last eight are read and moved into place.  SHORT: rows may have
// fewer than eight values, or be no whole number of eights.
template <int WK, int OK, bool SHORT>
__device__ __forceinline__ void fetch_up(const adapter_args& P, int a, int n0, int col, int r, int most, row8<WK> (&w)[4]) {
  const size_t w_row = ((size_t)a * P.N + n0) * P.R;
  const int c = !SHORT ? r : P.R >= 8 ? min(r, P.R - 8) : 0;   // (not SHORT: whole eights)
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int n = out_row(j, col);
    const bool on = r < most && n0 + n < P.N;
    if (!SHORT || P.R >= 8) w[j] = fetch8<WK>(P.B, w_row, (uint32_t)(n * P.R + c), on);
    else w[j] = row_fetch<WK>(P.B, w_row + n * P.R, on ? P.R : 0);
  }
  if (SHORT && P.R % 8 != 0 && P.R >= 8) {
#pragma unroll
    for (int j = 0; j < 4; ++j) drop_values(w[j], r < P.R ? r - c : 0);
  }
}

// Columns beyond the adapter's rank may be anything, and 0 times an infinite x is no 0: cleared in both operands.
template <int WK>
__device__ __forceinline__ void keep_rank(int r, int rank, row8<WK> (&w)[4]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) keep_values(w[j], 0, rank - r);
}
__device__ __forceinline__ void keep_rank(int r, int rank, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = r + i < rank ? v[i] : 0.f;
}

template <int WK, bool FINITE>
__device__ __forceinline__ void up_product(const row8<WK> (&w)[4], const float (&v)[8], cq_v4f (&acc)[4]) {
  if constexpr (WK == CQ_A_BF16) {
    const split_frag vs = split_pack(v);
    if constexpr (FINITE) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {   // (one after the other: the rare form adds few registers)
        const cq_v8bf16 rest = finite_weights(w[j].w[0]);
        acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(cq_v8bf16, w[j].w[0]), vs.part[0], acc[j], 0, 0, 0);
        acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(rest, vs.part[1], acc[j], 0, 0, 0);
        acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(rest, vs.part[2], acc[j], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
      return;
    }
#pragma unroll
    for (int p = 0; p < 3; ++p)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(cq_v8bf16, w[j].w[0]), vs.part[p], acc[j], 0, 0, 0);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float u[8];
      row_values<WK>(w[j], u);
#pragma unroll
      for (int q = 0; q < 8; ++q) acc[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(u[q], v[q], acc[j], 0, 0, 0);
    }
  }
}

// acc = sum<FINITE>(acc) on zeros, see finite_weights
template <int WK, typename SUM>
__device__ __forceinline__ void up_sums(cq_v4f (&acc)[4], SUM&& sum) {
#pragma unroll
  for (int j = 0; j < 4; ++j) acc[j] = cq_v4f{0.f, 0.f, 0.f, 0.f};
  sum(std::false_type{});
  if constexpr (WK == CQ_A_BF16) {
    if (__builtin_expect(!any_nan(acc), 1)) return;
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[j] = cq_v4f{0.f, 0.f, 0.f, 0.f};
    sum(std::true_type{});
  }
}

// out = base + scale acc of the lane's own token t (-1: none), and of its neighbours' (token)
template <int OK>
__device__ __forceinline__ void store_out(const adapter_args& P, int t, const int (&token)[out_pieces<OK>::kOuts], int n0, int g, bool any,
                                          float scale, const cq_v4f (&acc)[4], out_pieces<OK> base) {
  using L = out_pieces<OK>;
  base.exchange();
  L out;
#pragma unroll
  for (int o = 0; o < L::kOuts; ++o) {
    float add[8], v[8];
#pragma unroll
    for (int i = 0; i < L::kOut; ++i) add[i] = acc[o * (L::kOut / 4) + (i >> 2)][i & 3];
    if constexpr (OK == CQ_A_F32) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float b = __uint_as_float(base.w[o][i]);
        out.w[o][i] = __float_as_uint(any ? fmaf(scale, add[i], b) : b);
      }
    } else {
      row8<OK> b;
      b.w[0] = base.w[o];
      row_values<OK>(b, v);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t pair = 0;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float x = fmaf(scale, add[2 * i + h], v[2 * i + h]);
          const uint16_t bits = OK == CQ_A_BF16 ? __builtin_bit_cast(uint16_t, (__bf16)x) : __builtin_bit_cast(uint16_t, (_Float16)x);
          pair |= (uint32_t)bits << (16 * h);
        }
        out.w[o][i] = any ? pair : base.w[o][i];
      }
    }
    const int n = n0 + g * 16 + o * L::kOut;
    if (n + L::kOut > P.N && t >= 0) {   // the row ends within these outputs
#pragma unroll
      for (int i = 0; i < L::kOut; ++i) {
        if (n + i >= P.N) continue;
        float x = P.base ? elem_load<OK>(P.base, (size_t)t * P.ldb + n + i) : 0.f;
        if (any) x = fmaf(scale, add[i], x);
        elem_store<OK>(P.out, (size_t)t * P.ldo + n + i, x);
      }
    }
  }
  out.exchange();
  out.store(P, token, n0, g);
}

// Single tokens: up to 16 of one adapter per workgroup.  Bound by latency: base, low and the first 32 columns of B are asked for
// together, the latter before the adapter's own rank is known and cleared beyond it (B's rows are short).
// WIDE: several blocks of outputs per workgroup, one after the other.
template <int WK, int OK, bool WIDE>
__global__ __launch_bounds__(64 * kUpWaves, WIDE ? 3 : 4) void adapter_up_kernel(adapter_args P) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int col = lane & 15, g = lane >> 4;
  const int up_blocks = WIDE ? P.up_blocks : 1, wide = 64 * kUpWaves * up_blocks, blocks = (P.N + wide - 1) / wide, group = blockIdx.x / blocks;
  const int tile = tile_of_group(P, group), first = ((int)blockIdx.x - group * blocks) * wide + wave * 64;
  if (first >= P.N) return;
  int row, id;
  if (!find_rows<kTile>(P, tile, row, id)) return;
  const int t = __shfl(row, col), a = __builtin_amdgcn_readlane(id, 0);
  constexpr int kOuts = out_pieces<OK>::kOuts;
  int token[kOuts];
#pragma unroll
  for (int n = 0; n < kOuts; ++n) token[n] = __shfl(row, (col & (16 - kOuts)) + n);
  const int rank = rank_of(P, a);
  const float scale = a >= 0 && P.scale ? P.scale[a] : 1.f;
#pragma unroll 1
  for (int block = 0; block < up_blocks; ++block) {
    const int n0 = first + block * 64 * kUpWaves;
    if (n0 >= P.N) break;
    out_pieces<OK> base;
    base.fetch(P, token, n0, g);
    cq_v4f acc[4];
    up_sums<WK>(acc, [&](auto finite) {
      for (int rb = 0; a >= 0 && (rb == 0 || rb < rank); rb += 32) {
        const int r = rb + g * 8, most = rb == 0 ? P.R : rank;
        row8<WK> w[4];
        fetch_up<WK, OK, true>(P, a, n0, col, r, most, w);
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0.f;
        if (t >= 0 && r < most) {
#pragma unroll 4
          for (int p = 0; p < P.parts; ++p) {
            float u[8];
            row_values<CQ_A_F32>(fetch8<CQ_A_F32>(P.low, low_at(P, p, t, r), 0, true), u);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += u[i];
          }
        }
        if (rank < rb + 32) {
          keep_rank(r, rank, v);
          keep_rank<WK>(r, rank, w);
        }
        up_product<WK, finite.value>(w, v, acc);
      }
    });
    store_out<OK>(P, t, token, n0, g, rank > 0, scale, acc, base);
  }
}

// Few tokens of low rank in one launch: every workgroup of 512 outputs takes the whole of A_a x_t for itself, so that nothing
// passes through memory, at the price of reading A (from L2) once per workgroup.  Bound by latency: base and B are asked for
// before A.
template <int XK, int WK, int OK, int RT>
__global__ __launch_bounds__(64 * kFewWaves) void adapter_few_kernel(adapter_args P) {
  constexpr int UNITS = most_units<XK, WK, RT>(), LD = RT * 16 + 4;
  __shared__ float lds[kFewWaves][16][LD];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int col = lane & 15, g = lane >> 4;
  const int blocks = (P.N + 64 * kFewWaves - 1) / (64 * kFewWaves), group = blockIdx.x / blocks;
  const int tile = tile_of_group(P, group), n0 = (((int)blockIdx.x - group * blocks) * kFewWaves + wave) * 64;
  int row, id;
  if (!find_rows<kTile>(P, tile, row, id)) return;
  const int t = __shfl(row, col), a = __builtin_amdgcn_readlane(id, 0);
  down_place at;
  place_tokens(P, row, at);
  constexpr int kOuts = out_pieces<OK>::kOuts;
  int token[kOuts];
#pragma unroll
  for (int n = 0; n < kOuts; ++n) token[n] = __shfl(row, (col & (16 - kOuts)) + n);
  out_pieces<OK> base;
  base.fetch(P, token, n0, g);
  const int r = g * 8, rank = rank_of(P, a);
  const float scale = a >= 0 && P.scale ? P.scale[a] : 1.f;
  cq_v4f out[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) out[j] = cq_v4f{0.f, 0.f, 0.f, 0.f};
  if (rank > 0) {
    row8<WK> b[4];
    fetch_up<WK, OK, true>(P, a, n0, col, r, rank, b);
    at.a = a;
    at.rank = rank;
    at.r0 = 0;
    constexpr bool kOwn = XK == CQ_A_F32;
    if (kOwn) at.x_row[0] = at.own_row;
    k_unit<XK, kOwn> x[UNITS];
    cq_v4f acc[RT];
#pragma unroll
    for (int i = 0; i < RT; ++i) acc[i] = cq_v4f{0.f, 0.f, 0.f, 0.f};
    down_rounds<XK, WK, RT, UNITS, kFewWaves, false, kOwn>(P, at, 0, P.K, false, x, acc);
    down_again<XK, WK, RT, UNITS, kFewWaves, kOwn>(P, at, 0, P.K, x, acc);
#pragma unroll
    for (int i = 0; i < RT; ++i) *reinterpret_cast<cq_v4f*>(&lds[wave][col][i * 16 + g * 4]) = acc[i];
    __syncthreads();
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 0.f;
    if (r < rank) {
#pragma unroll
      for (int w = 0; w < kFewWaves; ++w)
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += lds[w][col][r + i];
    }
    keep_rank(r, rank, v);
    keep_rank<WK>(r, rank, b);
    up_sums<WK>(out, [&](auto finite) { up_product<WK, finite.value>(b, v, out); });
  }
  store_out<OK>(P, t, token, n0, g, rank > 0, scale, out, base);
}

// Prompts: two tiles of 16 neighbouring tokens, whose base and low are asked for before the ids are known; the adapter's first 32 NB
// columns of B stay in registers from tile to tile.  Bound by HBM (base in, out written).
// Outputs first, tokens second: workgroups that run together write whole rows, and where there is a multiple of 8 blocks of outputs
// an XCD meets the same rows of B again and again.
// ANY: ranks beyond 32 NB, below 8, or that are no multiple of 8.
template <int WK, int OK, int NB, bool ANY>
__global__ __launch_bounds__(64 * kUpWaves, ANY || (NB == 2 && (WK == CQ_A_F32 || OK == CQ_A_F32)) ? 2
                                            : NB == 1 && WK != CQ_A_F32 && OK != CQ_A_F32          ? 4
                                                                                                   : 3)
void adapter_up_prompt_kernel(adapter_args P) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int col = lane & 15, g = lane >> 4;
  const int blocks = (P.N + 64 * kUpWaves - 1) / (64 * kUpWaves), chunk = blockIdx.x / blocks;
  const int n0 = (((int)blockIdx.x - chunk * blocks) * kUpWaves + wave) * 64;
  if (n0 >= P.N) return;
  struct ahead {
    out_pieces<OK> base;
    row8<CQ_A_F32> low[NB];
  } tiles[kPromptTiles];
  constexpr int kOuts = out_pieces<OK>::kOuts;
  const int first = chunk * kPromptTiles;
  auto neighbour = [&](int i, int n) { return (first + i) * kTile + (col & (16 - kOuts)) + n; };
  const int mine = first * kTile + lane;
  const int id = lane < kPromptTiles * kTile && mine < P.T ? adapter_of(P, mine) : -1;
#pragma unroll
  for (int i = 0; i < kPromptTiles; ++i) {
    const int t = (first + i) * kTile + col;
    int token[kOuts];
#pragma unroll
    for (int n = 0; n < kOuts; ++n) token[n] = neighbour(i, n) < P.T ? neighbour(i, n) : -1;
    tiles[i].base.fetch(P, token, n0, g);
#pragma unroll
    for (int b = 0; b < NB; ++b)
      tiles[i].low[b] = fetch8<CQ_A_F32>(P.low, low_at(P, 0, t, b * 32 + g * 8), 0, t < P.T && b * 32 + g * 8 < P.R);
  }
  int have = -1, rank = 0;
  float scale = 1.f;
  row8<WK> w[NB][4];
#pragma unroll
  for (int i = 0; i < kPromptTiles; ++i) {
    const int t = (first + i) * kTile + col;
    unsigned todo = (unsigned)(__ballot(mine < P.T) >> (i * kTile)) & 0xffffu;
    while (todo) {
      const int a = __builtin_amdgcn_readlane(id, i * kTile + __ffs(todo) - 1);
      const unsigned match = (unsigned)(__ballot(id == a) >> (i * kTile)) & todo;
      todo &= ~match;
      if (a != have) {
        have = a;
        rank = rank_of(P, a);
        scale = a >= 0 && P.scale ? P.scale[a] : 1.f;
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          fetch_up<WK, OK, ANY>(P, a, n0, col, b * 32 + g * 8, a >= 0 ? rank : 0, w[b]);
          if (rank < b * 32 + 32) keep_rank<WK>(b * 32 + g * 8, rank, w[b]);
        }
      }
      cq_v4f acc[4];
      up_sums<WK>(acc, [&](auto finite) {
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          if (rank <= b * 32) continue;
          float v[8];
          row_values<CQ_A_F32>(tiles[i].low[b], v);
          if (rank < b * 32 + 32) keep_rank(b * 32 + g * 8, rank, v);
          up_product<WK, finite.value>(w[b], v, acc);
        }
#pragma unroll 1
        for (int rb = NB * 32; ANY && rb < rank; rb += 32) {   // ranks beyond the registers
          const int r = rb + g * 8;
          row8<WK> more[4];
          fetch_up<WK, OK, ANY>(P, a, n0, col, r, rank, more);
          float v[8];
          row_values<CQ_A_F32>(fetch8<CQ_A_F32>(P.low, low_at(P, 0, t, r), 0, t < P.T && r < rank), v);
          if (rank < rb + 32) {
            keep_rank(r, rank, v);
            keep_rank<WK>(r, rank, more);
          }
          up_product<WK, finite.value>(more, v, acc);
        }
      });
      int token[kOuts];
#pragma unroll
      for (int n = 0; n < kOuts; ++n) token[n] = match >> ((col & (16 - kOuts)) + n) & 1 ? neighbour(i, n) : -1;
      store_out<OK>(P, match >> col & 1 ? t : -1, token, n0, g, rank > 0, scale, acc, tiles[i].base);
    }
  }
}

cq_status check_adapters(const cq_adapters* W, int T) {
  if (!W) return CQ_ERR_NULL;
  if (T < 0 || T > 1 << 30 || W->n <= 0 || W->rank <= 0 || W->rank > kMaxRank || W->K <= 0 || W->N <= 0) return CQ_ERR_SHAPE;
  if (W->K > 1 << 23 || W->N > 1 << 23) return CQ_ERR_SHAPE;
  if (!cq_row_kind(W->kind)) return CQ_ERR_UNSUPPORTED;
  return CQ_OK;
}

int padded_rank(int R) { return (R + 15) / 16 * 16; }

// Units of 128 values per wavefront and round, and parts of K.  Prompts: one part.  Single tokens: parts of whole rounds, as many
// units as leave two workgroups per compute unit, at most 16 parts.
struct down_plan { int units, parts, kpart; };

down_plan plan_of(int T, int K) {
  down_plan d;
  d.units = 4;
  d.parts = 1;
  d.kpart = K;
  if (T > kLeaderTokens) return d;
  const int tiles = (T + kTile - 1) / kTile;
  auto rounds = [&](int units) { return (K + 128 * kDownWaves * units - 1) / (128 * kDownWaves * units); };
  while (d.units > 1 && tiles * rounds(d.units) < 512) d.units /= 2;
  const int n = rounds(d.units);
  int parts = 512 / tiles;
  if (parts > n) parts = n;
  if (parts > 16) parts = 16;
  if ((long)parts * T > kMostGroups) parts = kMostGroups / T;
  d.kpart = (n + parts - 1) / parts * 128 * kDownWaves * d.units;
  d.parts = (K + d.kpart - 1) / d.kpart;
  return d;
}

// One launch instead of two where A is small and its copies are few: up to 65536 values per adapter, read by up to 256 workgroups that
// read 2^23 values between them.  Every workgroup repeats the products of A, so K times the tiles of 16 ranks is bounded by what a product
// costs: 8192 for 16-bit types, 4096 for cut fp32 rows, 2048 on the fp32 matrix cores.  The bounds stand where the one launch's own time has
// caught up with the two's (graph replays); called from Python a launch is another 3 us.  One token, N = 2048 to 4096, one / two
// launches (us), graph, then Python:
//   bf16 rows, bf16 weights   rank 16, K = 2048  6.4 / 8.2, 8.5 / 12.6   rank 16, 4096  8.3 / 9.2, 8.5 / 12.5   rank 8, 8192  11.6 / 11.2, 11.6 / 12.5
//                             rank 4, 16384  19.5 / 13.1, 19.5 / 13.4
//   fp32 rows, bf16 weights   rank 16, K = 2048  7.9 / 9.2, 8.3 / 12.1   rank 16, 4096  10.9 / 10.6, 10.8 / 12.3   rank 8, 5120  12.0 / 10.9, 11.8 / 12.6
//                             rank 8, 8192  16.5 / 12.3, 16.3 / 12.7
//   bf16 rows, fp32 weights   rank 16, K = 2048  10.4 / 9.4, 10.3 / 12.7   rank 32, 2048  15.6 / 10.8, 15.3 / 12.6   rank 16, 4096  15.2 / 10.5, 15.0 / 12.7
bool takes_few(const cq_adapters* W, int x_kind, int T) {
  const long values = (long)W->rank * W->K, blocks = ((long)W->N + 64 * kFewWaves - 1) / (64 * kFewWaves);
  const int path = x_kind == W->kind && x_kind != CQ_A_F32 ? kSame16 : x_kind == CQ_A_F32 && W->kind == CQ_A_BF16 ? kSplit : kFloat;
  const long most = path == kSame16 ? 8192 : path == kSplit ? 4096 : 2048;
  return W->rank <= 32 && values <= 65536 && blocks * T <= 256 && values * blocks * T <= 1l << 23 && (long)W->K * ((W->rank + 15) / 16) <= most;
}

// Tokens of one pair of launches (at least 8192); longer batches take several.
int most_tokens(const cq_adapters* W) {
  const long blocks = ((long)W->N + 64 * kUpWaves - 1) / (64 * kUpWaves);
  const long down = kMostThreads / (64 * kPromptDownWaves) * kTile, up = kMostThreads / (64 * kUpWaves) / blocks * kTile * kPromptTiles;
  return (int)(down < up ? down : up);
}

}  // namespace

extern "C" size_t cq_adapter_workspace_bytes(const cq_adapters* W, int x_kind, int T) {
  if (check_adapters(W, T) != CQ_OK || !cq_row_kind(x_kind) || takes_few(W, x_kind, T)) return 0;
  if (T > most_tokens(W)) T = most_tokens(W);
  // no batch of T <= kLeaderTokens has more parts than 512 over its tiles, nor than 16, nor than there are rounds of one unit
  const long most = ((long)W->K + 128 * kDownWaves - 1) / (128 * kDownWaves), cap = most < 16 ? most : 16;
  long rows = ((long)T + kTile - 1) / kTile * kTile;
  for (long p = 2; p <= cap; ++p) {
    long last = 512 / p * kTile;   // the longest batch with p parts
    if (last > kLeaderTokens) last = kLeaderTokens;
    const long t = (T < last ? T : last) + kTile - 1;
    if (t / kTile * kTile * p > rows) rows = t / kTile * kTile * p;
  }
  return cq_align_up((size_t)rows * padded_rank(W->rank) * 4, 256);
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
  const size_t need = cq_adapter_workspace_bytes(W, x_kind, T);
  if (need > 0 && (!workspace || workspace_bytes < need)) return CQ_ERR_WORKSPACE;
  const int most = most_tokens(W);
  if (T > most) {
    cq_status done = CQ_OK;
    for (int t = 0; t < T && done == CQ_OK; t += most)
      done = cq_adapter_apply(W, row_at(X, x_kind, (size_t)t * ldx), x_kind, ldx, adapter_ids + t, T - t < most ? T - t : most,
                              row_at(base, out_kind, (size_t)t * ld_base), ld_base, row_at(out, out_kind, (size_t)t * ld_out), out_kind,
                              ld_out, workspace, workspace_bytes, stream);
    return done;
  }
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
  P.tiles = (T + kTile - 1) / kTile;
  const down_plan plan = plan_of(T, W->K);
  P.parts = plan.parts;
  P.kpart = plan.kpart;
  P.ldx = (size_t)ldx;
  P.ldb = base ? (size_t)ld_base : 0;
  P.ldo = (size_t)ld_out;
  hipStream_t s = (hipStream_t)stream;
  const bool leaders = T <= kLeaderTokens;
  if (takes_few(W, x_kind, T)) {
    const dim3 few((unsigned)((T + 7) / 8 * 8 * (((long)W->N + 64 * kFewWaves - 1) / (64 * kFewWaves))));
#define FEW3(XK, WK, OK, RT) hipLaunchKernelGGL((adapter_few_kernel<XK, WK, OK, RT>), few, dim3(64 * kFewWaves), 0, s, P)
#define FEW2(XK, WK, OK)                     \
  do {                                       \
    if (W->rank <= 16) FEW3(XK, WK, OK, 1);  \
    else FEW3(XK, WK, OK, 2);                \
  } while (0)
#define FEW1(XK, WK)                                     \
  do {                                                   \
    if (out_kind == CQ_A_F32) FEW2(XK, WK, CQ_A_F32);    \
    else if (out_kind == CQ_A_F16) FEW2(XK, WK, CQ_A_F16); \
    else FEW2(XK, WK, CQ_A_BF16);                        \
  } while (0)
#define FEW(XK)                                          \
  do {                                                   \
    if (W->kind == CQ_A_F32) FEW1(XK, CQ_A_F32);         \
    else if (W->kind == CQ_A_F16) FEW1(XK, CQ_A_F16);    \
    else FEW1(XK, CQ_A_BF16);                            \
  } while (0)
    if (x_kind == CQ_A_F32) FEW(CQ_A_F32);
    else if (x_kind == CQ_A_F16) FEW(CQ_A_F16);
    else FEW(CQ_A_BF16);
    return cq_check_launch();
  }
  const int singles = (T + 7) / 8 * 8;   // (tile_of_group stays within eight)
  const dim3 down(leaders ? singles : ((T + kTile - 1) / kTile + 7) / 8 * 8, P.parts, (W->rank + kRankBlock - 1) / kRankBlock);
  const long blocks = ((long)W->N + 64 * kUpWaves - 1) / (64 * kUpWaves);
  P.up_blocks = leaders ? (int)((blocks * T + kMostGroups - 1) / kMostGroups) : 1;
  const long up_tiles = leaders ? singles : ((long)T + kTile * kPromptTiles - 1) / (kTile * kPromptTiles);
  const dim3 up((unsigned)(up_tiles * ((blocks + P.up_blocks - 1) / P.up_blocks)));
#define DOWN3(XK, WK, RT, UNITS, WAVES) hipLaunchKernelGGL((adapter_down_kernel<XK, WK, RT, UNITS, WAVES>), down, dim3(64 * WAVES), 0, s, P)
#define DOWN2(XK, WK, RT)                                                              \
  do {                                                                                 \
    constexpr int kMost = most_units<XK, WK, RT>(), kTwo = kMost < 2 ? kMost : 2;      \
    if (!leaders) DOWN3(XK, WK, RT, kMost, kPromptDownWaves);                          \
    else if (plan.units == 1) DOWN3(XK, WK, RT, 1, kDownWaves);                        \
    else if (plan.units == 2) DOWN3(XK, WK, RT, kTwo, kDownWaves);                     \
    else DOWN3(XK, WK, RT, kMost, kDownWaves);                                         \
  } while (0)
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
#define UP_SINGLE(WK, OK, WIDE) hipLaunchKernelGGL((adapter_up_kernel<WK, OK, WIDE>), up, dim3(64 * kUpWaves), 0, s, P)
#define UP_PROMPT(WK, OK, NB, ANY) hipLaunchKernelGGL((adapter_up_prompt_kernel<WK, OK, NB, ANY>), up, dim3(64 * kUpWaves), 0, s, P)
#define UP2(WK, OK)                                                                                                     \
  do {                                                                                                                  \
    if (leaders && P.up_blocks > 1) UP_SINGLE(WK, OK, true);                                                            \
    else if (leaders) UP_SINGLE(WK, OK, false);                                                                         \
    else if (W->rank % 8 != 0 || W->rank > 64) UP_PROMPT(WK, OK, 1, true);                                                   \
    else if (W->rank <= 32) UP_PROMPT(WK, OK, 1, false);                                                                \
    else UP_PROMPT(WK, OK, 2, false);                                                                                   \
  } while (0)
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
