// Attention tiles on 32x32x16 MFMA: the pieces shared by the kernels whose waves hold 32
// query rows as the columns of their products.
//
//   S^T[token, row] = K[token, :] . q[row, :]     O^T[channel, row] += V^T[channel, token] P^T[token, row]
//
// Lane l of a wave holds query row l % 32 of every product, so a row's running maximum and
// sum live in lanes r and r + 32 and need no transposition.  Of a 32-token subtile S^T puts
// product rows 8 q + 4 h + r (q, r = 0..3) into half h = l / 32 as element e = 4 q + r, and
// the second product takes its k-slots in that order: k-step x = 0, 1 of the subtile reads the
// half's elements 8 x .. 8 x + 7, straight from the registers that the softmax left.
#pragma once

#include "kvk_device.h"

namespace kvkd {

typedef float f16v __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f2v __attribute__((ext_vector_type(2)));

constexpr float kLn2 = 0.6931471805599453f;

template <bool HALF>
__device__ __forceinline__ f16v mfma32(u4v a, u4v b, f16v c) {
  if constexpr (HALF) return __builtin_amdgcn_mfma_f32_32x32x16_f16(bitcast<half8>(a), bitcast<half8>(b), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_32x32x16_bf16(bitcast<bf16x8>(a), bitcast<bf16x8>(b), c, 0, 0, 0);
}

__device__ __forceinline__ f16v zero16() {
  f16v z;
#pragma unroll
  for (int e = 0; e < 16; ++e) z[e] = 0.0f;
  return z;
}

// Over the two halves of the wave (lanes l and l ^ 32).
__device__ __forceinline__ float halves_max(float x) {
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float halves_sum(float x) {
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// Two values rounded to nearest even, the first in the low half.
template <bool HALF>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  if constexpr (HALF) {
    return bitcast<uint32_t>(h2(a, b));
  } else {
    const bf16x2 r = __builtin_convertvector((f2v{a, b}), bf16x2);
    return bitcast<uint32_t>(r);
  }
}

// Product row of element e in half h of a 32-token subtile.
__device__ __forceinline__ constexpr int tile_row(int e, int h) { return 8 * (e >> 2) + 4 * h + (e & 3); }

// Transposing read of LDS: of sixteen lanes, four each point at sixteen consecutive 16-bit values
// of one row (lane 4 r + i at values 4 i .. 4 i + 3 of row r); lane n receives value n of the four
// rows.  (The layout was checked on gfx950 lane by lane.)
__device__ __forceinline__ u2v read_transposed(const uint8_t* p) {
  typedef short s4v __attribute__((ext_vector_type(4)));
  return bitcast<u2v>(__builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4v*)(p)));
}

// Running state of a wave's 32 query rows: output accumulators (32 NM channels), reference
// maximum in base-2 logits, and the lane's share of the sum.
// Scaled values: a subtile whose values enter the product multiplied by 2^drop gets its logits
// lowered by drop instead (softmax_step's argument), and its part of the sum multiplied by 2^drop;
// the reference is then the maximum of the lowered logits, so that probabilities and scaled
// values both stay in range.  (drop 0, the default, costs nothing: x - 0 and 1 x fold.)
template <int NM>
struct RowState {
  f16v o[NM];
  float m, l;
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < NM; ++i) o[i] = zero16();
    m = -INFINITY;
    l = 0.0f;
  }
};

// A row's reference moves only when a logit exceeds it by more than this (base-2): the
// accumulators hold values up to 2^kSlack times larger than with the true maximum, in fp32,
// and most steps need no rescaling.
constexpr float kSlack = 8.0f;

// The largest base-2 logit of a row's scores s (times c = log2-scale, c > 0).
__device__ __forceinline__ float top_logit(const f16v& s, float c, float drop) {
  float mx = s[0];
#pragma unroll
  for (int e = 0; e < 16; ++e) mx = fmaxf(mx, s[e]);
  return halves_max(mx) * c - drop;
}
// What a reference that moves from m to mnew leaves of the sums.  (A row without mass has outputs
// of 0, or infinities and NaN by take_nonfinite: they stay.)
__device__ __forceinline__ float rescale(float m, float mnew) {
  return m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - mnew);
}
// Probabilities 2^(c s - drop - m + bias) of scores s, packed for the second product in p; their
// sum.  A row whose logits have all been -inf so far keeps the reference -inf, and its
// probabilities 2^(-inf) = 0 are formed against 0.  rest: NULL, or what the rounding to bf16 left of them (p and
// rest together hold 16 bits).
template <bool HALF>
__device__ __forceinline__ float probabilities(float m, const f16v& s, float c, float bias, u4v (&p)[2],
                                               float drop, u4v* rest = nullptr) {
  const float ref = (m == -INFINITY ? 0.0f : m) - (bias - drop);
  float sum = 0.0f;
#pragma unroll
  for (int x = 0; x < 2; ++x)
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const int e = 8 * x + 2 * w;
      const float a = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], c, -ref));
      const float b = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e + 1], c, -ref));
      sum += a + b;
      p[x][w] = pack2<HALF>(a, b);
      if (rest)
        rest[x][w] = pack2<HALF>(a - __uint_as_float(p[x][w] << 16), b - __uint_as_float(p[x][w] & 0xffff0000u));
    }
  return sum;
}
// One online-softmax step over a subtile; grow = 2^drop.
template <int NM, bool HALF>
__device__ __forceinline__ void softmax_step(RowState<NM>& st, const f16v& s, float c, float bias, u4v (&p)[2],
                                             u4v* rest = nullptr, float drop = 0.0f, float grow = 1.0f) {
  const float mx = top_logit(s, c, drop);
  if (__any(mx > st.m + kSlack)) {
    const float mnew = fmaxf(st.m, mx), alpha = rescale(st.m, mnew);
    st.m = mnew;
    st.l *= alpha;
#pragma unroll
    for (int i = 0; i < NM; ++i) st.o[i] *= alpha;
  }
  st.l += grow * probabilities<HALF>(st.m, s, c, bias, p, drop, rest);
}

// Whether any of the eight bf16 / fp16 values of a 16-byte unit is infinite or NaN.
template <bool HALF>
__device__ __forceinline__ bool any_nonfinite(u4v w) {
  constexpr uint32_t kExp = HALF ? 0x7c00u : 0x7f80u;
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) bad |= (w[i] & kExp) == kExp || ((w[i] >> 16) & kExp) == kExp;
  return bad;
}
// The unit with its infinite and NaN values replaced by zero.
template <bool HALF>
__device__ __forceinline__ u4v only_finite(u4v w) {
  constexpr uint32_t kExp = HALF ? 0x7c00u : 0x7f80u;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if ((w[i] & kExp) == kExp) w[i] &= 0xffff0000u;
    if (((w[i] >> 16) & kExp) == kExp) w[i] &= 0x0000ffffu;
  }
  return w;
}

// Infinite and NaN values in a subtile that some rows may not see wholly: a masked place has
// probability 0, and 0 times infinity would reach every row of the product.  Before the subtile's
// softmax_step the values a row does see are counted by kind in products of indicators, and each
// kind present is added to the row's outputs, as the plain product would: a probability p > 0 times
// an infinity or a NaN is that value, p = 0 (a score of -inf, or underflow) times an infinity is
// NaN.  The caller then takes its steps with the finite values.  m: the reference before the
// subtile, st.m or what this call returned for the subtile before it; returns the one after it.
// unit(x, t): the value operand of k-step x, channel tile t; hidden(e): all ones where the row does
// not see element e, else 0.  Rare.
template <int NM, bool HALF, class Unit, class Hidden>
__device__ __forceinline__ float take_nonfinite(RowState<NM>& st, float m, const f16v& s, float c, float bias, Unit unit,
                                                Hidden hidden, float drop = 0.0f) {
  constexpr uint32_t kOne = HALF ? 0x3c00u : 0x3f80u, kExp = HALF ? 0x7c00u : 0x7f80u;
  const float mx = top_logit(s, c, drop);
  if (__any(mx > m + kSlack)) {
    const float mnew = fmaxf(m, mx), alpha = rescale(m, mnew);
    if (__any(alpha == 0.0f)) {  // now: after what is added here it would make NaN of it
      const float before = rescale(st.m, m);  // of the subtiles before, whose steps are yet to come
      st.m = mnew;
      st.l = st.l * before * alpha;
#pragma unroll
      for (int i = 0; i < NM; ++i) st.o[i] = st.o[i] * before * alpha;
    }
    m = mnew;
  }
  u4v p[2];
  probabilities<HALF>(m, s, c, bias, p, drop);
#pragma unroll 1
  for (int kind = 0; kind < 4; ++kind) {  // +infinity and -infinity (p > 0), NaN, either infinity (p = 0)
    asm volatile("" ::: "memory");  // (units read again for each kind, not held in registers)
    // a 16-bit value b is of the kind if (b & keep) - lo < span (unsigned)
    const uint32_t keep = kind >= 2 ? 0x7fffu : 0xffffu;
    const uint32_t lo = kind == 1 ? kExp | 0x8000u : (kind == 2 ? kExp + 1 : kExp);
    const uint32_t span = kind == 2 ? 0x8000u - (kExp + 1) : 1u;
    const bool some = kind != 3, none = kind >= 2;  // the probabilities that count: p > 0, p = 0
#pragma unroll
    for (int t = 0; t < NM; ++t) {
      f16v n = zero16();
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        u4v v = unit(x, t), seen;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const int e = 8 * x + 2 * w;
          const bool lo_counts = (p[x][w] & 0xffffu) ? some : none, hi_counts = (p[x][w] >> 16) ? some : none;
          seen[w] = (lo_counts ? kOne & ~hidden(e) : 0u) | (hi_counts ? (kOne << 16) & ~hidden(e + 1) : 0u);
          v[w] = ((v[w] & keep) - lo < span ? kOne : 0u) | (((v[w] >> 16) & keep) - lo < span ? kOne << 16 : 0u);
        }
        n = mfma32<HALF>(v, seen, n);
      }
      const float add = kind == 0 ? INFINITY : (kind == 1 ? -INFINITY : __builtin_nanf(""));
#pragma unroll
      for (int e = 0; e < 16; ++e) st.o[t][e] = n[e] > 0.0f ? st.o[t][e] + add : st.o[t][e];
    }
  }
  return m;
}

}  // namespace kvkd
