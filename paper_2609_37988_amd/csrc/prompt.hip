// Attention of whole prompts: the causal attention of a prefill (prompt_kernel) and the
// weight that each position collects over all later queries (weight_kernel), for grouped
// heads and packed or padded sequences of different lengths.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <utility>

#include "kvk_internal.h"
#include "tile_device.h"

using namespace kvkd;

namespace {

constexpr int kSeqs = KVK_MAX_BATCH_PLANS;
constexpr int64_t kMostWgs = 0xffffff;  // workgroups of 256 threads: a grid has less than 2^32 threads
constexpr float kLog2e = 1.4426950408889634f;

// The sequences of a launch, longest first, cut into blocks of rows.  The blocks with r blocks
// of their sequence left form level r; levels are launched from the largest r down, since the
// work of a block grows with r (prompt_kernel takes the r-th block of a sequence, whose rows
// see r blocks of keys; weight_kernel the one whose keys are seen by r blocks of rows).  Between
// the block counts of two neighbours in the sorted order every level has the same sequences, so
// level and sequence follow from an entry's number by one search.
struct SeqList {
  int32_t n;                // sequences with rows
  int32_t len[kSeqs];
  int32_t first[kSeqs];     // rows of the sequences before it
  int32_t begin[kSeqs];     // entries of the levels above sequence j's highest
  uint16_t index[kSeqs];    // its place in the caller's order
};

struct Strides {
  int64_t seq, head, token;  // elements; seq = 0: packed
};

struct PromptArgs {
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;
  uint16_t* out;
  float* lse;
  Strides sq, sk, sv, so;
  int32_t Hq, Hkv, G;
  int32_t qsign;  // 1, -1, 0: the sign of the scale, put on the queries
  float c;        // |scale| log2 e (1 where the scale is 0)
  SeqList sl;
};
static_assert(sizeof(PromptArgs) <= 4096, "kernel arguments");

struct WeightArgs {
  const uint16_t* q;
  const uint16_t* k;
  const float* lse;
  float* part;    // [Hq] weights per query head and position, sequence after sequence
  float* weight;
  Strides sq, sk;
  int32_t Hq, Hkv, G;
  int32_t qsign;
  float c;
  SeqList sl;
};
static_assert(sizeof(WeightArgs) <= 4096, "kernel arguments");

// An entry of a sequence list: its sequence j (of the sorted order) and level r >= 1.
struct Entry {
  int j, r;
};
template <int ROWS>
__device__ __forceinline__ Entry find_entry(const SeqList& s, int e, int lane) {
  int at = 0;
  for (int j0 = 0; j0 < s.n; j0 += 64) {
    const int j = j0 + lane;
    const uint64_t before = __ballot(j < s.n && s.begin[j < s.n ? j : 0] <= e);
    if (before) at = j0 + 63 - __clzll(before);
  }
  at = __builtin_amdgcn_readfirstlane(at);  // levels with sequences 0 .. at
  const int off = e - s.begin[at];
  return Entry{off % (at + 1), (s.len[at] + ROWS - 1) / ROWS - off / (at + 1)};
}

__device__ __forceinline__ int64_t row_base(const Strides& s, const SeqList& l, int j, int head) {
  return (s.seq ? (int64_t)l.index[j] * s.seq : (int64_t)l.first[j] * s.token) + (int64_t)head * s.head;
}

// ---------------------------------------------------------------------------
// Causal attention of whole prompts
// ---------------------------------------------------------------------------

// LDS image of a tile of kTok tokens: K rows of D bf16, padded by one 16-byte unit so that eight
// neighbouring tokens' units of one octet lie in different banks; V rows as they are, the units
// of a row exchanged by v_turn of its token.  The value operands come out of V by transposing
// reads (four tokens by sixteen channels for sixteen lanes); the exchange puts the four tokens'
// 32 bytes (and, for two such groups at a time, their 64 bytes) into different banks.
constexpr int kTok = 64;    // tokens of a tile
constexpr int kRows = 128;  // query rows of a workgroup
template <int D>
constexpr int kPitchK = 2 * D + 16;
template <int D>
constexpr int kBytesK = kTok * kPitchK<D>;
template <int D>
constexpr int kBytesV = kTok * 2 * D;
template <int D>
__device__ __forceinline__ int v_turn(int token) {
  const int r = token & 3;
  return D == 128 ? 4 * r + 2 * ((r & 1) ^ (r >> 1)) : 2 * r;
}

// A thread's share of a tile: 16-byte pieces of K and V rows.
template <int D>
struct Stage {
  static constexpr int kOct = D / 8, kStep = 256 / kOct;  // tokens between a thread's pieces
  static constexpr int kPieces = kTok / kStep;
  u4v k[kPieces], v[kPieces];

  // kp, vp: the row of the thread's first token in tile 0, at its octet; first: the tile's first
  // token; last: the sequence's last token (later ones read it).
  __device__ __forceinline__ void load(const uint16_t* kp, const uint16_t* vp, int64_t ks, int64_t vs, int first,
                                       int last, int r) {
    if (first + kTok - 1 <= last) {
      const uint16_t *ka = kp + (int64_t)first * ks, *va = vp + (int64_t)first * vs;
#pragma unroll
      for (int n = 0; n < kPieces; ++n) {
        k[n] = *reinterpret_cast<const u4v*>(ka + kStep * n * ks);
        v[n] = *reinterpret_cast<const u4v*>(va + kStep * n * vs);
      }
    } else {
#pragma unroll
      for (int n = 0; n < kPieces; ++n) {
        const int t = min(first + r + kStep * n, last) - r;
        k[n] = *reinterpret_cast<const u4v*>(kp + (int64_t)t * ks);
        v[n] = *reinterpret_cast<const u4v*>(vp + (int64_t)t * vs);
        if (first + r + kStep * n > last) v[n] = u4v{0, 0, 0, 0};  // no value past the sequence may enter a product
      }
    }
  }

  // Whether a value is infinite or NaN (its tile then needs the careful product).
  __device__ __forceinline__ bool nonfinite() const {
    bool bad = false;
#pragma unroll
    for (int n = 0; n < kPieces; ++n) bad |= any_nonfinite<false>(v[n]);
    return bad;
  }

  __device__ __forceinline__ void store(uint8_t* kimg, uint8_t* vimg, int o, int r) const {
#pragma unroll
    for (int n = 0; n < kPieces; ++n) {
      const int t = r + kStep * n;
      *reinterpret_cast<u4v*>(kimg + t * kPitchK<D> + 16 * o) = k[n];
      *reinterpret_cast<u4v*>(vimg + t * 2 * D + 16 * (o ^ v_turn<D>(t))) = v[n];
    }
  }
};

// One workgroup: 128 query rows of one head (four waves of 32) against the keys up to its last
// row, in tiles of kTok tokens, double-buffered in LDS and loaded one tile ahead through
// registers.  A wave works in steps of 32 tokens, each in two phases:
//   V(s)  softmax of the scores of step s: vector instructions
//   M(s)  O^T += V^T P^T of step s with the reads of the next keys between its products, then
//         S^T = K Q^T of step s + 1 with the reads of the next values: matrix instructions,
//         whose issue leaves the time that the reads take (24 reads in a row take 400 clocks)
// so that one wave's matrix instructions run beside the softmax of the other wave of its SIMD,
// which belongs to another workgroup (two share a CU).
// Tile t is read in M(2 t - 1) and M(2 t).  Tile t + 1, in the buffer of tile t - 1, goes to LDS
// after M(2 t - 1): the barrier after M(2 t - 2) lies behind the last reads of t - 1, the one
// after M(2 t) before the first ones of t + 1.
//
// Precision: scores, statistics and output sums are fp32; the probabilities enter the second
// product in bf16 (2^-8 relative each, of either sign), the type of the values, and the
// outputs are rounded to bf16 once.
//
// Bound: the chain of a step at two waves per SIMD.  40 / 8 heads of 128 over 8192 tokens take 724
// us (950 TFLOP/s; an 8192-wide bf16 library product reaches 1400 to 1550).  By the counters the
// matrix units are busy 43 % of that and the vector units active 43 %, hardly at the same time;
// a wave waits for issue 36 % of its time and for data 22 % (LDS bandwidth is used to 32 %), and the
// clock is 1.83 GHz.
// Measured and not kept: eight waves with the last four a phase behind (barriers between
// phases, 760 us), rows of 64 per wave at one wave per SIMD (1120: as built, with accumulator
// copies), direct loads to LDS in a ring of four steps (790), staging between the products (787).
template <int D>
__global__ __launch_bounds__(256, 2) void prompt_kernel(PromptArgs a) {
  constexpr int NM = D / 32, NK = D / 16;
  using St = Stage<D>;
  __shared__ __align__(16) uint8_t kimg[2][kBytesK<D>];
  __shared__ __align__(16) uint8_t vimg[2][kBytesV<D>];
  // One more than the last tile (of those with these low bits) whose values are not all finite:
  // tile t's is read up to V(2 t + 1), when a wave ahead may be storing tile t + 2.
  __shared__ int odd_tile[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, h = lane >> 5;
  // KV head fastest: where there are 8 KV heads (or a divisor of 8) the workgroups of one
  // share an XCD's L2
  const int hh = blockIdx.x % a.Hq;
  const int kvh = hh % a.Hkv, head = kvh * a.G + hh / a.Hkv;
  const Entry en = find_entry<kRows>(a.sl, blockIdx.x / a.Hq, lane);
  const int len = a.sl.len[en.j];
  const int q0 = (en.r - 1) * kRows;             // the block's first row
  const int last_row = min(len, q0 + kRows) - 1;
  const int w0 = q0 + 32 * wave;                 // the wave's first row
  const int row = min(w0 + col, len - 1);
  const int nt = last_row / kTok + 1;
  const int live = w0 < len ? w0 / 32 + 1 : 0;   // steps in which some row of the wave sees a token

  const int oct = tid % St::kOct, r0 = tid / St::kOct;
  const uint16_t* kp = a.k + row_base(a.sk, a.sl, en.j, kvh) + (int64_t)r0 * a.sk.token + 8 * oct;
  const uint16_t* vp = a.v + row_base(a.sv, a.sl, en.j, kvh) + (int64_t)r0 * a.sv.token + 8 * oct;
  St stg;
  const auto load = [&](int tile) { stg.load(kp, vp, a.sk.token, a.sv.token, tile * kTok, len - 1, r0); };
  const auto masked = [&](int tile) { return (tile + 1) * kTok - 1 > q0; };  // some row does not see all of it
  const auto store = [&](int tile) {
    stg.store(kimg[tile & 1], vimg[tile & 1], oct, r0);
    if (masked(tile))
      if (stg.nonfinite()) odd_tile[tile & 3] = tile + 1;
  };

  load(0);
  u4v qf[NK];
  {
    const uint16_t* qp = a.q + row_base(a.sq, a.sl, en.j, head) + (int64_t)row * a.sq.token + 8 * h;
#pragma unroll
    for (int j = 0; j < NK; ++j) qf[j] = *reinterpret_cast<const u4v*>(qp + 16 * j);
    if (a.qsign <= 0) {
#pragma unroll
      for (int j = 0; j < NK; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) qf[j][i] = a.qsign < 0 ? qf[j][i] ^ 0x80008000u : 0u;
    }
  }
  if (tid < 4) odd_tile[tid] = 0;
  RowState<NM> st;
  st.clear();
  __syncthreads();
  store(0);
  if (nt > 1) load(1);
  __syncthreads();

  // Key operand of step s, k-step j: token 32 s + col, octet 2 j + h.
  const int kat = col * kPitchK<D> + 16 * h;
  u4v kf[NK];
  const auto key_unit = [&](int s, int j) {
    return *reinterpret_cast<const u4v*>(kimg[(s >> 1) & 1] + 32 * (s & 1) * kPitchK<D> + kat + 32 * j);
  };
  // Value operand of step s, k-step x, channel tile m: channel 32 m + col, tokens
  // 16 x + 4 h + {0 .. 3, 8 .. 11} of the step.  The lane points at token 4 h + (lane / 4) % 4,
  // channels 16 (lane / 16 % 2) + 4 (lane % 4) of a transposing read.
  const int vtok = 4 * h + ((lane >> 2) & 3), vunit = 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1);
  int vat[NM];
#pragma unroll
  for (int m = 0; m < NM; ++m) vat[m] = vtok * 2 * D + 16 * ((4 * m + vunit) ^ v_turn<D>(vtok)) + 8 * (lane & 1);
  const auto value_unit = [&](int s, int x, int m) {
    const uint8_t* p = vimg[(s >> 1) & 1] + vat[m] + (32 * (s & 1) + 16 * x) * 2 * D;
    const u2v lo = read_transposed(p), hi = read_transposed(p + 8 * 2 * D);
    return u4v{lo[0], lo[1], hi[0], hi[1]};
  };

  f16v sc = zero16();
  u4v vf[2][NM];
  if (live > 0) {
#pragma unroll
    for (int j = 0; j < NK; ++j) kf[j] = key_unit(0, j);
#pragma unroll
    for (int j = 0; j < NK; ++j) sc = mfma32<false>(kf[j], qf[j], sc);
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int m = 0; m < NM; ++m) vf[x][m] = value_unit(0, x, m);
  }
  if (nt > 1) store(1);
  if (nt > 2) load(2);
  __syncthreads();
  for (int s = 0; s < 2 * nt; ++s) {
    u4v p[2];
    // V(s)
    if (s < live) {
      if (32 * s + 31 > w0) {
        asm volatile("");
#pragma unroll
        for (int k = 0; k < 16; ++k) sc[k] = 32 * s + tile_row(k, h) <= w0 + col ? sc[k] : -INFINITY;
      }
      if (masked(s >> 1) && odd_tile[(s >> 1) & 3] == (s >> 1) + 1) {
        asm volatile("");
        take_nonfinite<NM, false>(
            st, st.m, sc, a.c, 0.0f, [&](int x, int m) { return vf[x][m]; },
            [&](int k) { return (uint32_t)((row - 32 * s - tile_row(k, h)) >> 31); });
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int m = 0; m < NM; ++m) vf[x][m] = only_finite<false>(vf[x][m]);
      }
      softmax_step<NM, false>(st, sc, a.c, 0.0f, p);
      __builtin_amdgcn_sched_barrier(0);
      // M(s)
      const int sn = min(s + 1, 2 * nt - 1);  // (past the last step: the last one's operands again, not used)
#pragma unroll
      for (int i = 0; i < 2 * NM; ++i) {
        st.o[i % NM] = mfma32<false>(vf[i / NM][i % NM], p[i / NM], st.o[i % NM]);
#pragma unroll
        for (int j = i * NK / (2 * NM); j < (i + 1) * NK / (2 * NM); ++j) kf[j] = key_unit(sn, j);
        __builtin_amdgcn_sched_barrier(0);
      }
      sc = zero16();
#pragma unroll
      for (int j = 0; j < NK; ++j) {
        sc = mfma32<false>(kf[j], qf[j], sc);
#pragma unroll
        for (int i = j * 2 * NM / NK; i < (j + 1) * 2 * NM / NK; ++i) vf[i / NM][i % NM] = value_unit(sn, i / NM, i % NM);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    const int t = (s + 1) >> 1;   // odd s = 2 t - 1: tile t + 1 to LDS; even s = 2 t: tile t + 2 from memory
    if (s & 1) {
      if (t + 1 < nt) store(t + 1);
    } else {
      if (t > 0 && t + 2 < nt) load(t + 2);
      __syncthreads();
    }
  }

  if (w0 + col >= len) return;
  const float l = halves_sum(st.l);
  const float inv = 1.0f / l;
  uint16_t* op = a.out + row_base(a.so, a.sl, en.j, head) + (int64_t)row * a.so.token + 4 * h;
#pragma unroll
  for (int m = 0; m < NM; ++m)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      u2v w = {pack2<false>(st.o[m][4 * g] * inv, st.o[m][4 * g + 1] * inv),
               pack2<false>(st.o[m][4 * g + 2] * inv, st.o[m][4 * g + 3] * inv)};
      *reinterpret_cast<u2v*>(op + 32 * m + 8 * g) = w;
    }
  if (a.lse && h == 0) {
    // a sequence's log-sum-exps: [Hq][len], after those of the sequences before it
    a.lse[(int64_t)a.sl.first[en.j] * a.Hq + (int64_t)head * len + row] = (st.m + __log2f(l)) * kLn2;
  }
}

// ---------------------------------------------------------------------------
// The weight each position collects over the queries
// ---------------------------------------------------------------------------

constexpr int kKeys = 256;  // keys of a workgroup of eight waves: 32 per wave, in registers
constexpr int kWq = 128;    // query rows of a staged tile

// One workgroup: 256 keys against the later query rows of one query head,
//   part[t] = sum_{i >= t} exp(scale q_i . k_t - lse_i).
// S^T tiles with the keys as product rows: a lane adds its columns' probabilities up, and the
// lanes of a key meet once at the end.
// Bound: the vector units, 24 clocks per wave-wide probability (a product, an exponential of 16
// clocks, a sum) beside 16 of the matrix unit: 40 / 8 heads over 8192 tokens 356 us.  The counters
// show 7.1e5 clocks (1.91 GHz), of which the 24 add up to 4.9e5; vector units active 63 %, matrix
// units busy 47 %.  Four waves share a SIMD, so that one's products run beside another's
// exponentials (64 keys per wave and two waves, half the query reads: 371); the 128 registers that
// this leaves are two too few at d_h 128 (spilled).  Forming the next scores between the
// exponentials of the last ones within a wave spilled more (479 and 656), priorities of the waves
// changed nothing.
template <int D>
__global__ __launch_bounds__(512, 4) void weight_kernel(WeightArgs a) {
  constexpr int NK = D / 16, kOct = D / 8, kPieces = kWq * kOct / 512;
  __shared__ __align__(16) uint8_t qimg[2][kWq * kPitchK<D>];
  __shared__ float lse2[2][kWq];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, h = lane >> 5;
  const int hh = blockIdx.x % a.Hq;
  const int kvh = hh % a.Hkv, head = kvh * a.G + hh / a.Hkv;
  const Entry en = find_entry<kKeys>(a.sl, blockIdx.x / a.Hq, lane);
  const int len = a.sl.len[en.j];
  const int k0 = ((len + kKeys - 1) / kKeys - en.r) * kKeys;  // the block's first key
  const int kw = k0 + 32 * wave;                              // the wave's
  const uint16_t* qb = a.q + row_base(a.sq, a.sl, en.j, head);
  const float* lse = a.lse + (int64_t)a.sl.first[en.j] * a.Hq + (int64_t)head * len;

  u4v w[kPieces];
  float ls = 0.0f;
  const auto load = [&](int first) {
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int u = tid + 512 * i, r = min(first + u / kOct, len - 1);
      w[i] = *reinterpret_cast<const u4v*>(qb + (int64_t)r * a.sq.token + 8 * (u % kOct));
    }
    if (tid < kWq) {
      ls = first + tid < len ? lse[first + tid] * kLog2e : INFINITY;
      if (ls == -INFINITY) ls = INFINITY;  // rows past the end, and rows without mass, weigh nothing
    }
  };
  const auto store = [&](int buf) {
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int u = tid + 512 * i;
      *reinterpret_cast<u4v*>(qimg[buf] + (u / kOct) * kPitchK<D> + 16 * (u % kOct)) = w[i];
    }
    if (tid < kWq) lse2[buf][tid] = ls;
  };

  load(k0);
  u4v kf[NK];
  {
    const int r = min(kw + col, len - 1);
    const uint16_t* kp = a.k + row_base(a.sk, a.sl, en.j, kvh) + (int64_t)r * a.sk.token + 8 * h;
#pragma unroll
    for (int j = 0; j < NK; ++j) {
      kf[j] = *reinterpret_cast<const u4v*>(kp + 16 * j);
      if (a.qsign <= 0) {
#pragma unroll
        for (int x = 0; x < 4; ++x) kf[j][x] = a.qsign < 0 ? kf[j][x] ^ 0x80008000u : 0u;
      }
    }
  }
  f16v acc = zero16();
  store(0);
  if (k0 + kWq < len) load(k0 + kWq);
  __syncthreads();
  for (int q0 = k0, buf = 0; q0 < len; q0 += kWq, buf ^= 1) {
    if (q0 + kWq < len) store(buf ^ 1);
    if (q0 + 2 * kWq < len) load(q0 + 2 * kWq);
    if (q0 + kWq > kw && kw < len) {
#pragma unroll
      for (int y = 0; y < kWq / 32; ++y) {
        const uint8_t* qp = qimg[buf] + (32 * y + col) * kPitchK<D> + 16 * h;
        f16v s = zero16();
#pragma unroll
        for (int j = 0; j < NK; ++j) s = mfma32<false>(kf[j], *reinterpret_cast<const u4v*>(qp + 32 * j), s);
        const float l2 = lse2[buf][32 * y + col];
        const int row = q0 + 32 * y + col;
        if (q0 + 32 * y >= kw + 31) {  // every row of the subtile sees every key of the wave
#pragma unroll
          for (int e = 0; e < 16; ++e) acc[e] += __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], a.c, -l2));
        } else {
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], a.c, -l2));
            acc[e] += kw + tile_row(e, h) <= row ? p : 0.0f;  // (p of a hidden place may be NaN)
          }
        }
      }
    }
    __syncthreads();
  }
  float* out = (a.G > 1 ? a.part : a.weight) + (int64_t)a.sl.first[en.j] * a.Hq + (int64_t)head * len;
#pragma unroll
  for (int e = 0; e < 16; ++e) {  // over the 32 columns
    float x = sum16(acc[e]);
    const auto y = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(y[0]) + __uint_as_float(y[1]);
    const int t = kw + tile_row(e, h);
    if (col == 0 && t < len) out[t] = x;
  }
}

// weight[h][t] = the sum over the query heads of KV head h, in order.
__global__ __launch_bounds__(256) void weight_sum_kernel(WeightArgs a) {
  const int t = blockIdx.x * 256 + threadIdx.x, kvh = blockIdx.y, j = blockIdx.z;
  const int len = a.sl.len[j];
  if (t >= len) return;
  const float* p = a.part + (int64_t)a.sl.first[j] * a.Hq + (int64_t)kvh * a.G * len + t;
  float s = 0.0f;
  for (int g = 0; g < a.G; ++g) s += p[(int64_t)g * len];
  a.weight[(int64_t)a.sl.first[j] * a.Hkv + (int64_t)kvh * len + t] = s;
}

}  // namespace

using namespace kvk;

namespace {

// The geometry and lengths of a call: checked, and the total of the rows.
kvk_status check_seqs(const char* what, int32_t Hq, int32_t Hkv, int32_t D, int32_t n_seqs, const int32_t* seq_tokens,
                      int64_t* total) {
  if (Hkv < 1 || Hq < 1 || Hq % Hkv) return fail(KVK_ERR_INVALID, "%s: %d query heads over %d KV heads", what, Hq, Hkv);
  if (Hq > 65535) return fail(KVK_ERR_UNSUPPORTED, "%s: %d query heads (at most 65535)", what, Hq);
  if (D != 64 && D != 128) return fail(KVK_ERR_UNSUPPORTED, "%s: head_dim %d (64 or 128)", what, D);
  if (n_seqs < 1 || !seq_tokens) return fail(KVK_ERR_INVALID, "%s: no sequences", what);
  if (n_seqs > kSeqs) return fail(KVK_ERR_UNSUPPORTED, "%s: %d sequences (at most %d)", what, n_seqs, kSeqs);
  int64_t sum = 0;
  for (int j = 0; j < n_seqs; ++j) {
    if (seq_tokens[j] < 0) return fail(KVK_ERR_INVALID, "%s: sequence %d has %d tokens", what, j, seq_tokens[j]);
    sum += seq_tokens[j];
  }
  if (sum > 0x7fffff00LL) return fail(KVK_ERR_UNSUPPORTED, "%s: %lld tokens in all", what, (long long)sum);
  *total = sum;
  return KVK_OK;
}

// Element strides of a tensor: rows are read and written in 16-byte pieces.
kvk_status check_strides(const char* what, const char* name, const kvk_strides& s) {
  if (s.seq < 0 || s.head < 0 || s.token < 0 || s.seq % 8 || s.head % 8 || s.token % 8)
    return fail(KVK_ERR_INVALID, "%s: %s strides (%lld, %lld, %lld) must be multiples of 8 elements", what, name,
                (long long)s.seq, (long long)s.head, (long long)s.token);
  return KVK_OK;
}

// Rows that are written must not overlap: of the dimensions with more than one place, in the
// order of their strides, each steps over all of the ones before it.
kvk_status check_apart(const char* what, const char* name, const kvk_strides& s, int32_t D, int32_t heads, int32_t n_seqs,
                       const int32_t* seq_tokens, int64_t total) {
  const int64_t longest = *std::max_element(seq_tokens, seq_tokens + n_seqs);
  std::pair<int64_t, int64_t> dims[3] = {{s.token, s.seq ? longest : total}, {s.head, heads}, {s.seq, s.seq ? n_seqs : 1}};
  std::sort(dims, dims + 3);
  __int128 extent = D;
  for (const auto& [stride, count] : dims) {
    if (count < 2) continue;
    if (stride < extent)
      return fail(KVK_ERR_INVALID, "%s: %s rows overlap (strides %lld, %lld, %lld)", what, name, (long long)s.seq,
                  (long long)s.head, (long long)s.token);
    extent += (__int128)stride * (count - 1);
  }
  return KVK_OK;
}

// The launch order of the sequences with rows, in blocks of `rows` (see SeqList); the number
// of entries.
int64_t make_list(SeqList& sl, int32_t n_seqs, const int32_t* seq_tokens, int rows) {
  struct Seq {
    int32_t len, first, index;
  } s[kSeqs];
  int n = 0, first = 0;
  for (int j = 0; j < n_seqs; ++j) {
    if (seq_tokens[j] > 0) s[n++] = Seq{seq_tokens[j], first, j};
    first += seq_tokens[j];
  }
  std::sort(s, s + n, [](const Seq& x, const Seq& y) { return x.len != y.len ? x.len > y.len : x.index < y.index; });
  const auto blocks = [&](int j) { return j < n ? (s[j].len - 1) / rows + 1 : 0; };
  sl.n = n;
  int64_t entries = 0;
  for (int j = 0; j < n; ++j) {
    sl.len[j] = s[j].len;
    sl.first[j] = s[j].first;
    sl.index[j] = (uint16_t)s[j].index;
    sl.begin[j] = (int32_t)entries;
    entries += (int64_t)(j + 1) * (blocks(j) - blocks(j + 1));
  }
  return entries;
}

Strides strides_of(const kvk_strides& s) { return Strides{s.seq, s.head, s.token}; }

// The scale as a sign on one operand and a positive factor.
void split_scale(float scale, int32_t& sign, float& c) {
  sign = scale > 0.0f ? 1 : (scale < 0.0f ? -1 : 0);
  c = sign ? std::fabs(scale) * kLog2e : 1.0f;
}

bool misaligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) != 0; }

}  // namespace

extern "C" kvk_status kvk_prompt_attention(int32_t Hq, int32_t Hkv, int32_t D, int32_t n_seqs, const int32_t* seq_tokens,
                                           const void* q, const void* k, const void* v, const kvk_strides* strides,
                                           float scale, void* out, float* lse, hipStream_t stream) {
  const char* what = "kvk_prompt_attention";
  int64_t total = 0;
  if (kvk_status st = check_seqs(what, Hq, Hkv, D, n_seqs, seq_tokens, &total)) return st;
  if (!std::isfinite(scale)) return fail(KVK_ERR_INVALID, "%s: scale must be finite", what);
  if (total == 0) return KVK_OK;
  if (!q || !k || !v || !out) return fail(KVK_ERR_INVALID, "%s: NULL buffer", what);
  PromptArgs a;
  const kvk_strides packed[4] = {{0, D, (int64_t)Hq * D}, {0, D, (int64_t)Hkv * D}, {0, D, (int64_t)Hkv * D}, {0, D, (int64_t)Hq * D}};
  const kvk_strides* s = strides ? strides : packed;
  static const char* const names[4] = {"q", "k", "v", "out"};
  for (int i = 0; i < 4; ++i)
    if (kvk_status st = check_strides(what, names[i], s[i])) return st;
  if (kvk_status st = check_apart(what, "out", s[3], D, Hq, n_seqs, seq_tokens, total)) return st;
  if (misaligned(q, 16) || misaligned(k, 16) || misaligned(v, 16) || misaligned(out, 16) || misaligned(lse, 4))
    return fail(KVK_ERR_INVALID, "%s: misaligned buffer (q, k, v, out 16 B, lse 4 B)", what);
  if (kvk_status st = check_gpu_buffers({q, k, v, out, lse}, what)) return st;
  a.q = static_cast<const uint16_t*>(q);
  a.k = static_cast<const uint16_t*>(k);
  a.v = static_cast<const uint16_t*>(v);
  a.out = static_cast<uint16_t*>(out);
  a.lse = lse;
  a.sq = strides_of(s[0]);
  a.sk = strides_of(s[1]);
  a.sv = strides_of(s[2]);
  a.so = strides_of(s[3]);
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.G = Hq / Hkv;
  split_scale(scale, a.qsign, a.c);
  const int64_t grid = make_list(a.sl, n_seqs, seq_tokens, kRows) * Hq;
  if (grid > kMostWgs) return fail(KVK_ERR_UNSUPPORTED, "%s: grid too large", what);
  if (D == 128) hipLaunchKernelGGL(prompt_kernel<128>, dim3((unsigned)grid), dim3(256), 0, stream, a);
  else hipLaunchKernelGGL(prompt_kernel<64>, dim3((unsigned)grid), dim3(256), 0, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(KVK_ERR_DEVICE, "%s launch: %s", what, hipGetErrorString(e));
  return KVK_OK;
}

extern "C" kvk_status kvk_attention_weight_workspace_bytes(int32_t Hq, int32_t Hkv, int32_t D, int32_t n_seqs,
                                                           const int32_t* seq_tokens, size_t* out) {
  const char* what = "kvk_attention_weight_workspace_bytes";
  int64_t total = 0;
  if (kvk_status st = check_seqs(what, Hq, Hkv, D, n_seqs, seq_tokens, &total)) return st;
  if (!out) return fail(KVK_ERR_INVALID, "%s: NULL output", what);
  *out = Hq == Hkv ? 0 : (size_t)round256(total * Hq * 4);  // one head per KV head: no partial sums
  return KVK_OK;
}

extern "C" kvk_status kvk_attention_weight(int32_t Hq, int32_t Hkv, int32_t D, int32_t n_seqs, const int32_t* seq_tokens,
                                           const void* q, const void* k, const kvk_strides* strides, const float* lse,
                                           float scale, float* weight, void* workspace, size_t ws_bytes,
                                           hipStream_t stream) {
  const char* what = "kvk_attention_weight";
  int64_t total = 0;
  if (kvk_status st = check_seqs(what, Hq, Hkv, D, n_seqs, seq_tokens, &total)) return st;
  if (!std::isfinite(scale)) return fail(KVK_ERR_INVALID, "%s: scale must be finite", what);
  if (total == 0) return KVK_OK;
  size_t need = 0;
  if (kvk_status st = kvk_attention_weight_workspace_bytes(Hq, Hkv, D, n_seqs, seq_tokens, &need)) return st;
  if (!q || !k || !lse || !weight || (need && !workspace)) return fail(KVK_ERR_INVALID, "%s: NULL buffer", what);
  const kvk_strides packed[2] = {{0, D, (int64_t)Hq * D}, {0, D, (int64_t)Hkv * D}};
  const kvk_strides* s = strides ? strides : packed;
  for (int i = 0; i < 2; ++i)
    if (kvk_status st = check_strides(what, i ? "k" : "q", s[i])) return st;
  if (misaligned(q, 16) || misaligned(k, 16) || misaligned(lse, 4) || misaligned(weight, 4) ||
      (need && misaligned(workspace, 256)))
    return fail(KVK_ERR_INVALID, "%s: misaligned buffer (q, k 16 B, lse, weight 4 B, workspace 256 B)", what);
  if (need > ws_bytes) return fail(KVK_ERR_BUFFER, "%s: workspace %zu bytes < %zu needed", what, ws_bytes, need);
  if (kvk_status st = check_gpu_buffers({q, k, lse, weight, need ? workspace : nullptr}, what)) return st;
  WeightArgs a;
  a.q = static_cast<const uint16_t*>(q);
  a.k = static_cast<const uint16_t*>(k);
  a.lse = lse;
  a.part = static_cast<float*>(workspace);
  a.weight = weight;
  a.sq = strides_of(s[0]);
  a.sk = strides_of(s[1]);
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.G = Hq / Hkv;
  split_scale(scale, a.qsign, a.c);
  const int64_t grid = make_list(a.sl, n_seqs, seq_tokens, kKeys) * Hq;
  if (grid > kMostWgs / 2) return fail(KVK_ERR_UNSUPPORTED, "%s: grid too large", what);
  if (D == 128) hipLaunchKernelGGL(weight_kernel<128>, dim3((unsigned)grid), dim3(512), 0, stream, a);
  else hipLaunchKernelGGL(weight_kernel<64>, dim3((unsigned)grid), dim3(512), 0, stream, a);
  if (a.G > 1)
    hipLaunchKernelGGL(weight_sum_kernel, dim3((unsigned)((a.sl.len[0] + 255) / 256), (unsigned)Hkv, (unsigned)a.sl.n),
                       dim3(256), 0, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(KVK_ERR_DEVICE, "%s launch: %s", what, hipGetErrorString(e));
  return KVK_OK;
}
