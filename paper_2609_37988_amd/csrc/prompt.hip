// Attention of whole prompts: the causal attention of a prefill (prompt_kernel) and the
// weight that each position collects over all later queries (weight_kernel), for grouped
// heads and packed or padded sequences of different lengths.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <vector>

#include "kvk_internal.h"
#include "tile_device.h"

using namespace kvkd;

namespace {

constexpr int kSeqs = KVK_MAX_BATCH_PLANS;
constexpr float kLog2e = 1.4426950408889634f;

// The sequences of a launch, longest first, cut into blocks of rows.  The blocks with r blocks
// of their sequence left form level r; levels are launched from the largest r down, since the
// work of a block grows with r (prompt_kernel takes the r-th block of a sequence, whose rows
// see r blocks of keys; weight_kernel the one whose keys are seen by r blocks of rows).  Between
// the block counts of two neighbours in the sorted order every level has the same sequences, so
// level and sequence follow from an entry's number by one search.
struct SeqList {
  int32_t n;                // sequences with rows
  int32_t blocks0;          // blocks of the longest one
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

// LDS image of a tile of kTok<D> tokens: K rows of D bf16 padded by one 16-byte unit, and V
// transposed into units of eight tokens of one channel (the operand of one lane and k-step),
// one unit of padding after every eight channels.  Both the staging writes and the operand
// reads of eight neighbouring lanes then fall into different banks.
constexpr int kRows = 128;  // query rows of a workgroup
template <int D>
constexpr int kTok = D == 128 ? 64 : 128;  // 16 KiB of keys either way
template <int D>
constexpr int kPitchK = 2 * D + 16;
template <int D>
constexpr int kPitchV = 16 * (D + D / 8);  // one group of eight tokens
template <int D>
constexpr int kBytesK = kTok<D>* kPitchK<D>;
template <int D>
constexpr int kBytesV = kTok<D> / 8 * kPitchV<D>;

// Token n of the eight in V group g of a tile (group 2 x + h: k-step x, wave half h).
__device__ __forceinline__ constexpr int v_token(int g, int n) {
  return 16 * (g >> 1) + 8 * (n >> 2) + 4 * (g & 1) + (n & 3);
}

// A thread's share of a tile: eight 16-byte pieces.  Threads 0 .. 127 stage the keys (piece
// i: token t0 + 8 i... of one channel octet), threads 128 .. 255 the values (one octet of the
// eight tokens of one group).
template <int D>
struct Stage {
  static constexpr int kOct = D / 8;
  u4v w[8];

  // first: the tile's first token; last: the sequence's last token (later ones read it)
  __device__ __forceinline__ void load(const uint16_t* base, int64_t token_stride, int first, int last, bool values,
                                       int tid) {
    const int u = tid & 127, o = u % kOct, r = u / kOct;
    const uint16_t* p = base + (int64_t)first * token_stride;
#pragma unroll
    for (int n = 0; n < 8; ++n) {
      int t = values ? v_token(r, n) : r + (128 / kOct) * n;
      if (first + t > last) t = last - first;
      w[n] = *reinterpret_cast<const u4v*>(p + (int64_t)t * token_stride + 8 * o);
    }
  }

  // Whether a value is infinite or NaN (its tile then needs the careful product).
  __device__ __forceinline__ bool nonfinite() const {
    bool bad = false;
#pragma unroll
    for (int n = 0; n < 8; ++n) bad |= any_nonfinite<false>(w[n]);
    return bad;
  }

  __device__ __forceinline__ void store(uint8_t* kimg, uint8_t* vimg, int first, int last, bool values, int tid) {
    const int u = tid & 127, o = u % kOct, r = u / kOct;
    if (!values) {
#pragma unroll
      for (int n = 0; n < 8; ++n)
        *reinterpret_cast<u4v*>(kimg + (r + (128 / kOct) * n) * kPitchK<D> + 16 * o) = w[n];
      return;
    }
    if (first + kTok<D> - 1 > last) {  // tokens past the sequence: no value may enter a product
#pragma unroll
      for (int n = 0; n < 8; ++n)
        if (first + v_token(r, n) > last) w[n] = u4v{0, 0, 0, 0};
    }
#pragma unroll
    for (int ch = 0; ch < 8; ++ch) {
      u4v x;
#pragma unroll
      for (int p = 0; p < 4; ++p)
        x[p] = __builtin_amdgcn_perm(w[2 * p + 1][ch >> 1], w[2 * p][ch >> 1], ch & 1 ? 0x07060302u : 0x05040100u);
      *reinterpret_cast<u4v*>(vimg + r * kPitchV<D> + 16 * (9 * o + ch)) = x;
    }
  }
};

// One workgroup: 128 query rows of one head (four waves of 32) against the keys up to its
// last row, in tiles of kTok<D> tokens.
template <int D>
__global__ __launch_bounds__(256, 2) void prompt_kernel(PromptArgs a) {
  constexpr int NM = D / 32, NK = D / 16, TOK = kTok<D>, NT = TOK / 32;
  __shared__ __align__(16) uint8_t kimg[2][kBytesK<D>];
  __shared__ __align__(16) uint8_t vimg[2][kBytesV<D>];
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

  const uint16_t* kb = a.k + row_base(a.sk, a.sl, en.j, kvh);
  const uint16_t* vb = a.v + row_base(a.sv, a.sl, en.j, kvh);
  const bool values = wave >= 2;
  const uint16_t* sbase = values ? vb : kb;
  const int64_t sstride = values ? a.sv.token : a.sk.token;
  const int nt = last_row / TOK + 1;

  Stage<D> stg;
  stg.load(sbase, sstride, 0, len - 1, values, tid);
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
  RowState<NM> st;
  st.clear();
  stg.store(kimg[0], vimg[0], 0, len - 1, values, tid);
  bool bad = TOK - 1 > q0 && values && stg.nonfinite();
  if (nt > 1) stg.load(sbase, sstride, TOK, len - 1, values, tid);
  bool careful = false;
  if (TOK - 1 > q0) careful = __syncthreads_or(bad);
  else __syncthreads();

  for (int t = 0; t < nt; ++t) {
    const int t0 = t * TOK, buf = t & 1;
    const uint8_t* vp = vimg[buf] + h * kPitchV<D> + 16 * (col + (col >> 3));
    if (careful) {  // (the tile's values stay as they are until every wave has read them)
      take_nonfinite<NM, NT, false>(
          st, [&](int i, int x, int m) { return *reinterpret_cast<const u4v*>(vp + 2 * (2 * i + x) * kPitchV<D> + 16 * 36 * m); },
          [&](int i, int k) { return (uint32_t)((row - t0 - 32 * i - tile_row(k, h)) >> 31); });
      __syncthreads();
      for (int i = tid; i < kBytesV<D> / 16; i += 256) {
        u4v* p = reinterpret_cast<u4v*>(vimg[buf]) + i;
        *p = only_finite<false>(*p);
      }
      __syncthreads();
    }
    if (t + 1 < nt) {
      stg.store(kimg[buf ^ 1], vimg[buf ^ 1], t0 + TOK, len - 1, values, tid);
      bad = t0 + 2 * TOK - 1 > q0 && values && stg.nonfinite();
    }
    if (t + 2 < nt) stg.load(sbase, sstride, t0 + 2 * TOK, len - 1, values, tid);
    if (t0 <= w0 + 31 && w0 < len) {
      f16v s[NT];
#pragma unroll
      for (int i = 0; i < NT; ++i) s[i] = zero16();
      const uint8_t* kp = kimg[buf] + col * kPitchK<D> + 16 * h;
#pragma unroll
      for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int j = 0; j < NK; ++j)
          s[i] = mfma32<false>(*reinterpret_cast<const u4v*>(kp + 32 * i * kPitchK<D> + 32 * j), qf[j], s[i]);
      if (t0 + TOK - 1 > w0) {
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
          for (int k = 0; k < 16; ++k) s[i][k] = t0 + 32 * i + tile_row(k, h) <= w0 + col ? s[i][k] : -INFINITY;
      }
      u4v p[NT][2];
      softmax_step<NM, NT, false>(st, s, a.c, 0.0f, p);
#pragma unroll
      for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int m = 0; m < NM; ++m)
            st.o[m] = mfma32<false>(*reinterpret_cast<const u4v*>(vp + 2 * (2 * i + x) * kPitchV<D> + 16 * 36 * m), p[i][x], st.o[m]);
    }
    if (t0 + 2 * TOK - 1 > q0) careful = __syncthreads_or(bad);
    else __syncthreads();
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

constexpr int kKeys = 256;  // keys of a workgroup: 64 per wave, in registers
constexpr int kWq = 64;     // query rows of a staged tile

// One workgroup: 256 keys against the later query rows of one query head,
//   part[t] = sum_{i >= t} exp(scale q_i . k_t - lse_i).
// S^T tiles with the keys as product rows: a lane adds its columns' probabilities up, and the
// lanes of a key meet once at the end.
template <int D>
__global__ __launch_bounds__(256, 2) void weight_kernel(WeightArgs a) {
  constexpr int NK = D / 16, kOct = D / 8, kPieces = kWq * kOct / 256;
  __shared__ __align__(16) uint8_t qimg[2][kWq * kPitchK<D>];
  __shared__ float lse2[2][kWq];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, h = lane >> 5;
  const int hh = blockIdx.x % a.Hq;
  const int kvh = hh % a.Hkv, head = kvh * a.G + hh / a.Hkv;
  const Entry en = find_entry<kKeys>(a.sl, blockIdx.x / a.Hq, lane);
  const int len = a.sl.len[en.j];
  const int k0 = ((len + kKeys - 1) / kKeys - en.r) * kKeys;  // the block's first key
  const int kw = k0 + 64 * wave;                              // the wave's
  const uint16_t* qb = a.q + row_base(a.sq, a.sl, en.j, head);
  const float* lse = a.lse + (int64_t)a.sl.first[en.j] * a.Hq + (int64_t)head * len;

  u4v w[kPieces];
  float ls = 0.0f;
  const auto load = [&](int first) {
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int u = tid + 256 * i, r = min(first + u / kOct, len - 1);
      w[i] = *reinterpret_cast<const u4v*>(qb + (int64_t)r * a.sq.token + 8 * (u % kOct));
    }
    if (tid < kWq) ls = first + tid < len ? lse[first + tid] * kLog2e : INFINITY;  // rows past the end weigh nothing
  };
  const auto store = [&](int buf) {
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int u = tid + 256 * i;
      *reinterpret_cast<u4v*>(qimg[buf] + (u / kOct) * kPitchK<D> + 16 * (u % kOct)) = w[i];
    }
    if (tid < kWq) lse2[buf][tid] = ls;
  };

  load(k0);
  u4v kf[2][NK];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int r = min(kw + 32 * i + col, len - 1);
    const uint16_t* kp = a.k + row_base(a.sk, a.sl, en.j, kvh) + (int64_t)r * a.sk.token + 8 * h;
#pragma unroll
    for (int j = 0; j < NK; ++j) {
      kf[i][j] = *reinterpret_cast<const u4v*>(kp + 16 * j);
      if (a.qsign <= 0) {
#pragma unroll
        for (int x = 0; x < 4; ++x) kf[i][j][x] = a.qsign < 0 ? kf[i][j][x] ^ 0x80008000u : 0u;
      }
    }
  }
  f16v acc[2] = {zero16(), zero16()};
  store(0);
  if (k0 + kWq < len) load(k0 + kWq);
  __syncthreads();
  for (int q0 = k0, buf = 0; q0 < len; q0 += kWq, buf ^= 1) {
    if (q0 + kWq < len) store(buf ^ 1);
    if (q0 + 2 * kWq < len) load(q0 + 2 * kWq);
    if (q0 + kWq > kw && kw < len) {
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const uint8_t* qp = qimg[buf] + (32 * y + col) * kPitchK<D> + 16 * h;
        f16v s[2] = {zero16(), zero16()};
#pragma unroll
        for (int j = 0; j < NK; ++j) {
          const u4v qf = *reinterpret_cast<const u4v*>(qp + 32 * j);
          s[0] = mfma32<false>(kf[0][j], qf, s[0]);
          s[1] = mfma32<false>(kf[1][j], qf, s[1]);
        }
        const float l2 = lse2[buf][32 * y + col];
        const int row = q0 + 32 * y + col;
        if (q0 + 32 * y < kw + 63) {  // some row of the subtile precedes some key of the wave
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e)
              s[i][e] = kw + 32 * i + tile_row(e, h) <= row ? s[i][e] : -INFINITY;
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e) acc[i][e] += __builtin_amdgcn_exp2f(__builtin_fmaf(s[i][e], a.c, -l2));
      }
    }
    __syncthreads();
  }
  float* out = (a.G > 1 ? a.part : a.weight) + (int64_t)a.sl.first[en.j] * a.Hq + (int64_t)head * len;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) {  // over the 32 columns
      float x = sum16(acc[i][e]);
      const auto y = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
      x = __uint_as_float(y[0]) + __uint_as_float(y[1]);
      const int t = kw + 32 * i + tile_row(e, h);
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

// Element strides of a tensor of `heads` heads: rows are read and written in 16-byte pieces.
kvk_status check_strides(const char* what, const char* name, const kvk_strides& s, int32_t D, bool written) {
  if (s.seq < 0 || s.head < 0 || s.token < 0 || s.seq % 8 || s.head % 8 || s.token % 8)
    return fail(KVK_ERR_INVALID, "%s: %s strides (%lld, %lld, %lld) must be multiples of 8 elements", what, name,
                (long long)s.seq, (long long)s.head, (long long)s.token);
  if (written && (s.token < D || s.head < D))
    return fail(KVK_ERR_INVALID, "%s: %s rows overlap (head stride %lld, token stride %lld)", what, name,
                (long long)s.head, (long long)s.token);
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
  sl.blocks0 = blocks(0);
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
    if (kvk_status st = check_strides(what, names[i], s[i], D, i == 3)) return st;
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
  if (grid > 0x7fffffffLL) return fail(KVK_ERR_UNSUPPORTED, "%s: grid too large", what);
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
    if (kvk_status st = check_strides(what, i ? "k" : "q", s[i], D, false)) return st;
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
  if (grid > 0x7fffffffLL) return fail(KVK_ERR_UNSUPPORTED, "%s: grid too large", what);
  if (D == 128) hipLaunchKernelGGL(weight_kernel<128>, dim3((unsigned)grid), dim3(256), 0, stream, a);
  else hipLaunchKernelGGL(weight_kernel<64>, dim3((unsigned)grid), dim3(256), 0, stream, a);
  if (a.G > 1)
    hipLaunchKernelGGL(weight_sum_kernel, dim3((unsigned)((a.sl.len[0] + 255) / 256), (unsigned)Hkv, (unsigned)a.sl.n),
                       dim3(256), 0, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(KVK_ERR_DEVICE, "%s launch: %s", what, hipGetErrorString(e));
  return KVK_OK;
}
