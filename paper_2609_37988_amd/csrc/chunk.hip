// Attention of a chunk of new tokens over the compressed GQA caches (draft verification,
// chunked prefill, decoding of sequences of different lengths).
//
// KV-Kaizen §2.1: layers that share an anchor are served by one read of its bytes.  The query
// rows of an anchor's stream (sequence, KV head) are its new tokens x the layers that read it x
// the G query heads of the KV head, in this order, so that rows of one token sit together.
//
// One workgroup of four waves (eight for WR = 8) takes 32 WR rows and a range of the context,
// in tiles of TB 32-token blocks.  All waves dequantise a tile into LDS, once, in the operand
// order that the arena's layout has already (16-byte units of eight values), bf16 for 16-bit
// layers and fp16 for quantised ones; then wave (wr, wt) attends with row group wr to the tile's
// wt-th share of the tokens.  Many rows: WR = 4 or 8, every wave reads the whole tile.  Few rows (a
// draft, single tokens): WR = 1, the waves share the tokens, and their states meet in LDS at the
// end.  The bf16 window comes last, as one block of its own.  Where the rows alone leave the GPU
// idle the context is split over workgroups too; chunk_merge_kernel joins the partial results.
//
// Precision: in quantised layers fp16 holds a dequantised value to 2^-11 relative (bf16 would to
// 2^-8; SYMROW's blocks are scaled by a power of two each, as their bf16 scales reach further than
// fp16: see Part::lift), the queries (bf16, each row scaled by a power of two) exactly, and the
// probabilities, kept between 2^-24 and 2^15, to 2^-11; the window's probabilities enter as two
// bf16 parts, 16 bits.  In 16-bit layers keys, values and queries are exact and the probabilities
// bf16, to 2^-8: fp16 would lose small and large values.  Scores, sums and partial outputs are
// fp32, the outputs are rounded once, to bf16.
//
// Bound.  Few rows: the latency of a tile after another (8 ragged sequences up to 7000 tokens,
// one new token each, int4, 32 streams: 15 us for two tiles each, merge 7).  A draft of 40 rows per
// stream: the dequantisation beside the caches' loads (256 streams of 8192 tokens, int8: 145 us
// for 604 MB, 4.2 TB/s; vector units active 40 %, matrix units 21 %, LDS 33 %, a wave waits for
// data 37 % of its time; two tiles in flight, three workgroups per CU or tiles of four blocks for two
// row groups were slower, as built with spills).  Many rows: the chain of a step as in
// prompt_kernel, with the dequantisation before it and one workgroup per CU (2048 new of 12345
// tokens, 40 / 8 heads, int4: 558 us with its merge, 850 TFLOP/s; matrix units busy 38 %, vector
// units 45 %, a wave waits for data 39 % of its time, for issue 25 %).  SYMROW's powers of two cost
// 6 % there (int8, 583 us) and 2 % in the draft.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "kvk_internal.h"
#include "tile_device.h"

using namespace kvkd;

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kChunkSeqs = 96;  // sequences of a launch
// Largest power of two that scales a block, either way: a probability against values 2^80 apart is
// still a normal fp32 number, and counts in the sum.
constexpr int kBlockLift = 40;

struct ChunkArgs {
  const uint8_t* arena;
  const uint16_t* q;  // [nl][B][Hq][m][D]
  uint16_t* out;
  float* ws;
  int32_t n_seq;
  int32_t B, Hq, Hkv, G, m;
  int32_t layer0, geff;  // first reading layer (of the call's), query rows of a token
  int32_t block_bytes, nb_cap;
  int64_t stream_bytes;
  int32_t split_tiles;   // tiles of a split
  int32_t qsign;
  float c;
  int32_t most_lift;     // the largest power of two that a row of queries may be scaled by
  int32_t total_rows;    // rows of all streams
  int64_t region[kChunkSeqs];   // of the sequence's first stream
  int32_t stored[kChunkSeqs], fresh[kChunkSeqs];  // tokens stored, the last `fresh` of them new
  int32_t wg0[kChunkSeqs];      // workgroups, split records and rows of the sequences before it
  int32_t rec0[kChunkSeqs];
  int32_t row0[kChunkSeqs];
  uint16_t index[kChunkSeqs];   // the sequence's place in the batch
};
static_assert(sizeof(ChunkArgs) <= 4096, "kernel arguments");

// Waves over the rows, blocks of a tile, and subtiles of a wave's share of it.
template <int WR>
struct Shape {
  static constexpr int kRowsWg = 32 * WR;
  static constexpr int kWaves = WR == 8 ? 8 : 4;
  static constexpr int kWt = kWaves / WR;       // waves over the tokens
  static constexpr int kTb = WR == 1 ? 4 : 2;
  static constexpr int kBuffers = WR == 1 ? 1 : 2;  // tiles in LDS
  static constexpr int kNt = kTb / kWt;
  static constexpr int kOwn = 4 * kTb / kWaves;  // blocks of which a wave dequantises a part
};

__host__ __device__ inline int splits_of(int stored, int tb, int split_tiles) {
  const int tiles = (stored / 32 + tb - 1) / tb;
  return tiles <= split_tiles ? 1 : (tiles + split_tiles - 1) / split_tiles;
}

// The last sequence whose start is at or before x.
__device__ __forceinline__ int find_seq(const int32_t* start, int n, int x, int lane) {
  int at = 0;
  for (int j0 = 0; j0 < n; j0 += 64) {
    const int j = j0 + lane;
    const uint64_t before = __ballot(j < n && start[j < n ? j : 0] <= x);
    if (before) at = j0 + 63 - __clzll(before);
  }
  return __builtin_amdgcn_readfirstlane(at);
}

__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }  // |e| < 127

// A wave's part of a block: the keys of 16 tokens (roles 0, 1) or half the channels' values
// (roles 2, 3), D / 32 units of eight values per lane.  Raw codes as loaded ahead of use, and
// the part's scales and zeros, which go through a slot of LDS that is the wave's own.
template <int D, int BITS, int QS>
struct Part {
  static constexpr int UN = D / 32;
  static constexpr int PB = BITS == 16 ? 16 * UN : BITS * UN;  // code bytes per lane
  static constexpr int W = PB / 4;
  static constexpr int MBYTES = BITS == 16 ? 0 : (QS == kQsKivi ? 4 * D : (QS == kQsG64 ? 2 * D : 64));
  static constexpr int MW = (MBYTES + 255) / 256;  // metadata words per lane
  uint32_t w[W];
  uint32_t meta[MW > 0 ? MW : 1];

  // ONCE: no other workgroup reads the stream's bytes (plain loads else: the caches serve them)
  template <bool ONCE>
  __device__ __forceinline__ void load(const uint8_t* block, int role, int lane) {
    const uint8_t* p;
    if (role < 2) {
      p = block + role * (BITS == 16 ? 32 * D : 2 * D * BITS) + lane * (PB > 16 ? 16 : PB);
    } else {
      p = block + (BITS == 16 ? 64 * D : 4 * D * BITS);
      if constexpr (PB >= 16) p += (role - 2) * (PB / 16) * 1024 + lane * 16;
      else p += lane * 2 * PB + (role - 2) * PB;
    }
    if constexpr (PB >= 16) {
#pragma unroll
      for (int i = 0; i < PB / 16; ++i) {
        const u4v* at = reinterpret_cast<const u4v*>(p + 1024 * i);
        const u4v x = ONCE ? __builtin_nontemporal_load(at) : *at;
        w[4 * i] = x[0]; w[4 * i + 1] = x[1]; w[4 * i + 2] = x[2]; w[4 * i + 3] = x[3];
      }
    } else if constexpr (PB == 8) {
      const u2v x = *reinterpret_cast<const u2v*>(p);
      w[0] = x[0]; w[1] = x[1];
    } else {
      w[0] = *reinterpret_cast<const uint32_t*>(p);
    }
    if constexpr (BITS != 16) {
      const uint32_t* mp = reinterpret_cast<const uint32_t*>(block + 8 * D * BITS + (role < 2 ? 0 : MBYTES));
#pragma unroll
      for (int i = 0; i < MW; ++i)
        if (64 * i + lane < MBYTES / 4) meta[i] = mp[64 * i + lane];
    }
  }

  // Codes of unit u as fp16 integers, less `off`.
  __device__ __forceinline__ half8 codes(int u, float off) const {
    if constexpr (BITS == 8) return unpack8(w[2 * u], w[2 * u + 1], off);
    else if constexpr (BITS == 4) return unpack4(w[u], off);
    else return unpack2_half(w[u >> 1] >> (8 * (u & 1)), off);
  }

  // The power of two that a SYMROW block's values are stored multiplied by: it brings the largest
  // scale of the part's 32 tokens to [2^7, 2^8), so that every product with a code is in fp16's
  // range and the scales (bf16) are exact down to 2^-24 of the largest.  scales: the lane's two of
  // them so multiplied, in fp16.
  __device__ __forceinline__ int lift(int lane, uint32_t& scales) const {
    const uint32_t w = lane < 16 ? meta[0] : 0u, lo = w << 16, hi = w & 0xffff0000u;
    // (positive fp32 values order as their bits do; infinite scales do not count)
    uint32_t top = max(lo < 0x7f800000u ? lo : 0u, hi < 0x7f800000u ? hi : 0u);
    top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, kQuadXor1, 0xF, 0xF, false));
    top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, kQuadXor2, 0xF, 0xF, false));
    top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, kHalfRowMirror, 0xF, 0xF, false));
    top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, kRowMirror, 0xF, 0xF, false));
    const int ex = __builtin_amdgcn_readfirstlane((int)(top >> 23));
    const int up = ex == 0 ? 0 : max(min(127 + 7 - ex, kBlockLift), -kBlockLift);
    const float f = power_of_two(up);
    scales = bitcast<uint32_t>(h2(__uint_as_float(lo) * f, __uint_as_float(hi) * f));
    return up;
  }

  // The units' values to their places (1 KiB apart) at dst; SYMROW: times 2^up, the result.
  __device__ __forceinline__ int store(uint8_t* dst, uint32_t* slot, int role, int lane) const {
    int up = 0;
    u4v* out = reinterpret_cast<u4v*>(dst + 16 * lane);
    if constexpr (BITS == 16) {
#pragma unroll
      for (int u = 0; u < UN; ++u) out[64 * u] = u4v{w[4 * u], w[4 * u + 1], w[4 * u + 2], w[4 * u + 3]};
    } else {
      const int kg = lane >> 4, i = lane & 15;
#pragma unroll
      for (int j = 0; j < MW; ++j) {
        uint32_t word = meta[j];
        if constexpr (QS == kQsSym) up = lift(lane, word);
        if (64 * j + lane < MBYTES / 4) slot[64 * j + lane] = word;
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      const half8* h8 = reinterpret_cast<const half8*>(slot);
      const _Float16* h1 = reinterpret_cast<const _Float16*>(slot);
      if constexpr (QS == kQsSym) {
        half8 s;
        if (role < 2) {
          const _Float16 x = h1[16 * role + i];
          s = half8{x, x, x, x, x, x, x, x};
        } else {
          const u2v* h4 = reinterpret_cast<const u2v*>(slot);
          const u2v x = h4[kg], y = h4[4 + kg];
          s = bitcast<half8>(u4v{x[0], x[1], y[0], y[1]});
        }
#pragma unroll
        for (int u = 0; u < UN; ++u) out[64 * u] = bitcast<u4v>(codes(u, (float)(1 << (BITS - 1))) * s);
      } else {
#pragma unroll
        for (int u = 0; u < UN; ++u) {
          half8 s, z;
          if (role >= 2) {
            const int g = ((role - 2) * UN + u) / (QS == kQsKivi ? 2 : 4);
            s = h8[(2 * g + 0) * 4 + kg];
            z = h8[(2 * g + 1) * 4 + kg];
          } else if constexpr (QS == kQsKivi) {
            s = h8[4 * u + kg];
            z = h8[D / 8 + 4 * u + kg];
          } else {
            const int at = ((role * 4 + (i >> 2)) * (D / 64) * 2 + (u >> 1) * 2) * 4 + (i & 3);
            const _Float16 s1 = h1[at], z1 = h1[at + 4];
            s = half8{s1, s1, s1, s1, s1, s1, s1, s1};
            z = half8{z1, z1, z1, z1, z1, z1, z1, z1};
          }
          out[64 * u] = bitcast<u4v>(__builtin_elementwise_fma(codes(u, 0.0f), s, z));
        }
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
    return up;
  }
};

// A row of bf16 queries (the lane's half of it) as fp16, exactly but for values 2^29 times smaller
// than the row's largest: fp16 has bf16's digits but fewer exponents, so the row is scaled by
// the power of two that brings its largest value to 2^15 (at most 2^most), and c, the scores'
// factor, takes it back.  Rows of zeros, and with infinities or NaN, are left as they are.
template <int NK>
__device__ __forceinline__ float queries_to_half(u4v (&q)[NK], float c, int most) {
  typedef uint16_t us2 __attribute__((ext_vector_type(2)));
  us2 top = {0, 0};
#pragma unroll
  for (int j = 0; j < NK; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) top = __builtin_elementwise_max(top, bitcast<us2>(q[j][i] & 0x7fff7fffu));
  // (positive bf16 values order as their bits do, NaN above infinity)
  const float mx = halves_max(__uint_as_float((uint32_t)max(top[0], top[1]) << 16));
  const int ex = (int)(__float_as_uint(mx) >> 23);
  const int up = mx == 0.0f || ex == 255 ? 0 : min(127 + 15 - ex, most);
  const float f = power_of_two(up);
#pragma unroll
  for (int j = 0; j < NK; ++j) {
    half8 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      r[2 * i] = (_Float16)(__uint_as_float(q[j][i] << 16) * f);
      r[2 * i + 1] = (_Float16)(__uint_as_float(q[j][i] & 0xffff0000u) * f);
    }
    q[j] = bitcast<u4v>(r);
  }
  return __builtin_ldexpf(c, -up);
}

// Token of element e in half h of a 32-token subtile: the key rows of the first product are
// read in the order that gives each half, k-step by k-step, the tokens of a value unit.
__device__ __forceinline__ constexpr int subtile_token(int e, int h) {
  return 16 * ((e >> 2) & 1) + 8 * (e >> 3) + 4 * h + (e & 3);
}

// A SYMROW block's powers of two (Part::lift): 2^-up of its keys, up and 2^up of its values.
struct Lift {
  float keys, drop, grow;
};

template <int D, int BITS, int QS, int WR>
__global__ __launch_bounds__(64 * Shape<WR>::kWaves, 2) void chunk_kernel(ChunkArgs a) {
  using S = Shape<WR>;
  using P = Part<D, BITS, QS>;
  constexpr bool HALF = BITS != 16;
  constexpr int NM = D / 32, NK = D / 16, TB = S::kTb, NT = S::kNt, WT = S::kWt, OWN = S::kOwn;
  constexpr int kBlk = 128 * D;  // LDS bytes of a block: keys, then values
  constexpr int kSlot = P::MBYTES > 0 ? P::MBYTES / 4 : 1;
  constexpr int kTile = S::kBuffers * TB * kBlk, kJoin = (WT - 1) * WR * 64 * NM * 64;
  __shared__ __align__(16) uint8_t img[kTile > kJoin ? kTile : kJoin];
  __shared__ __align__(16) uint32_t slots[S::kWaves][kSlot];
  __shared__ float2 stats[4][32];
  constexpr bool SYM = BITS != 16 && QS == kQsSym;
  __shared__ Lift lifts[S::kBuffers][SYM ? TB : 1];  // of a tile's blocks
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, h = lane >> 5;
  const int wr = wave % WR, wt = wave / WR;
  const int role = wave & 3, own0 = (wave >> 2) * OWN;  // the wave's part, of blocks own0 .. of a tile

  const int sj = find_seq(a.wg0, a.n_seq, blockIdx.x, lane);
  const int stored = a.stored[sj], fresh = a.fresh[sj], seq = a.index[sj];
  const int R = a.geff * fresh, nrb = (R + S::kRowsWg - 1) / S::kRowsWg;
  const int nsplit = splits_of(stored, TB, a.split_tiles);
  int local = blockIdx.x - a.wg0[sj];
  const int kvh = local % a.Hkv;
  local /= a.Hkv;
  const int rb = nrb - 1 - local % nrb, split = local / nrb;
  const uint8_t* stream = a.arena + a.region[sj] + kvh * a.stream_bytes;

  // the lane's query row: token, then layer, then head
  const int row = rb * S::kRowsWg + 32 * wr + col, rc = min(row, R - 1);
  const int tok = rc / a.geff, rl = (rc - tok * a.geff) / a.G, g = rc - tok * a.geff - rl * a.G;
  const int64_t qrow = ((((int64_t)(a.layer0 + rl) * a.B + seq) * a.Hq + kvh * a.G + g) * a.m + tok) * D;
  const int limit = stored - fresh + tok;  // the last position the row sees
  const int seen_by_all = stored - fresh + (rb * S::kRowsWg) / a.geff;  // ... and the block's first row
  const int last_row = min(R, (rb + 1) * S::kRowsWg) - 1;
  const int seen_by_any = stored - fresh + last_row / a.geff;

  const int nbf = stored / 32;
  const int tile0 = split * a.split_tiles;
  const int tiles = min((nbf + TB - 1) / TB, tile0 + a.split_tiles);          // one past the split's last
  const int tile1 = min(tiles, seen_by_any / (32 * TB) + 1);                  // one past the last one seen
  const bool tail = split == nsplit - 1 && stored % 32 && 32 * nbf <= seen_by_any;

  P part[OWN];
  const auto load = [&](int tile) {
#pragma unroll
    for (int i = 0; i < OWN; ++i)
      part[i].template load<(WR < 4)>(stream + (int64_t)min(tile * TB + own0 + i, nbf - 1) * a.block_bytes, role, lane);
  };
  uint8_t* buf = img;  // the tile in work
  const auto place = [&](int blk) { return buf + blk * kBlk + (role < 2 ? role * 32 * D : 64 * D + (role - 2) * 1024 * P::UN); };
  if (tile0 < tile1) load(tile0);

  const auto load_queries = [&](u4v (&x)[NK]) {
#pragma unroll
    for (int j = 0; j < NK; ++j) {
      x[j] = *reinterpret_cast<const u4v*>(a.q + qrow + 16 * j + 8 * h);
      if (a.qsign <= 0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[j][i] = a.qsign < 0 ? x[j][i] ^ 0x80008000u : 0u;
      }
    }
  };
  u4v qf[NK];
  load_queries(qf);
  float c = a.c;
  if constexpr (HALF) c = queries_to_half(qf, a.c, a.most_lift);
  RowState<NM> st;
  st.clear();
  constexpr float kBias = HALF ? 7.0f : 0.0f;  // 2^(kBias + kSlack) is the largest probability

  // Key operand: product row col reads the token that puts the values in place (see above).
  const int ktok = 16 * ((col >> 3) & 1) + 8 * (col >> 4) + (col & 7);
  const int kat = (ktok >> 4) * 32 * D + 16 * (16 * h + (ktok & 15));
  const int vat = 64 * D + 1024 * (col >> 4) + 16 * (16 * h + (col & 15));
  const auto key_unit = [&](int blk, int j) {  // octet 2 j + h: sub-chunk j / 2, kg = 2 (j % 2) + h
    return *reinterpret_cast<const u4v*>(buf + kat + blk * kBlk + 1024 * (j >> 1) + 512 * (j & 1));
  };
  const auto value_unit = [&](int blk, int x, int m) {  // kg = 2 x + h
    return *reinterpret_cast<const u4v*>(buf + vat + blk * kBlk + 2048 * m + 512 * x);
  };

  // Whether a value of the blocks [k0, k1) of the tile is infinite or NaN (the wave's part of
  // them), and those values replaced by zero.
  const auto nonfinite = [&]<bool H>(std::bool_constant<H>, int k0, int k1) {
    bool bad = false;
    for (int k = k0; k < k1 && role >= 2; ++k) {
      const u4v* u = reinterpret_cast<const u4v*>(place(k) + 16 * lane);
      for (int y = 0; y < P::UN; ++y) bad |= any_nonfinite<H>(u[64 * y]);
    }
    return bad;
  };
  const auto clean = [&]<bool H>(std::bool_constant<H>, int k0, int k1) {
    for (int k = k0; k < k1 && role >= 2; ++k) {
      u4v* u = reinterpret_cast<u4v*>(place(k) + 16 * lane);
      for (int y = 0; y < P::UN; ++y) u[64 * y] = only_finite<H>(u[64 * y]);
    }
  };
  // Scores of block blk; of a masked tile -inf where the row does not see them: past token `last`
  // of the block.
  const auto scores = [&]<bool H>(std::bool_constant<H>, const u4v (&q)[NK], int blk, bool masked, int last) {
    f16v s = zero16();
#pragma unroll
    for (int j = 0; j < NK; ++j) s = mfma32<H>(key_unit(blk, j), q[j], s);
    if (masked) {
      asm volatile("");  // a branch: as selects these would cost every tile vector work
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = subtile_token(e, h) <= last ? s[e] : -INFINITY;
    }
    return s;
  };
  const auto hidden = [&](int last, int e) { return (uint32_t)((last - subtile_token(e, h)) >> 31); };
  constexpr std::bool_constant<HALF> kTileType;

  Lift* lift = lifts[0];  // of the tile in work

  for (int tile = tile0; tile < tile1; ++tile) {
    const int p0 = 32 * TB * tile, bound = 32 * nbf - 1;  // the first token's position; the last full block's
#pragma unroll
    for (int k = 0; k < OWN; ++k) {
      if (tile * TB + own0 + k < nbf) {
        const int up = part[k].store(place(own0 + k), slots[wave], role, lane);
        if (SYM && role == 0 && lane == 0) lift[own0 + k].keys = power_of_two(-up);
        if (SYM && role == 2 && lane == 0) {
          lift[own0 + k].drop = (float)up;
          lift[own0 + k].grow = power_of_two(up);
        }
      } else if (role >= 2) {  // past the full blocks: no value may enter a product
#pragma unroll
        for (int u = 0; u < P::UN; ++u) reinterpret_cast<u4v*>(place(own0 + k) + 16 * lane)[64 * u] = u4v{0, 0, 0, 0};
      }
    }
    if (tile + 1 < tile1) load(tile + 1);
    // A tile that some row does not see wholly: masked scores, and a look for infinities and NaN
    // among its values (see take_nonfinite).
    const bool masked = p0 + 32 * TB - 1 > min(seen_by_all, bound);
    const int b0 = wt * NT;  // the wave's blocks
    const int last = min(limit, bound) - p0 - 32 * b0;  // the last token of them that the row sees
    if (masked) {
      if (__syncthreads_or(nonfinite(kTileType, own0, own0 + OWN))) {
        asm volatile("");
        float m = st.m;
#pragma unroll 1
        for (int k = 0; k < NT; ++k) {
          if (p0 + 32 * (b0 + k) > min(bound, seen_by_any)) break;
          const Lift x2 = SYM ? lift[b0 + k] : Lift{1.0f, 0.0f, 1.0f};
          m = take_nonfinite<NM, HALF>(st, m, scores(kTileType, qf, b0 + k, true, last - 32 * k), c * x2.keys, kBias,
                                       [&](int x, int t) { return value_unit(b0 + k, x, t); },
                                       [&](int e) { return hidden(last - 32 * k, e); }, x2.drop);
        }
        __syncthreads();
        clean(kTileType, own0, own0 + OWN);
        __syncthreads();
      }
    } else {
      __syncthreads();
    }
#pragma unroll
    for (int k = 0; k < NT; ++k) {
      if (p0 + 32 * (b0 + k) > min(bound, seen_by_any)) break;
      const Lift x2 = SYM ? lift[b0 + k] : Lift{1.0f, 0.0f, 1.0f};
      const f16v s = scores(kTileType, qf, b0 + k, masked, last - 32 * k);
      u4v p[2];
      softmax_step<NM, HALF>(st, s, c * x2.keys, kBias, p, nullptr, x2.drop, x2.grow);
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int m = 0; m < NM; ++m) st.o[m] = mfma32<HALF>(value_unit(b0 + k, x, m), p[x], st.o[m]);
    }
    if constexpr (S::kBuffers == 1) __syncthreads();
    else {  // (its last readers are behind this tile's barrier)
      buf = buf == img ? img + TB * kBlk : img;
      lift = lift == lifts[0] ? lifts[S::kBuffers - 1] : lifts[0];
    }
  }

  // The window, one block of bf16 tokens, in bf16 products for every layer (its values are any
  // bf16; fp16 would lose the small ones).  Quantised layers keep their probabilities' precision
  // by a second product with what the rounding left.  The waves of the first share take it.
  if (tail) {
    if (own0 == 0) {
      const uint8_t* tb = stream + (int64_t)a.nb_cap * a.block_bytes;
      const u4v* in = reinterpret_cast<const u4v*>(tb + (role < 2 ? role * 32 * D : 64 * D + (role - 2) * 1024 * P::UN)) + lane;
#pragma unroll
      for (int u = 0; u < P::UN; ++u) {
        u4v x = in[64 * u];
        if (role >= 2) {  // slots past the tokens hold anything
#pragma unroll
          for (int n = 0; n < 8; ++n)
            if (16 * (n >> 2) + 4 * (lane >> 4) + (n & 3) >= stored % 32) x[n >> 1] &= n & 1 ? 0x0000ffffu : 0xffff0000u;
        }
        reinterpret_cast<u4v*>(place(0) + 16 * lane)[64 * u] = x;
      }
    }
    const int k1 = own0 == 0 ? 1 : 0, last = limit - 32 * nbf;
    const bool odd = __syncthreads_or(nonfinite(std::false_type(), 0, k1));
    f16v s;
    if (wt == 0) {
      if constexpr (HALF) load_queries(qf);
      s = scores(std::false_type(), qf, 0, true, last);
    }
    if (odd) {
      asm volatile("");
      if (wt == 0)
        take_nonfinite<NM, false>(st, st.m, s, a.c, kBias, [&](int x, int t) { return value_unit(0, x, t); },
                                  [&](int e) { return hidden(last, e); });
      __syncthreads();
      clean(std::false_type(), 0, k1);
      __syncthreads();
    }
    if (wt == 0) {
      u4v p[2], rest[2];
      softmax_step<NM, false>(st, s, a.c, kBias, p, HALF ? rest : nullptr);
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int m = 0; m < NM; ++m) {
          const u4v v = value_unit(0, x, m);
          st.o[m] = mfma32<false>(v, p[x], st.o[m]);
          if constexpr (HALF) st.o[m] = mfma32<false>(v, rest[x], st.o[m]);
        }
    }
  }
  __syncthreads();

  // The states of the waves that share rows meet in the wave with wt = 0.
  float l = halves_sum(st.l);
  if constexpr (WT > 1) {
    if (h == 0) stats[wave][col] = make_float2(st.m, l);
    __syncthreads();
    float M = -INFINITY;
    l = 0.0f;
#pragma unroll
    for (int t = 0; t < WT; ++t) M = fmaxf(M, stats[t * WR + wr][col].x);
#pragma unroll
    for (int t = 0; t < WT; ++t) {
      const float2 s = stats[t * WR + wr][col];
      l += s.x == -INFINITY ? s.y : s.y * __builtin_amdgcn_exp2f(s.x - M);  // (no mass, or NaN)
    }
    const float f = st.m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(st.m - M);
    f4* join = reinterpret_cast<f4*>(img);
    if (wt > 0) {
#pragma unroll
      for (int m = 0; m < NM; ++m)
#pragma unroll
        for (int k = 0; k < 4; ++k)
          join[(((wt - 1) * WR + wr) * NM * 4 + 4 * m + k) * 64 + lane] =
              f4{st.o[m][4 * k] * f, st.o[m][4 * k + 1] * f, st.o[m][4 * k + 2] * f, st.o[m][4 * k + 3] * f};
    }
    __syncthreads();
    if (wt > 0) return;
#pragma unroll
    for (int m = 0; m < NM; ++m) {
      st.o[m] *= f;
#pragma unroll
      for (int t = 1; t < WT; ++t)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const f4 x = join[(((t - 1) * WR + wr) * NM * 4 + 4 * m + k) * 64 + lane];
#pragma unroll
          for (int y = 0; y < 4; ++y) st.o[m][4 * k + y] += x[y];
        }
    }
    st.m = M;
  }
  if (row >= R) return;
  if (nsplit == 1) {
    const float inv = 1.0f / l;
    uint16_t* op = a.out + qrow + 4 * h;
#pragma unroll
    for (int m = 0; m < NM; ++m)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        u2v w = {pack2<false>(st.o[m][4 * k] * inv, st.o[m][4 * k + 1] * inv),
                 pack2<false>(st.o[m][4 * k + 2] * inv, st.o[m][4 * k + 3] * inv)};
        *reinterpret_cast<u2v*>(op + 32 * m + 8 * k) = w;
      }
    return;
  }
  float* rec = a.ws + (a.rec0[sj] + (int64_t)(kvh * nsplit + split) * R + row) * (D + 4);
#pragma unroll
  for (int m = 0; m < NM; ++m)
#pragma unroll
    for (int k = 0; k < 4; ++k)
      *reinterpret_cast<f4*>(rec + 32 * m + 8 * k + 4 * h) =
          f4{st.o[m][4 * k], st.o[m][4 * k + 1], st.o[m][4 * k + 2], st.o[m][4 * k + 3]};
  if (h == 0) *reinterpret_cast<float2*>(rec + D) = make_float2(st.m, l);
}

// The splits of every row joined, half a wave per row, D / 32 channels a lane, eight records at a
// time (two, where no more are left: a record read twice costs like another) with a running
// maximum.  Bound: latency where rows are few (224 rows of up to 28 splits 7 us, most of it the
// launch), else the records' bytes (81920 rows of two: 86 MB, 30 us).
template <int D>
__global__ __launch_bounds__(256) void chunk_merge_kernel(ChunkArgs a, int tb) {
  constexpr int V = D / 32;
  typedef float fv __attribute__((ext_vector_type(V)));
  const int lane = threadIdx.x & 63, l32 = lane & 31;
  const int r0 = __builtin_amdgcn_readfirstlane(2 * (blockIdx.x * 4 + (threadIdx.x >> 6)));
  if (r0 >= a.total_rows) return;
  const int r1 = min(r0 + 1, a.total_rows - 1);
  const int s0j = find_seq(a.row0, a.n_seq, r0, lane), s1j = find_seq(a.row0, a.n_seq, r1, lane);
  const int r = lane < 32 ? r0 : r1, sj = lane < 32 ? s0j : s1j;
  const int nsplit = splits_of(a.stored[sj], tb, a.split_tiles);
  const bool live = nsplit > 1 && r0 + (lane >> 5) < a.total_rows;  // (one split: written by its workgroup)
  const int n = live ? nsplit : 0;
  const int R = a.geff * a.fresh[sj], x = r - a.row0[sj], kvh = x / R, row = x - kvh * R;
  const float* rec = a.ws + (a.rec0[sj] + (int64_t)kvh * nsplit * R + row) * (D + 4);
  const int64_t step = (int64_t)R * (D + 4);
  float M = -INFINITY, l = 0.0f;
  fv o;
#pragma unroll
  for (int k = 0; k < V; ++k) o[k] = 0.0f;
  const auto take = [&]<int N>(std::integral_constant<int, N>, int i0) {  // records i0 .. i0 + N - 1
    fv v[N];
    float2 ml[N];
    float m = M;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float* p = rec + min(i0 + i, n - 1) * step;
      v[i] = *reinterpret_cast<const fv*>(p + V * l32);
      ml[i] = *reinterpret_cast<const float2*>(p + D);
      m = fmaxf(m, ml[i].x);
    }
    const float f = M == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(M - m);
    M = m;
    l *= f;
    o *= f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (i0 + i < n) {
        const float w = ml[i].x == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(ml[i].x - M);  // (no mass, or NaN)
        l += ml[i].y * w;
        o += v[i] * w;
      }
    }
  };
  int i0 = 0;
  for (; n - i0 > 2; i0 += 8) take(std::integral_constant<int, 8>(), i0);
  if (i0 < n) take(std::integral_constant<int, 2>(), i0);
  if (!live) return;
  const float inv = 1.0f / l;
  const int tok = row / a.geff, rl = (row - tok * a.geff) / a.G, g = row - tok * a.geff - rl * a.G;
  uint32_t* op = reinterpret_cast<uint32_t*>(
      a.out + ((((int64_t)(a.layer0 + rl) * a.B + a.index[sj]) * a.Hq + kvh * a.G + g) * a.m + tok) * D + V * l32);
#pragma unroll
  for (int k = 0; k < V / 2; ++k) op[k] = pack2<false>(o[2 * k] * inv, o[2 * k + 1] * inv);
}

}  // namespace

using namespace kvk;

namespace {

// Workgroups that a launch's splits aim at: four per CU, so that the last ones to end leave
// little idle, or the two that a CU holds at once where four would be short (a split pays its
// start, and a record per row written and read), or two of those of eight waves.  4-bit, 64
// streams of 8192 tokens, one new token: two per CU 37 us, four 42; 8-bit, 256 streams, four new
// tokens: 131 and 122.
constexpr int64_t kAimWgs = 1024;
constexpr int kLongSplit = 16;  // tiles
constexpr int kMinTiles = 2;

// Eight waves halve the dequantisation per row but leave a CU one workgroup, whose barriers
// nothing covers, and wide row blocks part empty.  4-bit, one sequence of 8192 tokens, query rows
// per KV head and times with four and eight waves: 1280 76 and 89 us, 2560 131 and 125, 5120
// 225 and 206; 12345 tokens, 10240 rows 594 and 545.
constexpr int64_t kManyRows = 2048;

int waves_over_rows(int64_t rows) { return rows <= 32 ? 1 : (rows <= 64 ? 2 : (rows < kManyRows ? 4 : 8)); }
int64_t aim_of(int wr, int64_t work) { return wr < 8 && work / kAimWgs >= kLongSplit ? kAimWgs : kAimWgs / 2; }
int blocks_of_tile(int wr) { return wr == 1 ? 4 : 2; }

// Split records of a launch at most, for up to rows_of_stream rows in each of up to `streams`
// streams.  The splits of all row blocks are at most the number aimed at and one more for each
// block, and a launch with that many row blocks does not split; a row has at most the splits
// of a full stream.
int64_t most_records(const kvk_table* t, int64_t rows_of_stream, int64_t streams) {
  int64_t most = 0;
  for (int w = waves_over_rows(rows_of_stream); w >= 1; w /= 2) {  // (fewer new tokens take narrower blocks)
    const int64_t rows = std::min<int64_t>(rows_of_stream, w < 4 ? 32 * w : (w == 4 ? kManyRows - 1 : rows_of_stream));
    const int64_t aim = w < 8 ? kAimWgs : kAimWgs / 2;  // (at most)
    const int64_t blocks = streams * ((rows + 32 * w - 1) / (32 * w));
    const int64_t tiles = (t->nb_cap + blocks_of_tile(w) - 1) / blocks_of_tile(w);
    const int64_t splits = (tiles + kMinTiles - 1) / kMinTiles;
    if (splits > 1)
      most = std::max(most, std::min((aim + std::min(blocks, aim)) * 32 * w, streams * rows * splits));
  }
  return most;
}

struct ChunkLaunch {
  ChunkArgs a;
  int bits, wr;
  int64_t wgs, recs;
};

// Fills the sequences' launch fields (lengths and regions are set); the split rule.
kvk_status lay_out(ChunkLaunch& L) {
  ChunkArgs& a = L.a;
  int64_t most = 0;
  for (int j = 0; j < a.n_seq; ++j) most = std::max<int64_t>(most, (int64_t)a.geff * a.fresh[j]);
  L.wr = waves_over_rows(most);
  const int rows = 32 * L.wr, tb = blocks_of_tile(L.wr);
  int64_t wgs = 0, work = 0;
  for (int j = 0; j < a.n_seq; ++j) {
    const int64_t n = (int64_t)a.Hkv * (((int64_t)a.geff * a.fresh[j] + rows - 1) / rows);
    wgs += n;
    work += n * ((a.stored[j] / 32 + tb - 1) / tb);
  }
  const int64_t aim = aim_of(L.wr, work);
  a.split_tiles = wgs >= aim ? 0x7fffffff : (int32_t)std::max<int64_t>(kMinTiles, (work + aim - 1) / aim);
  int64_t wg = 0, rec = 0, row = 0;
  for (int j = 0; j < a.n_seq; ++j) {
    const int64_t R = (int64_t)a.geff * a.fresh[j], nrb = (R + rows - 1) / rows;
    const int ns = splits_of(a.stored[j], tb, a.split_tiles);
    if (wg > 0x7fffffffLL || rec > 0x7fffffffLL || row > 0x7fffffffLL) break;
    a.wg0[j] = (int32_t)wg;
    a.rec0[j] = (int32_t)rec;
    a.row0[j] = (int32_t)row;
    wg += a.Hkv * nrb * ns;
    rec += ns > 1 ? a.Hkv * R * ns : 0;
    row += a.Hkv * R;
  }
  if (wg > 0xffffffLL || rec > 0x7fffffffLL || row > 0x7ffffff0LL)  // (a grid has less than 2^32 threads)
    return fail(KVK_ERR_UNSUPPORTED, "kvk_chunk_attention: too many query rows in one call");
  L.wgs = wg;
  L.recs = rec;
  a.total_rows = (int32_t)row;
  return KVK_OK;
}

template <int D, int BITS, int QS>
void launch_rows(const ChunkLaunch& L, hipStream_t st) {
  const dim3 g((unsigned)L.wgs), b(256);
  if (L.wr == 1) hipLaunchKernelGGL((chunk_kernel<D, BITS, QS, 1>), g, b, 0, st, L.a);
  else if (L.wr == 2) hipLaunchKernelGGL((chunk_kernel<D, BITS, QS, 2>), g, b, 0, st, L.a);
  else if (L.wr == 4) hipLaunchKernelGGL((chunk_kernel<D, BITS, QS, 4>), g, b, 0, st, L.a);
  else hipLaunchKernelGGL((chunk_kernel<D, BITS, QS, 8>), g, dim3(512), 0, st, L.a);
}
template <int D, int QS>
void launch_bits(const ChunkLaunch& L, hipStream_t st) {
  if (L.bits == 16) launch_rows<D, 16, kQsKivi>(L, st);
  else if (L.bits == 8) launch_rows<D, 8, QS>(L, st);
  else if (L.bits == 4) launch_rows<D, 4, QS>(L, st);
  else launch_rows<D, 2, QS>(L, st);
}
template <int D>
kvk_status launch(const ChunkLaunch& L, int qs, hipStream_t st) {
  if (qs == KVK_Q_KIVI32) launch_bits<D, kQsKivi>(L, st);
  else if (qs == KVK_Q_GROUP64) launch_bits<D, kQsG64>(L, st);
  else launch_bits<D, kQsSym>(L, st);
  if (L.recs > 0)
    hipLaunchKernelGGL(chunk_merge_kernel<D>, dim3((unsigned)((L.a.total_rows + 7) / 8)), dim3(256), 0, st, L.a,
                       blocks_of_tile(L.wr));
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(KVK_ERR_DEVICE, "kvk_chunk_attention launch: %s", hipGetErrorString(e));
  return KVK_OK;
}

kvk_status check_range(const kvk_table* t, const char* what, int32_t l0, int32_t l1, int32_t n_chunk) {
  if (!t) return fail(KVK_ERR_INVALID, "%s: NULL table", what);
  if (t->d.kind != KVK_GQA) return fail(KVK_ERR_UNSUPPORTED, "%s: GQA tables (MLA: token by token)", what);
  if (l0 < 0 || l1 > t->d.n_layers || l0 >= l1)
    return fail(KVK_ERR_INVALID, "layer range [%d, %d) invalid for %d layers", l0, l1, t->d.n_layers);
  if (n_chunk < 1 || n_chunk > t->cap)
    return fail(KVK_ERR_INVALID, "%s: n_chunk %d outside 1..%d", what, n_chunk, t->cap);
  return KVK_OK;
}

}  // namespace

extern "C" kvk_status kvk_chunk_workspace_bytes(const kvk_table* t, int32_t l0, int32_t l1, int32_t n_chunk, size_t* out) {
  if (kvk_status st = check_range(t, "kvk_chunk_workspace_bytes", l0, l1, n_chunk)) return st;
  if (!out) return fail(KVK_ERR_INVALID, "kvk_chunk_workspace_bytes: NULL output");
  const kvk_dims& d = t->d;
  const int64_t G = d.n_q_heads / d.n_kv_heads;
  // launches run one after another and share the workspace
  const int64_t recs = most_records(t, G * (l1 - l0) * n_chunk, std::min<int64_t>(d.batch, kChunkSeqs) * d.n_kv_heads);
  *out = (size_t)round256(std::max<int64_t>(recs * (d.head_dim + 4) * 4, 256));
  return KVK_OK;
}

extern "C" kvk_status kvk_chunk_attention(const kvk_table* t, int32_t l0, int32_t l1, const void* q, int32_t n_chunk,
                                          const int32_t* n_stored, const int32_t* n_new, float scale,
                                          const void* arena, void* out, void* workspace, size_t ws_bytes,
                                          hipStream_t stream) {
  const char* what = "kvk_chunk_attention";
  if (kvk_status st = check_range(t, what, l0, l1, n_chunk)) return st;
  const kvk_dims& d = t->d;
  if (!q || !n_stored || !arena || !out || !workspace) return fail(KVK_ERR_INVALID, "%s: NULL buffer", what);
  if (!std::isfinite(scale)) return fail(KVK_ERR_INVALID, "%s: scale must be finite", what);
  if (d.batch > 65535) return fail(KVK_ERR_UNSUPPORTED, "%s: %d sequences (at most 65535)", what, d.batch);
  bool any = false;
  for (int b = 0; b < d.batch; ++b) {
    const int32_t m = n_new ? n_new[b] : n_chunk;
    if (n_stored[b] < 0 || n_stored[b] > t->cap)
      return fail(KVK_ERR_INVALID, "%s: n_stored[%d] = %d outside 0..%d", what, b, n_stored[b], t->cap);
    if (m < 0 || m > n_chunk || m > n_stored[b])
      return fail(KVK_ERR_INVALID, "%s: n_new[%d] = %d outside 0..min(n_chunk %d, n_stored %d)", what, b, m, n_chunk,
                  n_stored[b]);
    any |= m > 0;
  }
  if ((reinterpret_cast<uintptr_t>(q) & 15) || (reinterpret_cast<uintptr_t>(arena) & 15) ||
      (reinterpret_cast<uintptr_t>(out) & 15) || (reinterpret_cast<uintptr_t>(workspace) & 255))
    return fail(KVK_ERR_INVALID, "%s: misaligned buffer (q, arena, out 16 B, workspace 256 B)", what);
  if (!any) return KVK_OK;
  if (kvk_status st = check_gpu_buffers({q, arena, out, workspace}, what)) return st;

  const bool per_seq = !t->seq.empty();
  const int32_t G = d.n_q_heads / d.n_kv_heads;
  ChunkLaunch L;
  ChunkArgs& a = L.a;
  a.arena = static_cast<const uint8_t*>(arena);
  a.q = static_cast<const uint16_t*>(q);
  a.out = static_cast<uint16_t*>(out);
  a.ws = static_cast<float*>(workspace);
  a.B = d.batch;
  a.Hq = d.n_q_heads;
  a.Hkv = d.n_kv_heads;
  a.G = G;
  a.m = n_chunk;
  a.nb_cap = t->nb_cap;
  a.qsign = scale > 0.0f ? 1 : (scale < 0.0f ? -1 : 0);
  a.c = a.qsign ? std::fabs(scale) * kLog2e : 1.0f;
  // c / 2^(most_lift + kBlockLift) stays a normal number; queries so small that this binds give
  // logits that do not count.  (c itself may have overflowed)
  a.most_lift = std::isinf(a.c) ? 120 : std::min(120, std::ilogb(a.c) + 60);
  // One launch for the sequences that read the same layers from an anchor of one bit-width (one
  // plan: all of them), in groups of kChunkSeqs.  Two passes: every launch is laid out and
  // checked before the first one is made.
  for (const bool go : {false, true}) {
    const auto flush = [&]() -> kvk_status {
      if (a.n_seq == 0) return KVK_OK;
      if (kvk_status st = lay_out(L)) return st;
      const size_t need = (size_t)L.recs * (d.head_dim + 4) * 4;
      if (need > ws_bytes) return fail(KVK_ERR_BUFFER, "%s: workspace %zu bytes < %zu needed", what, ws_bytes, need);
      if (go) {
        const kvk_status st = d.head_dim == 128 ? launch<128>(L, d.qscheme, stream) : launch<64>(L, d.qscheme, stream);
        if (st != KVK_OK) return st;
      }
      a.n_seq = 0;
      return KVK_OK;
    };
    const int n_plans = per_seq ? d.batch : 1;
    // (first, one past the last reading layer, bits) of the group that plan s opens at layer lb
    const auto opens = [&](const kvk_table* s, int lb, int& le, int& bits) {
      const int anc = s->info.anchor_of[lb];
      le = std::min(s->next_anchor[anc], l1);
      bits = s->bits[anc];
      return std::max(anc, l0) == lb;
    };
    for (int lb = l0; lb < l1; ++lb) {
      bool done[KVK_MAX_BATCH_PLANS] = {};
      for (int p = 0; p < n_plans; ++p) {
        int le, bits;
        if (done[p] || !opens(per_seq ? t->seq[p] : t, lb, le, bits)) continue;
        a.n_seq = 0;
        for (int b = p; b < d.batch; ++b) {
          const kvk_table* s = per_seq ? t->seq[b] : t;
          int le_b = le, bits_b = bits;
          if (per_seq && (!opens(s, lb, le_b, bits_b) || le_b != le || bits_b != bits)) continue;
          if (per_seq) done[b] = true;
          const int32_t m = n_new ? n_new[b] : n_chunk;
          if (m == 0) continue;
          const int anc = s->info.anchor_of[lb];
          L.bits = bits;
          a.layer0 = lb - l0;
          a.geff = G * (le - lb);
          a.block_bytes = (int32_t)s->block_bytes[anc];
          a.stream_bytes = s->info.stream_bytes[anc];
          a.region[a.n_seq] = per_seq ? t->seq_base[b] + s->info.layer_offset[anc]
                                      : s->info.layer_offset[anc] + (int64_t)b * d.n_kv_heads * s->info.stream_bytes[anc];
          a.stored[a.n_seq] = n_stored[b];
          a.fresh[a.n_seq] = m;
          a.index[a.n_seq] = (uint16_t)b;
          if (++a.n_seq == kChunkSeqs)
            if (kvk_status st = flush()) return st;
        }
        if (kvk_status st = flush()) return st;
      }
    }
  }
  return KVK_OK;
}
