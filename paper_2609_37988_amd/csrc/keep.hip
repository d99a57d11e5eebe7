// The keep list of the heaviest positions: eviction by accumulated attention weight.
//
// The want-th largest weight of a stream is found digit by digit (11, 11 and 10 bits of the
// weight as an ordered unsigned key) from histograms of the keys that share the digits found so
// far.  Keys above it are kept, and of the equal ones the first as many as are missing.  A
// workgroup holds up to 16384 keys in registers, each wave a contiguous run of positions, so
// the list comes out in order from per-wave counts.
//   keep_kernel        streams of up to 16384 competing positions: one workgroup each, one launch
//   keep_slice_kernel  longer ones, cut into slices: one launch per digit, which writes each
//                      slice's histogram, and one that writes the lists.  (One workgroup per
//                      stream that reads its keys again for every digit is bound by that CU's
//                      vector instructions: 32 streams of 131072 positions 127 us, sliced 38.)
// Bound: latency.  8 streams of 1024 positions take 6.5 us, 4 of it the launch.  The four launches
// of the long list take 7.5, 9.5, 9.5 and 12.7 us in a kernel trace (38.5 in all without one): the
// keys' loads (from the caches after the first), a histogram in LDS, and the sum of the slices'
// histograms, which every slice forms for itself.  Slices of half
// the size have twice as many of those to read (45 us), of twice the size leave CUs idle (42).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "kvk_device.h"
#include "kvk_internal.h"

using namespace kvkd;

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kBins = 2048;                    // two per thread
constexpr int kResident = 16;                  // keys a lane of keep_kernel keeps in registers
constexpr int kSliceKeys = 16;                 // ... of keep_slice_kernel (two workgroups share a CU)
constexpr int kWhole = kThreads * kResident, kSlice = kThreads * kSliceKeys;

struct KeepArgs {
  const float* weight;  // [streams][n]
  int32_t* keep;        // [streams][keep_n]
  int32_t n, keep_n;
  int32_t np;           // positions that compete: n less the recent ones
  int32_t want;         // of them kept
  // sliced streams, S streams of P slices of `slice` positions:
  int32_t S, P, slice;
  uint32_t* hist;       // [3][S][P][kBins]
  uint32_t* above;      // [2][S][P]: a slice's keys above the first and the second digit
  uint32_t* state;      // [S][2]: digits found, keys still wanted
};

// The weight as an unsigned key of the same order: NaN below everything, -0 equal to 0.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = __float_as_uint(x + 0.0f);
  const uint32_t u = b & 0x80000000u ? ~b : b | 0x80000000u;
  return x != x ? 0u : u;
}

// Digit d of a key: where it starts, its bits, and the mask of the digits before it.
__device__ __forceinline__ constexpr int digit_shift(int d) { return d == 0 ? 21 : (d == 1 ? 10 : 0); }
__device__ __forceinline__ constexpr uint32_t digit_mask(int d) { return d == 2 ? 1023u : 2047u; }
__device__ __forceinline__ constexpr uint32_t digits_before(int d) { return d == 0 ? 0u : (d == 1 ? ~0u << 21 : ~0u << 10); }

template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t dpp_add(uint32_t x) {
  return x + (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xF, false);
}
// Inclusive prefix sum over the wave.
__device__ __forceinline__ uint32_t wave_scan(uint32_t x) {
  x = dpp_add<0x111, 0xF>(x);  // row_shr 1, 2, 4, 8: within 16 lanes
  x = dpp_add<0x112, 0xF>(x);
  x = dpp_add<0x114, 0xF>(x);
  x = dpp_add<0x118, 0xF>(x);
  x = dpp_add<0x142, 0xA>(x);  // the last lane of a row to the next row
  return dpp_add<0x143, 0xC>(x);  // ... of the first half to the second
}

struct Shared {
  uint32_t hist[kBins];
  uint32_t wave[2][kWaves];
  uint32_t found[4];
};

// The sum of x over the waves before the caller's and over all waves (x uniform in a wave).
struct Sums {
  uint32_t before, all;
};
__device__ __forceinline__ Sums over_waves(uint32_t x, uint32_t* slots, int lane, int wave) {
  if (lane == 0) slots[wave] = x;
  __syncthreads();
  const uint32_t s = wave_scan(lane < kWaves ? slots[lane] : 0u);
  const uint32_t incl = __builtin_amdgcn_readlane(s, wave), all = __builtin_amdgcn_readlane(s, kWaves - 1);
  return Sums{incl - x, all};
}

// The lane's keys of a slice of `count` positions at w: position 64 (steps wave + j) + lane, j < steps.
template <int N>
struct Keys {
  uint32_t x[N];
  int steps, p0, has;  // has: steps in which the lane has a position
  __device__ __forceinline__ void load(const float* w, int n, int lane, int wave) {
    steps = (n + kThreads - 1) / kThreads;
    p0 = 64 * steps * wave + lane;
    has = min(steps, (n - p0 + 63) >> 6);
    float f[N];
#pragma unroll
    for (int j = 0; j < N; ++j) f[j] = j < has ? w[p0 + 64 * j] : 0.0f;
#pragma unroll
    for (int j = 0; j < N; ++j) x[j] = key_of(f[j]);
  }
  // f(position, key, whether there is one), in order
  template <class F>
  __device__ __forceinline__ void each(F f) const {
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (j < steps) f(p0 + 64 * j, x[j], j < has);
  }
};

// Digit d of the keys that share the digits of `prefix`, counted into sh.hist (ends with a barrier).
template <int N>
__device__ __forceinline__ void count_digit(const Keys<N>& keys, int d, uint32_t prefix, Shared& sh, int tid, int lane) {
  sh.hist[2 * tid] = 0;
  sh.hist[2 * tid + 1] = 0;
  __syncthreads();
  const int shift = digit_shift(d);
  const uint32_t mask = digit_mask(d), high = digits_before(d);
  keys.each([&](int, uint32_t key, bool has) {
    has = has && (key & high) == prefix;
    const uint32_t bin = (key >> shift) & mask;
    const uint64_t m = __ballot(has);
    if (!m) return;
    // lanes that all fall into one bin count once (equal weights would take a turn each)
    const uint32_t b0 = __builtin_amdgcn_readlane(bin, __ffsll((unsigned long long)m) - 1);
    if (__ballot(has && bin == b0) == m) {
      if (lane == 0) atomicAdd(&sh.hist[b0], (uint32_t)__popcll(m));
    } else if (has) {
      atomicAdd(&sh.hist[bin], 1u);
    }
  });
  __syncthreads();
}

// From the counts h1, h0 of the thread's bins 2 (1023 - tid) + 1 and 2 (1023 - tid): the digit in
// which the need-th largest key lies, and how many are wanted of it (to every thread; ends with
// a barrier).
__device__ __forceinline__ void find_digit(uint32_t h1, uint32_t h0, uint32_t need, Shared& sh, int tid, int lane,
                                           int wave, uint32_t& digit, uint32_t& left) {
  const int top = kBins - 1 - 2 * tid;
  const uint32_t incl = wave_scan(h0 + h1);
  const Sums s = over_waves(__builtin_amdgcn_readlane(incl, 63), sh.wave[0], lane, wave);
  const uint32_t before = s.before + incl - h0 - h1;  // keys in higher bins
  if (before < need && before + h0 + h1 >= need) {
    const bool first = before + h1 >= need;
    sh.found[0] = first ? top : top - 1;
    sh.found[1] = need - before - (first ? 0u : h1);
  }
  __syncthreads();
  digit = sh.found[0];
  left = sh.found[1];
}

// The kept positions of the keys into `keep` (offset by pos0): those above `cut`, and the first
// `ties` equal ones.
template <int N>
__device__ __forceinline__ void write_kept(const Keys<N>& keys, uint32_t cut, uint32_t ties, int pos0, int32_t* keep,
                                           Shared& sh, int lane, int wave) {
  uint32_t na = 0, ne = 0;
  keys.each([&](int, uint32_t key, bool has) {
    na += __popcll(__ballot(has && key > cut));
    ne += __popcll(__ballot(has && key == cut));
  });
  if (lane == 0) {
    sh.wave[0][wave] = na;
    sh.wave[1][wave] = ne;
  }
  __syncthreads();
  const uint32_t sa = wave_scan(lane < kWaves ? sh.wave[0][lane] : 0u), se = wave_scan(lane < kWaves ? sh.wave[1][lane] : 0u);
  const uint32_t equal_before = __builtin_amdgcn_readlane(se, wave) - ne;
  uint32_t at = __builtin_amdgcn_readlane(sa, wave) - na + min(equal_before, ties);  // the wave's first place
  uint32_t left = ties - min(equal_before, ties);
  // bits of m below the lane's own, added to x
  const auto below = [](uint64_t m, uint32_t x) {
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, x));
  };
  keys.each([&](int p, uint32_t key, bool has) {
    bool kept = has && key > cut;
    const uint64_t e = __ballot(has && key == cut);
    if (e && left) {
      kept |= has && key == cut && below(e, 0) < left;
      left -= min(left, (uint32_t)__popcll(e));
    }
    const uint64_t m = __ballot(kept);
    if (kept) keep[below(m, at)] = pos0 + p;
    at += __popcll(m);
  });
}

__global__ __launch_bounds__(kThreads) void keep_kernel(KeepArgs a) {
  __shared__ Shared sh;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int32_t* keep = a.keep + (int64_t)blockIdx.x * a.keep_n;
  Keys<kResident> keys;
  keys.load(a.weight + (int64_t)blockIdx.x * a.n, a.np, lane, wave);
  for (int i = tid; i < a.keep_n - a.want; i += kThreads) keep[a.want + i] = a.np + i;  // the recent ones
  if (a.want == 0) return;
  uint32_t prefix = 0, need = a.want;
#pragma unroll 1
  for (int d = 0; d < 3; ++d) {
    count_digit(keys, d, prefix, sh, tid, lane);
    uint32_t digit;
    const int top = kBins - 1 - 2 * tid;
    find_digit(sh.hist[top], sh.hist[top - 1], need, sh, tid, lane, wave, digit, need);
    prefix |= digit << digit_shift(d);
    __syncthreads();
  }
  write_kept(keys, prefix, need, 0, keep, sh, lane, wave);
}

// STAGE 0, 1, 2: the slice's histogram of that digit, the digit before it fixed first from all
// slices' histograms.  STAGE 3: the last digit fixed, and the slice's part of the list written.
template <int STAGE>
__global__ __launch_bounds__(kThreads) void keep_slice_kernel(KeepArgs a) {
  __shared__ Shared sh;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int p = blockIdx.x, s = blockIdx.y, pos0 = p * a.slice, count = min(a.np - pos0, a.slice);
  int32_t* keep = a.keep + (int64_t)s * a.keep_n;
  Keys<kSliceKeys> keys;
  keys.load(a.weight + (int64_t)s * a.n + pos0, count, lane, wave);
  uint32_t prefix = 0, need = a.want, above = 0, equal = 0;  // above, equal: of the slices before
  if constexpr (STAGE > 0) {
    constexpr int d = STAGE - 1;
    if (d > 0) {
      prefix = a.state[(d - 1) * 2 * a.S + 2 * s];
      need = a.state[(d - 1) * 2 * a.S + 2 * s + 1];
    }
    // the thread's bins over all slices, over the slices before this one, and of this one
    const uint32_t* h = a.hist + ((int64_t)d * a.S + s) * a.P * kBins + (kBins - 2 - 2 * tid);
    uint2 all = make_uint2(0, 0), before = all, mine = all;
    for (int i0 = 0; i0 < a.P; i0 += 8) {  // eight loads in flight
      uint2 x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = *reinterpret_cast<const uint2*>(h + (int64_t)min(i0 + i, a.P - 1) * kBins);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (i0 + i >= a.P) break;
        if (i0 + i == p) {
          before = all;
          mine = x[i];
        }
        all.x += x[i].x;
        all.y += x[i].y;
      }
    }
    uint32_t digit;
    find_digit(all.y, all.x, need, sh, tid, lane, wave, digit, need);
    prefix |= digit << digit_shift(d);
    // keys above the digit: of this slice (first digits), of the slices before (last digit)
    const uint2 part = STAGE < 3 ? mine : before;
    const uint32_t b0 = kBins - 2 - 2 * tid;
    uint32_t x = (b0 > digit ? part.x : 0u) + (b0 + 1 > digit ? part.y : 0u);
    if (STAGE == 3 && (b0 == digit || b0 + 1 == digit)) sh.found[2] = b0 == digit ? before.x : before.y;
    x = __builtin_amdgcn_readlane(wave_scan(x), 63);
    above = over_waves(x, sh.wave[1], lane, wave).all;
    if (STAGE < 3 && tid == 0) {
      a.above[((STAGE - 1) * a.S + s) * a.P + p] = above;
      if (p == 0) {
        a.state[d * 2 * a.S + 2 * s] = prefix;
        a.state[d * 2 * a.S + 2 * s + 1] = need;
      }
    }
    if constexpr (STAGE == 3) equal = sh.found[2];
    __syncthreads();
  }
  if constexpr (STAGE < 3) {
    count_digit(keys, STAGE, prefix, sh, tid, lane);
    uint2* out = reinterpret_cast<uint2*>(a.hist + (((int64_t)STAGE * a.S + s) * a.P + p) * kBins);
    out[tid] = make_uint2(sh.hist[2 * tid], sh.hist[2 * tid + 1]);
  } else {
    uint32_t sum = 0;
    for (int i = lane; i < p; i += 64) sum += a.above[s * a.P + i] + a.above[(a.S + s) * a.P + i];
    above += __builtin_amdgcn_readlane(wave_scan(sum), 63);
    const uint32_t ties = need - min(equal, need);
    write_kept(keys, prefix, ties, pos0, keep + above + min(equal, need), sh, lane, wave);
    if (p == 0)
      for (int i = tid; i < a.keep_n - a.want; i += kThreads) keep[a.want + i] = a.np + i;  // the recent ones
  }
}

// Slices of a stream of n positions, and the workspace's parts (bytes).
struct Sizes {
  int32_t P;
  int64_t hist, above, state;
};
Sizes sizes_of(int64_t streams, int32_t n) {
  Sizes z;
  z.P = (n + kSlice - 1) / kSlice;
  z.hist = kvk::round256(3 * streams * z.P * kBins * 4);
  z.above = kvk::round256(2 * streams * z.P * 4);
  z.state = kvk::round256(4 * streams * 4);
  return z;
}

}  // namespace

using namespace kvk;

static kvk_status keep_check(const kvk_table* t, int32_t n_tokens, const char* what, int64_t* streams) {
  if (!t) return fail(KVK_ERR_INVALID, "%s: NULL table", what);
  const kvk_dims& d = t->d;
  if (d.keep_tokens < 1) return fail(KVK_ERR_INVALID, "%s: the table does not evict", what);
  if (n_tokens < d.keep_tokens || n_tokens > d.max_tokens)
    return fail(KVK_ERR_INVALID, "%s: n_tokens %d outside keep_tokens..max_tokens (%d..%d)", what, n_tokens,
                d.keep_tokens, d.max_tokens);
  *streams = d.kind == KVK_MLA ? d.batch : (int64_t)d.batch * d.n_kv_heads;
  return KVK_OK;
}

extern "C" kvk_status kvk_keep_workspace_bytes(const kvk_table* t, int32_t n_tokens, size_t* out) {
  int64_t streams = 0;
  if (kvk_status st = keep_check(t, n_tokens, "kvk_keep_workspace_bytes", &streams)) return st;
  if (!out) return fail(KVK_ERR_INVALID, "kvk_keep_workspace_bytes: NULL output");
  const Sizes z = sizes_of(streams, n_tokens);
  *out = n_tokens <= kWhole ? 0 : (size_t)(z.hist + z.above + z.state);
  return KVK_OK;
}

extern "C" kvk_status kvk_keep_heaviest(const kvk_table* t, const float* weight, int32_t n_tokens, int32_t n_recent,
                                        int32_t* keep_out, void* workspace, size_t ws_bytes, hipStream_t stream) {
  const char* what = "kvk_keep_heaviest";
  int64_t streams = 0;
  if (kvk_status st = keep_check(t, n_tokens, what, &streams)) return st;
  const kvk_dims& d = t->d;
  if (n_recent < 0 || n_recent > d.keep_tokens)
    return fail(KVK_ERR_INVALID, "%s: n_recent %d outside 0..keep_tokens (%d)", what, n_recent, d.keep_tokens);
  KeepArgs a;
  a.weight = weight;
  a.keep = keep_out;
  a.n = n_tokens;
  a.keep_n = d.keep_tokens;
  a.np = n_tokens - n_recent;
  a.want = d.keep_tokens - n_recent;
  const bool sliced = a.want > 0 && a.np > kWhole;
  if (!weight || !keep_out || (sliced && !workspace)) return fail(KVK_ERR_INVALID, "%s: NULL buffer", what);
  if ((reinterpret_cast<uintptr_t>(weight) & 3) || (reinterpret_cast<uintptr_t>(keep_out) & 3) ||
      (sliced && (reinterpret_cast<uintptr_t>(workspace) & 255)))
    return fail(KVK_ERR_INVALID, "%s: misaligned buffer (weight, keep_out 4 B, workspace 256 B)", what);
  const Sizes z = sizes_of(streams, a.np);
  if (sliced && (size_t)(z.hist + z.above + z.state) > ws_bytes)
    return fail(KVK_ERR_BUFFER, "%s: workspace %zu bytes < %lld needed", what, ws_bytes,
                (long long)(z.hist + z.above + z.state));
  if (kvk_status st = check_gpu_buffers({weight, keep_out, sliced ? workspace : nullptr}, what)) return st;
  if (streams > (sliced ? 65535 : 0x3fffff)) return  // (a grid has less than 2^32 threads)
    fail(KVK_ERR_UNSUPPORTED, "%s: grid too large", what);
  if (!sliced) {
    hipLaunchKernelGGL(keep_kernel, dim3((unsigned)streams), dim3(kThreads), 0, stream, a);
  } else {
    a.S = (int32_t)streams;
    a.P = z.P;
    a.slice = ((a.np + z.P - 1) / z.P + 63) / 64 * 64;
    uint8_t* w = static_cast<uint8_t*>(workspace);
    a.hist = reinterpret_cast<uint32_t*>(w);
    a.above = reinterpret_cast<uint32_t*>(w + z.hist);
    a.state = reinterpret_cast<uint32_t*>(w + z.hist + z.above);
    const dim3 g((unsigned)z.P, (unsigned)streams), b(kThreads);
    hipLaunchKernelGGL(keep_slice_kernel<0>, g, b, 0, stream, a);
    hipLaunchKernelGGL(keep_slice_kernel<1>, g, b, 0, stream, a);
    hipLaunchKernelGGL(keep_slice_kernel<2>, g, b, 0, stream, a);
    hipLaunchKernelGGL(keep_slice_kernel<3>, g, b, 0, stream, a);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(KVK_ERR_DEVICE, "%s launch: %s", what, hipGetErrorString(e));
  return KVK_OK;
}
