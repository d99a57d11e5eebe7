// The keep list of the heaviest positions: eviction by accumulated attention weight.
#include <hip/hip_runtime.h>

#include "kvk_device.h"
#include "kvk_internal.h"

using namespace kvkd;

namespace {

struct KeepArgs {
  const float* weight;  // [streams][n]
  int32_t* keep;        // [streams][keep_n]
  int32_t n, keep_n;
  int32_t np;           // positions that compete: n less the recent ones
  int32_t want;         // of them kept
};

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kBins = 2048;    // digits of 11, 11 and 10 bits
constexpr int kResident = 16;  // keys a lane keeps in registers

// The weight as an unsigned key of the same order: NaN below everything, -0 equal to 0.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = __float_as_uint(x + 0.0f);
  const uint32_t u = b & 0x80000000u ? ~b : b | 0x80000000u;
  return x != x ? 0u : u;
}

// One workgroup per stream.  Wave w owns the positions [w seg, (w + 1) seg), so the list comes
// out in order from per-wave counts.  The want-th largest key is found digit by digit from LDS
// histograms of the keys that share the digits found so far; keys above it are kept, and of
// the equal ones the first as many as are missing.  Up to kResident keys per lane stay in
// registers; longer streams are read again in each of the five passes (from the L2).
template <bool RESIDENT>
__global__ __launch_bounds__(kThreads) void keep_kernel(KeepArgs a) {
  __shared__ uint32_t hist[kBins];
  __shared__ uint32_t above[kWaves], equal[kWaves], found[2];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const float* w = a.weight + (int64_t)blockIdx.x * a.n;
  int32_t* keep = a.keep + (int64_t)blockIdx.x * a.keep_n;
  for (int i = tid; i < a.keep_n - a.want; i += kThreads) keep[a.want + i] = a.np + i;  // the recent ones
  if (a.want == 0) return;

  const int steps = (a.np + kThreads - 1) / kThreads;  // 64-position steps of a wave
  const int p0 = wave * steps * 64 + lane;
  uint32_t x[kResident];
  if constexpr (RESIDENT) {
    float f[kResident];
#pragma unroll
    for (int j = 0; j < kResident; ++j) f[j] = j < steps && p0 + 64 * j < a.np ? w[p0 + 64 * j] : 0.0f;
#pragma unroll
    for (int j = 0; j < kResident; ++j) x[j] = key_of(f[j]);
  }
  // f(position, key, whether there is one) for each of the lane's positions, in order
  const auto each = [&](auto f) {
    if constexpr (RESIDENT) {
#pragma unroll
      for (int j = 0; j < kResident; ++j)
        if (j < steps) f(p0 + 64 * j, x[j], p0 + 64 * j < a.np);
    } else {
      for (int j0 = 0; j0 < steps; j0 += 8) {
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int p = p0 + 64 * (j0 + j);
          v[j] = w[p < a.np ? p : a.np - 1];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (j0 + j < steps) f(p0 + 64 * (j0 + j), key_of(v[j]), p0 + 64 * (j0 + j) < a.np);
      }
    }
  };

  uint32_t prefix = 0, need = a.want;  // digits found; keys still wanted among those that share them
#pragma unroll 1
  for (int d = 0; d < 3; ++d) {
    const int shift = d == 0 ? 21 : (d == 1 ? 10 : 0), bits = d == 2 ? 10 : 11;
    const uint32_t high = d == 0 ? 0u : ~0u << (shift + bits);
    for (int i = tid; i < kBins; i += kThreads) hist[i] = 0;
    __syncthreads();
    each([&](int, uint32_t key, bool has) {
      has = has && (key & high) == prefix;
      const uint32_t bin = (key >> shift) & ((1u << bits) - 1u);
      const uint64_t m = __ballot(has);
      if (!m) return;
      // lanes that all fall into one bin count once (equal weights would take a turn each)
      const uint32_t b0 = __builtin_amdgcn_readlane(bin, __ffsll((unsigned long long)m) - 1);
      if (__ballot(has && bin == b0) == m) {
        if (lane == 0) atomicAdd(&hist[b0], (uint32_t)__popcll(m));
      } else if (has) {
        atomicAdd(&hist[bin], 1u);
      }
    });
    __syncthreads();
    // from the top bin down: thread i holds bins 2 i', 2 i' + 1 with i' = 1023 - i
    const int top = kBins - 1 - 2 * tid;
    const uint32_t h1 = hist[top], h0 = hist[top - 1];
    uint32_t s = h0 + h1;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t y = __shfl_up(s, o);
      if (lane >= o) s += y;
    }
    if (lane == 63) above[wave] = s;
    __syncthreads();
    for (int i = 0; i < wave; ++i) s += above[i];
    const uint32_t before = s - h0 - h1;  // keys in higher bins
    if (before < need && s >= need) {
      const bool first = before + h1 >= need;
      found[0] = first ? top : top - 1;
      found[1] = need - before - (first ? 0 : h1);
    }
    __syncthreads();
    prefix |= found[0] << shift;
    need = found[1];
    __syncthreads();
  }

  uint32_t na = 0, ne = 0;
  each([&](int, uint32_t key, bool has) {
    na += __popcll(__ballot(has && key > prefix));
    ne += __popcll(__ballot(has && key == prefix));
  });
  if (lane == 0) {
    above[wave] = na;
    equal[wave] = ne;
  }
  __syncthreads();
  uint32_t sum_above = 0, sum_equal = 0;
  for (int i = 0; i < wave; ++i) {
    sum_above += above[i];
    sum_equal += equal[i];
  }
  uint32_t at = sum_above + min(sum_equal, need);                 // the wave's first place in the list
  uint32_t ties = need - min(sum_equal, need);                    // equal keys left to keep
  const uint64_t below = (1ull << lane) - 1;
  each([&](int p, uint32_t key, bool has) {
    const uint64_t e = __ballot(has && key == prefix);
    const bool kept = has && (key > prefix || (key == prefix && (uint32_t)__popcll(e & below) < ties));
    const uint64_t m = __ballot(kept);
    if (kept) keep[at + __popcll(m & below)] = p;
    at += __popcll(m);
    ties -= min(ties, (uint32_t)__popcll(e));
  });
}

}  // namespace

using namespace kvk;

extern "C" kvk_status kvk_keep_heaviest(const kvk_table* t, const float* weight, int32_t n_tokens, int32_t n_recent,
                                        int32_t* keep_out, hipStream_t stream) {
  if (!t) return fail(KVK_ERR_INVALID, "kvk_keep_heaviest: NULL table");
  const kvk_dims& d = t->d;
  if (d.keep_tokens < 1) return fail(KVK_ERR_INVALID, "kvk_keep_heaviest: the table does not evict");
  if (n_tokens < d.keep_tokens || n_tokens > d.max_tokens)
    return fail(KVK_ERR_INVALID, "kvk_keep_heaviest: n_tokens %d outside keep_tokens..max_tokens (%d..%d)", n_tokens,
                d.keep_tokens, d.max_tokens);
  if (n_recent < 0 || n_recent > d.keep_tokens)
    return fail(KVK_ERR_INVALID, "kvk_keep_heaviest: n_recent %d outside 0..keep_tokens (%d)", n_recent, d.keep_tokens);
  if (!weight || !keep_out) return fail(KVK_ERR_INVALID, "kvk_keep_heaviest: NULL buffer");
  if ((reinterpret_cast<uintptr_t>(weight) & 3) || (reinterpret_cast<uintptr_t>(keep_out) & 3))
    return fail(KVK_ERR_INVALID, "kvk_keep_heaviest: misaligned buffer (4 B)");
  if (kvk_status st = check_gpu_buffers({weight, keep_out}, "kvk_keep_heaviest")) return st;
  const int64_t streams = d.kind == KVK_MLA ? d.batch : (int64_t)d.batch * d.n_kv_heads;
  if (streams > 0x7fffffffLL) return fail(KVK_ERR_UNSUPPORTED, "kvk_keep_heaviest: grid too large");
  KeepArgs a;
  a.weight = weight;
  a.keep = keep_out;
  a.n = n_tokens;
  a.keep_n = d.keep_tokens;
  a.np = n_tokens - n_recent;
  a.want = d.keep_tokens - n_recent;
  if (a.np <= kThreads * kResident)
    hipLaunchKernelGGL(keep_kernel<true>, dim3((unsigned)streams), dim3(kThreads), 0, stream, a);
  else hipLaunchKernelGGL(keep_kernel<false>, dim3((unsigned)streams), dim3(kThreads), 0, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(KVK_ERR_DEVICE, "kvk_keep_heaviest launch: %s", hipGetErrorString(e));
  return KVK_OK;
}
