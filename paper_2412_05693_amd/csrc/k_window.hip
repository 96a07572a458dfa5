// Tokens through a window cache (bm_window.h): a prompt's attention, and the storing of
// its rows behind it.
#include <type_traits>

#include "bm_internal.h"
#include "bm_lanes.h"
#include "bm_window_dev.h"

namespace bm {
namespace {

constexpr float kNegInf = -__builtin_huge_valf();

__device__ __forceinline__ float as_float(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
__device__ __forceinline__ float as_float(float x) { return x; }
__device__ __forceinline__ void put(uint16_t* p, float x) { *reinterpret_cast<__bf16*>(p) = (__bf16)x; }
__device__ __forceinline__ void put(float* p, float x) { *p = x; }

// one wave a query row
template <typename E, int D>
__global__ void __launch_bounds__(256) window_prompt_kernel(PromptArgs a) {
  constexpr int P = D / 64;
  const int group = a.n_heads / a.n_kv_heads;
  const int64_t wave = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (wave >= (int64_t)a.units * group * a.n_tok) return;
  const int t = (int)(wave % a.n_tok);
  const int64_t head = wave / a.n_tok;                 // sample * n_heads + query head
  const int bi = (int)(head / a.n_heads), u = (int)(head / group);
  const int pad = a.pad ? max(0, a.pad[bi]) : 0;
  const int r0 = a.t0 - pad, i = r0 + t;
  const E* q = static_cast<const E*>(a.q) + (head * a.seq_ld + t) * D;
  E* o = static_cast<E*>(a.o) + (head * a.seq_ld + t) * D;
  float x[P], acc[P], m = kNegInf, l = 0.0f;
#pragma unroll
  for (int e = 0; e < P; ++e) {
    x[e] = as_float(q[lane * P + e]) * a.scale_log2;
    acc[e] = 0.0f;
  }
  const int lo = max(0, i - a.window + 1), lead = min(a.sinks, lo);
  for (int c = 0; c < lead + (i + 1 - lo) && i >= 0; ++c) {
    const int j = c < lead ? c : lo + c - lead;
    const bool old = j < r0;
    const int64_t row = old ? (int64_t)u * (a.window + a.sinks) + window_slot(j, a.sinks, a.window)
                            : (int64_t)u * a.seq_ld + (j - r0);
    const E* k = static_cast<const E*>(old ? a.kc : a.kin) + row * D;
    const E* v = static_cast<const E*>(old ? a.vc : a.vin) + row * D;
    float z = 0.0f;
#pragma unroll
    for (int e = 0; e < P; ++e) z = fmaf(x[e], as_float(k[lane * P + e]), z);
    z = lanes::wave_sum(z);
    const float mn = fmaxf(m, z), f = __builtin_amdgcn_exp2f(m - mn), p = __builtin_amdgcn_exp2f(z - mn);
    l = l * f + p;
#pragma unroll
    for (int e = 0; e < P; ++e) acc[e] = acc[e] * f + p * as_float(v[lane * P + e]);
    m = mn;
  }
#pragma unroll
  for (int e = 0; e < P; ++e) put(o + lane * P + e, i >= 0 ? acc[e] / l : 0.0f);
}

// Rows of the tokens that the cache keeps, 16 bytes a thread: token t of the call's last
// min(n_tok, window), and the sinks among the others.  Grid (units, chunks of rows).
template <int RB>
__global__ void __launch_bounds__(256) window_store_kernel(PromptArgs a, int rows) {
  constexpr int CPR = RB / 16;
  const int u = blockIdx.x;
  const int pad = a.pad ? max(0, a.pad[u / a.n_kv_heads]) : 0;
  const int c = blockIdx.y * 256 + threadIdx.x;
  // the first `lead` rows are those of possible sinks, then the call's last ones
  const int r = c / CPR, ch = c % CPR;
  if (r >= rows) return;
  const int first = a.n_tok - min(a.n_tok, a.window);      // the first token kept for the window
  const int r0 = a.t0 - pad;
  // sinks of the call that lie before `first`: tokens max(0, -r0) on
  const int lead = rows - (a.n_tok - first);
  const int t = r < lead ? max(0, -r0) + r : first + r - lead;
  const int i = r0 + t;
  if (i < 0 || (r < lead && (i >= a.sinks || t >= first))) return;
  const int64_t src = ((int64_t)u * a.seq_ld + t) * RB + ch * 16;
  const int64_t dst =
      ((int64_t)u * (a.window + a.sinks) + window_slot(i, a.sinks, a.window)) * RB + ch * 16;
  *reinterpret_cast<uint4*>(static_cast<char*>(a.kc) + dst) =
      *reinterpret_cast<const uint4*>(static_cast<const char*>(a.kin) + src);
  *reinterpret_cast<uint4*>(static_cast<char*>(a.vc) + dst) =
      *reinterpret_cast<const uint4*>(static_cast<const char*>(a.vin) + src);
}

template <typename E, int D>
hipError_t launch_t(const PromptArgs& a, hipStream_t stream) {
  const int group = a.n_heads / a.n_kv_heads;
  const int64_t waves = (int64_t)a.units * group * a.n_tok;
  hipLaunchKernelGGL((window_prompt_kernel<E, D>), dim3((unsigned)((waves + 3) / 4)), dim3(256), 0,
                     stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int kept = a.n_tok < a.window ? a.n_tok : a.window;
  const int lead = a.sinks < a.n_tok - kept ? a.sinks : a.n_tok - kept;
  constexpr int RB = D * (int)sizeof(E);
  const unsigned chunks = (unsigned)(((int64_t)(kept + lead) * (RB / 16) + 255) / 256);
  hipLaunchKernelGGL((window_store_kernel<RB>), dim3((unsigned)a.units, chunks), dim3(256), 0, stream, a,
                     kept + lead);
  return hipGetLastError();
}

}  // namespace

bool prompt_fits(int units, int group, int n_tok) {
  return (int64_t)units * group * n_tok / 4 < 0x7FFFFFFF;
}

hipError_t launch_prompt(const PromptArgs& a, int dtype, int head_dim, int group, hipStream_t stream) {
  (void)group;
  if (dtype == BM_BF16)
    return head_dim == 128 ? launch_t<uint16_t, 128>(a, stream) : launch_t<uint16_t, 64>(a, stream);
  return head_dim == 128 ? launch_t<float, 128>(a, stream) : launch_t<float, 64>(a, stream);
}

}  // namespace bm
