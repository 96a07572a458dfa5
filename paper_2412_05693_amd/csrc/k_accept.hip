// A path of drafted tokens behind a cache (bm_draft.h).
//
// Bounded cache: the m accepted queries' probabilities are added to the scores of the
// entries they see, exp2(z - lse) with the log-sum-exps that the attention left, and the
// path's rows are appended; a sample that takes fewer than m tokens has its entries'
// positions moved on and gets hidden entries in the place of the others.  The cut is the
// context's own.  Every slot has one writer and its sum one order.
// Window cache: the rows go to their slots.
#include <type_traits>

#include "bm_internal.h"
#include "bm_lanes.h"
#include "bm_window_dev.h"

namespace bm {
namespace {

constexpr float kNegInf = -__builtin_huge_valf();
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float as_float(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
__device__ __forceinline__ float as_float(float x) { return x; }

// tokens that a sample takes, and path nodes within the tree
__device__ __forceinline__ int taken(const AcceptArgs& a, int bi) {
  return a.count ? min(max(a.count[bi], 0), a.m) : a.m;
}
__device__ __forceinline__ int node_at(const AcceptArgs& a, int bi, int i) {
  return min(max(a.path[(int64_t)bi * a.m + i], 0), a.n - 1);
}

// one wave a slot, the m new ones included; grid (units, chunks of 4 slots)
template <typename E, int D>
__global__ void __launch_bounds__(256) accept_kernel(AcceptArgs a) {
  constexpr int P = D / 64;
  const int group = a.n_heads / a.n_kv_heads;
  const int u = blockIdx.x, bi = u / a.n_kv_heads, hk = u - bi * a.n_kv_heads;
  const int s = blockIdx.y * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (s >= a.len0 + a.m) return;
  const int pad = a.pad ? max(0, a.pad[bi]) : 0;
  const int c = taken(a, bi), late = a.m - c;
  const int64_t slot = (int64_t)u * a.slots + s;
  const int mine = s - a.len0;                 // the token that a new slot is for
  const bool hidden = mine >= c;               // a token that the sample does not take
  E* k = static_cast<E*>(a.kc) + slot * D;
  E* v = static_cast<E*>(a.vc) + slot * D;
  float x[P];
  int pos;
  if (mine >= 0) {
    const int64_t row = ((int64_t)u * a.seq_ld + (hidden ? 0 : node_at(a, bi, mine))) * D;
#pragma unroll
    for (int e = 0; e < P; ++e) {
      const int d = lane * P + e;
      const E kx = hidden ? E(0) : static_cast<const E*>(a.kin)[row + d];
      k[d] = kx;
      v[d] = hidden ? E(0) : static_cast<const E*>(a.vin)[row + d];
      x[e] = as_float(kx);
    }
    pos = a.next_pos + mine;
  } else {
#pragma unroll
    for (int e = 0; e < P; ++e) x[e] = as_float(k[lane * P + e]);
    pos = a.pos[slot];
  }
  float sum = 0.0f, last = 0.0f;
  if (a.lse && !hidden && pos >= pad) {
    for (int i = max(mine, 0); i < c; ++i) {
      const int node = node_at(a, bi, i);
      float both = 0.0f;
      for (int g = 0; g < group; ++g) {
        const int64_t head = (int64_t)bi * a.n_heads + hk * group + g;
        const E* q = static_cast<const E*>(a.q) + (head * a.seq_ld + node) * D;
        float z = 0.0f;
#pragma unroll
        for (int e = 0; e < P; ++e) z = fmaf(as_float(q[lane * P + e]) * a.scale_log2, x[e], z);
        z = lanes::wave_sum(z);
        const float lse = a.lse[head * a.n + node];
        both += lse == kNegInf ? 0.0f : __builtin_amdgcn_exp2f(z - lse * kLog2e);
      }
      sum += both;
      last = i == c - 1 ? both : 0.0f;
    }
  }
  if (lane == 0) {
    a.score[slot] = (mine >= 0 ? 0.0f : a.score[slot]) + sum;
    a.pos[slot] = hidden ? mine - c : pos + late;
    if (a.lastw) a.lastw[slot] = last;
    if (s == 0) a.len[u] = a.len0 + a.m;
  }
}

// the samples' pads behind the kernel that reads them
__global__ void __launch_bounds__(256) pad_kernel(AcceptArgs a, int b) {
  const int bi = blockIdx.x * 256 + threadIdx.x;
  if (bi < b) a.pad[bi] = max(0, a.pad[bi]) + a.m - taken(a, bi);
}

// Window cache: a workgroup a sample, all KV heads' rows, and then the sample's pad.
template <int RB>
__global__ void __launch_bounds__(256) window_accept_kernel(AcceptArgs a) {
  constexpr int CPR = RB / 16;
  const int bi = blockIdx.x;
  const int pad = a.pad ? max(0, a.pad[bi]) : 0;
  const int c = taken(a, bi), end = a.next_pos - pad;
  const int rows = a.n_kv_heads * c;
  for (int x = threadIdx.x; x < rows * CPR; x += 256) {
    const int r = x / CPR, ch = x % CPR, hk = r / c, i = r - hk * c;
    // (of tokens that share a slot the last one stays)
    if (end + i < 0 || (end + i >= a.sinks && i < c - a.window)) continue;
    const int64_t u = (int64_t)bi * a.n_kv_heads + hk;
    const int64_t src = (u * a.seq_ld + node_at(a, bi, i)) * RB + ch * 16;
    const int64_t dst = (u * a.slots + window_slot(end + i, a.sinks, a.window)) * RB + ch * 16;
    *reinterpret_cast<uint4*>(static_cast<char*>(a.kc) + dst) =
        *reinterpret_cast<const uint4*>(static_cast<const char*>(a.kin) + src);
    *reinterpret_cast<uint4*>(static_cast<char*>(a.vc) + dst) =
        *reinterpret_cast<const uint4*>(static_cast<const char*>(a.vin) + src);
  }
  __syncthreads();
  if (a.count && threadIdx.x == 0) a.pad[bi] = pad + a.m - c;
}

template <typename E, int D>
hipError_t launch_t(const AcceptArgs& a, hipStream_t stream) {
  const int b = a.units / a.n_kv_heads;
  if (a.window) {
    hipLaunchKernelGGL((window_accept_kernel<D * (int)sizeof(E)>), dim3((unsigned)b), dim3(256), 0,
                       stream, a);
    return hipGetLastError();
  }
  const unsigned chunks = (unsigned)((a.len0 + a.m + 3) / 4);
  hipLaunchKernelGGL((accept_kernel<E, D>), dim3((unsigned)a.units, chunks), dim3(256), 0, stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.count) return e;
  hipLaunchKernelGGL(pad_kernel, dim3((unsigned)((b + 255) / 256)), dim3(256), 0, stream, a, b);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_accept(const AcceptArgs& a, int dtype, int head_dim, int group, hipStream_t stream) {
  (void)group;
  if (dtype == BM_BF16)
    return head_dim == 128 ? launch_t<uint16_t, 128>(a, stream) : launch_t<uint16_t, 64>(a, stream);
  return head_dim == 128 ? launch_t<float, 128>(a, stream) : launch_t<float, 64>(a, stream);
}

}  // namespace bm
