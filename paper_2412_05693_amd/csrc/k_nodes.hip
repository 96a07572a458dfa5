// The nodes of a tree of drafted tokens (or one generated token) over a cache: a bounded
// one or a window cache (bm_draft.h, bm_window.h).
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

// one wave a row (node, head)
template <typename E, int D>
__global__ void __launch_bounds__(256) nodes_kernel(NodesArgs a) {
  constexpr int P = D / 64;
  const int group = a.n_heads / a.n_kv_heads;
  const int64_t wave = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (wave >= (int64_t)a.units * group * a.n) return;
  const int node = (int)(wave % a.n);
  const int64_t head = wave / a.n;
  const int bi = (int)(head / a.n_heads), u = (int)(head / group);
  const int pad = a.pad ? max(0, a.pad[bi]) : 0;
  const int32_t* parent = a.parent ? a.parent + (int64_t)bi * a.n : nullptr;
  auto up = [&](int x) {
    const int p = parent ? parent[x] : -1;
    return p >= 0 && p < x ? p : -1;
  };
  int depth = 0;
  for (int x = up(node); x >= 0; x = up(x)) ++depth;
  const int i = a.next_pos + depth - pad;
  const E* q = static_cast<const E*>(a.q) + (head * a.seq_ld + node) * D;
  float x[P], acc[P], m = kNegInf, l = 0.0f;
#pragma unroll
  for (int e = 0; e < P; ++e) {
    x[e] = as_float(q[lane * P + e]) * a.scale_log2;
    acc[e] = 0.0f;
  }
  auto add = [&](const E* k, const E* v) {
    float z = 0.0f;
#pragma unroll
    for (int e = 0; e < P; ++e) z = fmaf(x[e], as_float(k[lane * P + e]), z);
    z = lanes::wave_sum(z);
    const float mn = fmaxf(m, z), f = __builtin_amdgcn_exp2f(m - mn), p = __builtin_amdgcn_exp2f(z - mn);
    l = l * f + p;
#pragma unroll
    for (int e = 0; e < P; ++e) acc[e] = acc[e] * f + p * as_float(v[lane * P + e]);
    m = mn;
  };
  if (i >= 0) {
    const Ring ring(a.next_pos - pad, a.sinks, max(a.window, 1));
    const int entries = a.window ? ring.filled() : a.len0;
    for (int s = 0; s < entries; ++s) {
      const int64_t row = (int64_t)u * a.slots + s;
      const bool seen = a.window ? window_sees(i, ring.index(s), a.sinks, a.window)
                                 : a.pos[row] >= pad;
      if (seen) add(static_cast<const E*>(a.kc) + row * D, static_cast<const E*>(a.vc) + row * D);
    }
    int j = i;
    for (int y = node; y >= 0; y = up(y), --j) {
      const int64_t row = (int64_t)u * a.seq_ld + y;
      if (j >= 0 && (!a.window || window_sees(i, j, a.sinks, a.window)))
        add(static_cast<const E*>(a.kin) + row * D, static_cast<const E*>(a.vin) + row * D);
    }
  }
  E* o = static_cast<E*>(a.o) + (head * a.seq_ld + node) * D;
#pragma unroll
  for (int e = 0; e < P; ++e) put(o + lane * P + e, l > 0.0f ? acc[e] / l : 0.0f);
  if (a.lse && lane == 0)
    a.lse[head * a.n + node] =
        l > 0.0f ? (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f : kNegInf;
}

// The node's rows into the window cache (n == 1), a workgroup a unit.
__global__ void __launch_bounds__(64) nodes_store_kernel(NodesArgs a, int row_bytes) {
  const int u = blockIdx.x, pad = a.pad ? max(0, a.pad[u / a.n_kv_heads]) : 0;
  const int i = a.next_pos - pad, c = threadIdx.x * 16;
  if (i < 0 || c >= row_bytes) return;
  const int64_t src = (int64_t)u * a.seq_ld * row_bytes + c;
  const int64_t dst = ((int64_t)u * a.slots + window_slot(i, a.sinks, a.window)) * row_bytes + c;
  *reinterpret_cast<uint4*>(static_cast<char*>(a.kc) + dst) =
      *reinterpret_cast<const uint4*>(static_cast<const char*>(a.kin) + src);
  *reinterpret_cast<uint4*>(static_cast<char*>(a.vc) + dst) =
      *reinterpret_cast<const uint4*>(static_cast<const char*>(a.vin) + src);
}

template <typename E, int D>
hipError_t launch_t(const NodesArgs& a, hipStream_t stream) {
  const int64_t waves = (int64_t)a.units * (a.n_heads / a.n_kv_heads) * a.n;
  hipLaunchKernelGGL((nodes_kernel<E, D>), dim3((unsigned)((waves + 3) / 4)), dim3(256), 0, stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.store) return e;
  hipLaunchKernelGGL(nodes_store_kernel, dim3((unsigned)a.units), dim3(64), 0, stream, a,
                     D * (int)sizeof(E));
  return hipGetLastError();
}

}  // namespace

size_t nodes_work_bytes(int units, int head_dim, int group, int n) {
  (void)units;
  (void)head_dim;
  (void)group;
  (void)n;
  return 16;
}

hipError_t launch_nodes(const NodesArgs& a, int dtype, int head_dim, int group, hipStream_t stream) {
  (void)group;
  if (dtype == BM_BF16)
    return head_dim == 128 ? launch_t<uint16_t, 128>(a, stream) : launch_t<uint16_t, 64>(a, stream);
  return head_dim == 128 ? launch_t<float, 128>(a, stream) : launch_t<float, 64>(a, stream);
}

}  // namespace bm
