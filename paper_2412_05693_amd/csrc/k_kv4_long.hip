// K10: one decode step over a long cache held in 4 bits, outputs only: K6's step
// (a cache that is never cut, more entries than a scoring step takes) with the
// rows as 4-bit floats.  kv4_split_kernel, grid (units, splits): a workgroup's
// waves attend to kSplit cached slots and leave one partial softmax per head;
// kv4_combine_kernel, one workgroup per unit and head, joins them with the step's own
// pair, writes the outputs and stores that pair in the slot behind the last.
#include <type_traits>

#include "bm_internal.h"
#include "bm_kv4_attn.h"
#include "bm_kv4_dev.h"
#include "bm_lanes.h"

namespace bm {
namespace {

using kv4::kChunk;
using kv4::kNegInf;

constexpr int kSplit = 512;              // slots per split workgroup
constexpr int kMaxSplits = kMaxCapAny / kSplit;
constexpr int NW = 4;

template <bool BF16, int D, int G>
__global__ void __launch_bounds__(64 * NW) kv4_split_kernel(Kv4DecodeArgs a) {
  using E = typename std::conditional<BF16, uint16_t, float>::type;
  using Attn = kv4::Attn<BF16, D, G>;
  constexpr int RB = Attn::RB, SB = Attn::SB;
  __shared__ float red[NW][G][D];
  __shared__ float s_m[NW][G], s_l[NW][G];
  const int u = blockIdx.x, c = blockIdx.y;
  const int bi = u / a.n_kv_heads, hk = u - bi * a.n_kv_heads;
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int64_t row0 = (int64_t)u * a.cap;
  const kv4::Planes pl = {static_cast<const uint8_t*>(a.kq) + row0 * RB,
                          static_cast<const uint8_t*>(a.ks) + row0 * SB,
                          static_cast<const uint8_t*>(a.vq) + row0 * RB,
                          static_cast<const uint8_t*>(a.vs) + row0 * SB, a.pos + row0};
  const E* qb = static_cast<const E*>(a.q) + ((int64_t)bi * a.n_heads + hk * G) * a.seq_ld * D;
  const int pad = a.pad ? max(0, a.pad[bi]) : 0;
  const int end = min(a.len0, (c + 1) * kSplit);

  Attn at;
  at.init(qb, a.seq_ld * D, lane);
  for (int base = c * kSplit + w * kChunk; base < end; base += NW * kChunk)
    at.chunk(pl, base, end, pad, a.scale_log2, [](int, const kv4::f32x4&) {});
  const float l = at.sum();
  if (lane < G) {
    s_m[w][lane] = at.m;
    s_l[w][lane] = l;
  }
  if (at.i < G) at.store_o(&red[w][at.i][0]);
  __syncthreads();
  // partial record of this split: [G][D + 2] floats (o, then m, l)
  float* out = a.part + ((int64_t)u * a.nsplit + c) * G * (D + 2);
  for (int idx = tid; idx < G * (D + 1); idx += 64 * NW) {
    const int g = idx / (D + 1), d = idx - g * (D + 1);
    float m = s_m[0][g];
#pragma unroll
    for (int i = 1; i < NW; ++i) m = fmaxf(m, s_m[i][g]);
    const float ref = m == kNegInf ? 0.0f : m;    // a split of hidden entries only
    float x = 0.0f;
#pragma unroll
    for (int i = 0; i < NW; ++i)
      x = fmaf(d < D ? red[i][g][d] : s_l[i][g], __builtin_amdgcn_exp2f(s_m[i][g] - ref), x);
    out[g * (D + 2) + (d < D ? d : D + 1)] = x;
    if (d == D) out[g * (D + 2) + D] = m;
  }
}

template <bool BF16, int D, int G>
__global__ void __launch_bounds__(256) kv4_combine_kernel(Kv4DecodeArgs a) {
  using E = typename std::conditional<BF16, uint16_t, float>::type;
  constexpr int NG = 256 / D;               // groups of D threads
  constexpr int RB = D / 2, SB = D / 32;
  __shared__ float wgt[kMaxSplits];
  __shared__ float red[NG][D];
  __shared__ float s_max[4], s_den[4], s_own;
  static_assert(kMaxSplits <= 256, "a thread per split");
  const int u = blockIdx.x, g = blockIdx.y;
  const int bi = u / a.n_kv_heads, hk = u - bi * a.n_kv_heads;
  const int tid = threadIdx.x, w = tid >> 6, lane = tid & 63;
  const int64_t plane = ((int64_t)bi * a.n_kv_heads + hk) * a.seq_ld;
  const E* knew = static_cast<const E*>(a.kin) + plane * D;
  const E* vnew = static_cast<const E*>(a.vin) + plane * D;
  const int64_t qrow = ((int64_t)bi * a.n_heads + hk * G + g) * a.seq_ld * D;
  const float* part = a.part + ((int64_t)u * a.nsplit * G + g) * (D + 2);
  const int64_t stride = (int64_t)G * (D + 2);
  const int n = a.nsplit;
  if (w == 0) {
    const float s = lanes::wave_sum(kv4::dot_part<BF16, D>(static_cast<const E*>(a.q) + qrow, knew, lane));
    if (lane == 0) s_own = s * a.scale_log2;
  }
  float m = tid < n ? part[tid * stride + D] : kNegInf;
  const float ll = tid < n ? part[tid * stride + D + 1] : 0.0f;
  const float wm = lanes::wave_max(m);
  if (lane == 0) s_max[w] = wm;
  __syncthreads();
  const float own = s_own;
  const float M = fmaxf(fmaxf(fmaxf(s_max[0], s_max[1]), fmaxf(s_max[2], s_max[3])), own);
  const float f = __builtin_amdgcn_exp2f(m - M);
  if (tid < n) wgt[tid] = f;
  const float den = lanes::wave_sum(tid < n ? f * ll : 0.0f);
  if (lane == 0) s_den[w] = den;
  __syncthreads();
  const int gi = tid / D, e = tid - gi * D;
  float num = 0.0f;
#pragma unroll 4
  for (int c = gi; c < n; c += NG) num = fmaf(wgt[c], part[c * stride + e], num);
  red[gi][e] = num;
  __syncthreads();
  if (tid < D) {
    const float p = __builtin_amdgcn_exp2f(own - M);
    float v;
    if constexpr (BF16) v = __uint_as_float((uint32_t)vnew[e] << 16);
    else v = vnew[e];
    float x = p * v;
#pragma unroll
    for (int i = 0; i < NG; ++i) x += red[i][e];
    x /= s_den[0] + s_den[1] + s_den[2] + s_den[3] + p;
    E* o = static_cast<E*>(a.o) + qrow + e;
    if constexpr (BF16) *o = __builtin_bit_cast(uint16_t, (__bf16)x);
    else *o = x;
  }
  if (g != 0) return;
  // the step's pair into slot len0
  if (tid < D / 4) {
    const int wh = tid / (D / 8), c = tid - wh * (D / 8);
    float x[8];
    uint32_t byte;
    kv4::load8<BF16>((wh ? vnew : knew) + c * 8, x);
    const uint32_t code = kv4::quantise8(x, &byte);
    const int64_t row = (int64_t)u * a.cap + a.len0;
    *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(wh ? a.vq : a.kq) + row * RB + 4 * c) = code;
    if ((c & 3) == 0) (static_cast<uint8_t*>(wh ? a.vs : a.ks))[row * SB + c / 4] = (uint8_t)byte;
  }
  if (tid == 0) {
    a.score[(int64_t)u * a.cap + a.len0] = 0.0f;
    a.pos[(int64_t)u * a.cap + a.len0] = a.cur_pos;
    a.len[u] = a.len0 + 1;
  }
}

template <bool BF16, int D, int G>
hipError_t launch_t(const Kv4DecodeArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL((kv4_split_kernel<BF16, D, G>), dim3((unsigned)a.units, (unsigned)a.nsplit),
                     dim3(64 * NW), 0, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((kv4_combine_kernel<BF16, D, G>), dim3((unsigned)a.units, (unsigned)G), dim3(256),
                     0, stream, a);
  return hipGetLastError();
}

template <bool BF16, int D>
hipError_t launch_g(const Kv4DecodeArgs& a, int group, hipStream_t stream) {
  switch (group) {
    case 1: return launch_t<BF16, D, 1>(a, stream);
    case 2: return launch_t<BF16, D, 2>(a, stream);
    case 4: return launch_t<BF16, D, 4>(a, stream);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace

int kv4_long_splits(int len0) { return (len0 + kSplit - 1) / kSplit; }

hipError_t launch_kv4_long(const Kv4DecodeArgs& a, int dtype, int head_dim, int group,
                           hipStream_t stream) {
  if (dtype == BM_BF16)
    return head_dim == 128 ? launch_g<true, 128>(a, group, stream) : launch_g<true, 64>(a, group, stream);
  return head_dim == 128 ? launch_g<false, 128>(a, group, stream) : launch_g<false, 64>(a, group, stream);
}

}  // namespace bm
