// K9: one decode step per unit over a cache held in 4 bits (include/bm_kv4.h): K4's
// step -- attention over the cached entries and the step's own pair, score
// update, ranking, one removal, in-place write -- with the cached rows as 4-bit
// floats (bm_kv4_attn.h) and the step's pair quantised into the slot it gets.
//
// One workgroup per unit; its waves take chunks of 64 cached slots in turn, each
// with its own running maximum and sum; logits stay in LDS, because the scores
// need every entry's probability under the whole unit's normaliser.  The step's own
// pair (as given, float32 products) joins where the waves' outputs do.
#include <type_traits>

#include "bm_internal.h"
#include "bm_kv4_attn.h"
#include "bm_kv4_dev.h"
#include "bm_lanes.h"

namespace bm {
namespace {

using kv4::kChunk;
using kv4::kNegInf;

// a probability: rounded once, never fused into the sum that uses it
__device__ __forceinline__ float prob(float z, float m, float inv) {
#pragma clang fp contract(off)
  return __builtin_amdgcn_exp2f(z - m) * inv;
}

template <bool BF16, int D, int G, int NW>
__global__ void __launch_bounds__(64 * NW) kv4_decode_kernel(Kv4DecodeArgs a) {
  using E = typename std::conditional<BF16, uint16_t, float>::type;
  using Attn = kv4::Attn<BF16, D, G>;
  constexpr int NT = 64 * NW;
  constexpr int RB = Attn::RB, SB = Attn::SB;
  constexpr int ZP = G < 2 ? 2 : G;       // planes of z: scores and weights end up in two of them
  extern __shared__ float dsm[];
  __shared__ float s_m[NW][G], s_l[NW][G], s_own[G];
  __shared__ uint64_t s_wkey[NW];
  __shared__ int s_wslot[NW];

  const int u = blockIdx.x;
  const int bi = u / a.n_kv_heads, hk = u - bi * a.n_kv_heads;
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int n = a.len0;
  const int nz = (n + kChunk - 1) & ~(kChunk - 1);
  float* z = dsm;                          // [ZP][nz] logits, by kv4::z_place
  float* red = z + ZP * nz;                // [NW][G][D] partial outputs
  const int64_t row0 = (int64_t)u * a.cap;
  const kv4::Planes pl = {static_cast<const uint8_t*>(a.kq) + row0 * RB,
                          static_cast<const uint8_t*>(a.ks) + row0 * SB,
                          static_cast<const uint8_t*>(a.vq) + row0 * RB,
                          static_cast<const uint8_t*>(a.vs) + row0 * SB, a.pos + row0};
  float* score = a.score + row0;
  int32_t* pos = a.pos + row0;
  const int64_t plane = ((int64_t)bi * a.n_kv_heads + hk) * a.seq_ld;
  const E* knew = static_cast<const E*>(a.kin) + plane * D;
  const E* vnew = static_cast<const E*>(a.vin) + plane * D;
  const E* qb = static_cast<const E*>(a.q) + ((int64_t)bi * a.n_heads + hk * G) * a.seq_ld * D;
  const int64_t head_stride = a.seq_ld * D;
  const int pad = a.pad ? max(0, a.pad[bi]) : 0;

  // the step's own pair in 4 bits (D / 8 lanes for each of the two rows)
  uint32_t code = 0, byte = 0;
  if (tid < D / 4) {
    float x[8];
    kv4::load8<BF16>((tid < D / 8 ? knew : vnew) + (tid % (D / 8)) * 8, x);
    code = kv4::quantise8(x, &byte);
  }
  for (int g = w; g < G; g += NW) {
    const float s = lanes::wave_sum(kv4::dot_part<BF16, D>(qb + g * head_stride, knew, lane));
    if (lane == 0) s_own[g] = s * a.scale_log2;
  }

  // 1. attention over the cached entries
  Attn at;
  at.init(qb, head_stride, lane);
  for (int base = w * kChunk; base < n; base += NW * kChunk) {
    at.chunk(pl, base, n, pad, a.scale_log2,
             [&](int t, const kv4::f32x4& zt) {
                   if (at.i < G)
                     *reinterpret_cast<kv4::f32x4*>(z + at.i * nz + base + 16 * t + 4 * at.h) = zt;
                 });
  }
  const float l = at.sum();
  if (lane < G) {
    s_m[w][lane] = at.m;
    s_l[w][lane] = l;
  }
  if (at.i < G) at.store_o(red + (w * G + at.i) * D);
  __syncthreads();

  // the unit's maximum and sum per head, the step's own pair included
  float mg[G], inv[G], p_own[G];
#pragma unroll
  for (int g = 0; g < G; ++g) {
    float m = s_own[g];
#pragma unroll
    for (int i = 0; i < NW; ++i) m = fmaxf(m, s_m[i][g]);
    const float e = __builtin_amdgcn_exp2f(s_own[g] - m);
    float sum = e;
#pragma unroll
    for (int i = 0; i < NW; ++i) sum += s_l[i][g] * __builtin_amdgcn_exp2f(s_m[i][g] - m);
    mg[g] = m;
    inv[g] = 1.0f / sum;
    p_own[g] = e;
  }

  // 2. outputs
  for (int idx = tid; idx < G * D; idx += NT) {
    const int g = idx / D, d = idx - g * D;
    float m = mg[0], r = inv[0], p = p_own[0];
#pragma unroll
    for (int k = 1; k < G; ++k)
      if (g == k) m = mg[k], r = inv[k], p = p_own[k];
    float v;
    if constexpr (BF16) v = __uint_as_float((uint32_t)vnew[d] << 16);
    else v = vnew[d];
    float x = p * v;
#pragma unroll
    for (int i = 0; i < NW; ++i)
      x = fmaf(red[(i * G + g) * D + d], __builtin_amdgcn_exp2f(s_m[i][g] - m), x);
    x *= r;
    E* o = static_cast<E*>(a.o) + (((int64_t)bi * a.n_heads + hk * G + g) * a.seq_ld) * D + d;
    if constexpr (BF16) *o = __builtin_bit_cast(uint16_t, (__bf16)x);
    else *o = x;
  }

  // 3. scores and ranking (entry n is the step's own)
  float w_own = 0.0f;
#pragma unroll
  for (int g = 0; g < G; ++g) w_own += prob(s_own[g], mg[g], inv[g]);
  const bool evict = n + 1 > a.kv_max;
  uint64_t best = ~0ull;
  int bslot = n;
  for (int j = tid; j < n; j += NT) {
    float* zj = z + kv4::z_place(j);
    float ps = 0.0f;
#pragma unroll
    for (int g = 0; g < G; ++g) ps += prob(zj[g * nz], mg[g], inv[g]);
    const float s = score[j] + ps;
    zj[0] = s;
    zj[nz] = ps;
    const uint64_t key = rank_key(a.rule, s, ps, pos[j], a.cur_pos);
    if (key < best) {
      best = key;
      bslot = j;
    }
  }
  if (tid == 0) {
    const uint64_t key = rank_key(a.rule, w_own, w_own, a.cur_pos, a.cur_pos);
    if (key < best) {
      best = key;
      bslot = n;
    }
  }
  int dst = n;                             // the slot that receives the step's pair
  if (evict) {
    const uint64_t wmin = lanes::wave_min_u64(best);
    const uint64_t holders = __ballot(best == wmin);
    bslot = __builtin_amdgcn_readlane(bslot, (int)__builtin_ctzll(holders));
    if (lane == 0) {
      s_wkey[w] = wmin;
      s_wslot[w] = bslot;
    }
    __syncthreads();
    uint64_t k0 = s_wkey[0];
    dst = s_wslot[0];
#pragma unroll
    for (int i = 1; i < NW; ++i)
      if (s_wkey[i] < k0) {
        k0 = s_wkey[i];
        dst = s_wslot[i];
      }
  }

  // 4. write back: scores (and the step's weights), each by the thread that formed them
  float* lw = a.lastw ? a.lastw + row0 : nullptr;
  for (int j = tid; j < n; j += NT) {
    const float* zj = z + kv4::z_place(j);
    score[j] = j == dst ? w_own : zj[0];
    if (lw) lw[j] = j == dst ? w_own : zj[nz];
  }
  if (tid == 0) a.len[u] = evict ? n : n + 1;
  // the step's pair, unless it is the one removed (entry n of a full cache)
  if (evict && dst == n) return;
  if (tid < D / 4) {
    const int wh = tid / (D / 8), c = tid - wh * (D / 8);
    uint8_t* q8 = static_cast<uint8_t*>(wh ? a.vq : a.kq) + (row0 + dst) * RB;
    *reinterpret_cast<uint32_t*>(q8 + 4 * c) = code;
    if ((c & 3) == 0) (static_cast<uint8_t*>(wh ? a.vs : a.ks))[(row0 + dst) * SB + c / 4] = (uint8_t)byte;
  }
  if (tid == 0) {
    pos[dst] = a.cur_pos;
    if (!evict) {
      score[n] = w_own;
      if (lw) lw[n] = w_own;
    }
  }
}

template <bool BF16, int D, int G, int NW>
hipError_t launch_w(const Kv4DecodeArgs& a, hipStream_t stream) {
  const size_t nz = ((size_t)a.len0 + kChunk - 1) & ~(size_t)(kChunk - 1);
  const size_t lds = sizeof(float) * ((G < 2 ? 2 : G) * nz + NW * G * D);
  hipLaunchKernelGGL((kv4_decode_kernel<BF16, D, G, NW>), dim3((unsigned)a.units), dim3(64 * NW),
                     lds, stream, a);
  return hipGetLastError();
}

template <bool BF16, int D, int G>
hipError_t launch_t(const Kv4DecodeArgs& a, hipStream_t stream) {
  return a.len0 > 256 ? launch_w<BF16, D, G, 8>(a, stream) : launch_w<BF16, D, G, 4>(a, stream);
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

hipError_t launch_kv4_decode(const Kv4DecodeArgs& a, int dtype, int head_dim, int group,
                             hipStream_t stream) {
  if (dtype == BM_BF16)
    return head_dim == 128 ? launch_g<true, 128>(a, group, stream) : launch_g<true, 64>(a, group, stream);
  return head_dim == 128 ? launch_g<false, 128>(a, group, stream) : launch_g<false, 64>(a, group, stream);
}

}  // namespace bm
