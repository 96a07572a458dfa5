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

constexpr int kTile = 32;     // keys of a wave

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

// tokens that a sample takes, and path nodes within the tree
__device__ __forceinline__ int taken(const AcceptArgs& a, int bi) {
  return a.count ? min(max(a.count[bi], 0), a.m) : a.m;
}
__device__ __forceinline__ int node_at(const AcceptArgs& a, int bi, int i) {
  return min(max(a.path[(int64_t)bi * a.m + i], 0), a.n - 1);
}

// a sample's pad behind the call; the largest stays (a sample that never begins)
__device__ __forceinline__ int grown(int pad, int late) {
  return pad > 0x7FFFFFFF - late ? 0x7FFFFFFF : pad + late;
}

template <bool BF16, int D>
struct AcceptCfg {
  using E = typename std::conditional<BF16, uint16_t, float>::type;
  static constexpr int RB = D * (int)sizeof(E);   // bytes of a row
  static constexpr int KL = RB / 64;              // 16-byte loads of a lane a row
};

// Scores, 32 keys a wave at a time: S = Q K^T in 16 x 16 tiles (rows: accepted token i and
// head g, row G i + g; columns: keys), exp2(S - lse), summed over the rows of a lane and
// then over the lanes of a key.  HBM-bound: the K rows are read once, the queries stay in
// the caches (512 units of 512 entries, d = 128: 18.8 us, 3.8 TB/s).  Grid (units, shares of the cached tiles and one more for the new tokens).
template <bool BF16, int D>
__global__ void __launch_bounds__(256) accept_kernel(AcceptArgs a) {
  using C = AcceptCfg<BF16, D>;
  constexpr int RB = C::RB, KL = C::KL, CPR = RB / 16;
  const int group = a.n_heads / a.n_kv_heads;
  const int u = blockIdx.x, bi = u / a.n_kv_heads, hk = u - bi * a.n_kv_heads;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int i16 = lane & 15, h = lane >> 4;
  const int pad = a.pad ? max(0, __builtin_amdgcn_readfirstlane(a.pad[bi])) : 0;
  const int c = __builtin_amdgcn_readfirstlane(taken(a, bi)), late = a.m - c;
  const int rows = c * group;
  const bool fresh = blockIdx.y + 1 == gridDim.y;      // the new tokens
  const int64_t plane = (int64_t)u * a.slots;
  const char* kin = static_cast<const char*>(a.kin) + (int64_t)u * a.seq_ld * RB;
  const char* vin = static_cast<const char*>(a.vin) + (int64_t)u * a.seq_ld * RB;
  if (fresh) {
    // their rows, zeros for the tokens that the sample does not take
    for (int x = threadIdx.x; x < a.m * CPR; x += 256) {
      const int i = x / CPR, ch = x % CPR;
      u32x4 k = {0, 0, 0, 0}, v = {0, 0, 0, 0};
      if (i < c) {
        const int64_t src = (int64_t)node_at(a, bi, i) * RB + ch * 16;
        k = *reinterpret_cast<const u32x4*>(kin + src);
        v = *reinterpret_cast<const u32x4*>(vin + src);
      }
      const int64_t dst = (plane + a.len0 + i) * RB + ch * 16;
      *reinterpret_cast<u32x4*>(static_cast<char*>(a.kc) + dst) = k;
      *reinterpret_cast<u32x4*>(static_cast<char*>(a.vc) + dst) = v;
    }
    if (threadIdx.x == 0) a.len[u] = a.len0 + a.m;
  }
  const int count = fresh ? a.m : a.len0;              // keys of this share's kind
  const int step = fresh ? 4 : 4 * ((int)gridDim.y - 1);
  const float c2 = a.scale_log2;
  for (int t = fresh ? w : (int)blockIdx.y * 4 + w; t * kTile < count; t += step) {
    u32x4 kf[2][KL];
    float sum[2] = {0.0f, 0.0f}, last[2] = {0.0f, 0.0f};
    if (a.lse) {
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const int key = min(t * kTile + 16 * s + i16, count - 1);
        const char* k = fresh ? kin + (int64_t)node_at(a, bi, key) * RB
                              : static_cast<const char*>(a.kc) + (plane + key) * RB;
#pragma unroll
        for (int kk = 0; kk < KL; ++kk) kf[s][kk] = *reinterpret_cast<const u32x4*>(k + 16 * h + 64 * kk);
      }
      for (int r0 = 0; r0 < rows; r0 += 16) {
        const int row = min(r0 + i16, rows - 1), i = row / group, g = row - i * group;
        const int64_t head = (int64_t)bi * a.n_heads + hk * group + g;
        const int node = node_at(a, bi, i);
        const char* q = static_cast<const char*>(a.q) + (head * a.seq_ld + node) * RB;
        u32x4 qf[KL];
#pragma unroll
        for (int kk = 0; kk < KL; ++kk) qf[kk] = *reinterpret_cast<const u32x4*>(q + 16 * h + 64 * kk);
        // (no weight: a row that sees nothing, or that is none)
        const float x = a.lse[head * a.n + node];
        const float lse2 = x == kNegInf || r0 + i16 >= rows ? -kNegInf : x * kLog2e;
        f32x4 z[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
#pragma unroll
        for (int kk = 0; kk < KL; ++kk)
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            if constexpr (BF16) {
              z[s] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, qf[kk]),
                                                             __builtin_bit_cast(bf16x8, kf[s][kk]), z[s], 0, 0, 0);
            } else {
#pragma unroll
              for (int j = 0; j < 4; ++j)
                z[s] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(qf[kk][j]), __uint_as_float(kf[s][kk][j]),
                                                            z[s], 0, 0, 0);
            }
          }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float l2 = __shfl(lse2, 4 * h + r);
          const int token = (r0 + 4 * h + r) / group;
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            float p = __builtin_amdgcn_exp2f(fmaf(z[s][r], c2, -l2));
            // a token sees itself and those before it
            if (fresh && token < t * kTile + 16 * s + i16) p = 0.0f;
            sum[s] += p;
            last[s] += token == c - 1 ? p : 0.0f;
          }
        }
      }
    }
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      sum[s] = lanes::add_xor<32>(lanes::add_xor<16>(sum[s]));
      if (a.lastw) last[s] = lanes::add_xor<32>(lanes::add_xor<16>(last[s]));
    }
    // lanes of quarter s hold the keys of half s
    const int key = t * kTile + 16 * h + i16;
    if (h < 2 && key < count) {
      const int64_t slot = plane + (fresh ? a.len0 + key : key);
      float all = h ? sum[1] : sum[0], end = h ? last[1] : last[0];
      int pos = fresh ? a.next_pos + key : pad > 0 || late > 0 ? a.pos[slot] : pad;
      // (a hidden entry has no score, whatever its row holds)
      if (pos < pad || (fresh && key >= c)) all = end = 0.0f;
      if (fresh) {
        a.score[slot] = all;
        a.pos[slot] = key < c ? pos + late : key - c;
      } else {
        if (a.lse) a.score[slot] += all;
        if (late > 0) a.pos[slot] = pos + late;
      }
      // (of a sample that takes none the last query stays the one before)
      if (a.lastw && (fresh || c > 0)) a.lastw[slot] = end;
    }
  }
}

// the samples' pads behind the kernel that reads them
__global__ void __launch_bounds__(256) pad_kernel(AcceptArgs a, int b) {
  const int bi = blockIdx.x * 256 + threadIdx.x;
  if (bi < b) a.pad[bi] = grown(max(0, a.pad[bi]), a.m - taken(a, bi));
}

// Window cache: a workgroup a sample, all KV heads' rows, and then the sample's pad.  Latency-bound
// for short paths (8 KV heads, d = 128, a call within a graph: 64 samples that take 4 tokens 3.3 us,
// 512 4.4); 64 samples that take 64 29 us, 2.3 TB/s, with 64 compute units at work.
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
    *reinterpret_cast<u32x4*>(static_cast<char*>(a.kc) + dst) =
        *reinterpret_cast<const u32x4*>(static_cast<const char*>(a.kin) + src);
    *reinterpret_cast<u32x4*>(static_cast<char*>(a.vc) + dst) =
        *reinterpret_cast<const u32x4*>(static_cast<const char*>(a.vin) + src);
  }
  __syncthreads();
  if (a.count && threadIdx.x == 0) a.pad[bi] = grown(pad, a.m - c);
}

// Workgroups over a unit's cached tiles: a wave's tile costs what a workgroup's start does, so
// as many as the compute units take at once, and no more than one tile a wave.
constexpr int kAcceptWorkgroups = 2048;

template <bool BF16, int D>
hipError_t launch_t(const AcceptArgs& a, hipStream_t stream) {
  const int b = a.units / a.n_kv_heads;
  if (a.window) {
    hipLaunchKernelGGL((window_accept_kernel<AcceptCfg<BF16, D>::RB>), dim3((unsigned)b), dim3(256), 0,
                       stream, a);
    return hipGetLastError();
  }
  const int most = ((a.len0 + kTile - 1) / kTile + 3) / 4;
  int shares = (kAcceptWorkgroups + a.units - 1) / a.units;
  if (shares > most) shares = most;
  // (without scores and with all positions as they are, only the new tokens)
  if (!a.lse && !a.count) shares = 0;
  hipLaunchKernelGGL((accept_kernel<BF16, D>), dim3((unsigned)a.units, (unsigned)shares + 1), dim3(256), 0, stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.count) return e;
  hipLaunchKernelGGL(pad_kernel, dim3((unsigned)((b + 255) / 256)), dim3(256), 0, stream, a, b);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_accept(const AcceptArgs& a, int dtype, int head_dim, int group, hipStream_t stream) {
  (void)group;
  if (dtype == BM_BF16)
    return head_dim == 128 ? launch_t<true, 128>(a, stream) : launch_t<true, 64>(a, stream);
  return head_dim == 128 ? launch_t<false, 128>(a, stream) : launch_t<false, 64>(a, stream);
}

}  // namespace bm
