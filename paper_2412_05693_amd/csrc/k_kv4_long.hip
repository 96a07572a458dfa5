// K10: one decode step over a long cache held in 4 bits, outputs only: K6's step
// (a cache that is never cut, more entries than a scoring step takes) with the
// rows as 4-bit floats.  kv4_split_kernel, grid (units, splits): a workgroup's
// waves attend to a split of the cached slots and leave one partial softmax per head;
// kv4_combine_kernel, one workgroup per unit and head, joins them with the step's own
// pair, writes the outputs and stores that pair in the slot behind the last.
//
// d=128, G=4: 64 units of 8192 entries take 16.4 + 5.0 us (shortest 15.7 + 3.5) for 71 MB, a
// chain of loads and products per wave with the vector pipes busy 32% of the time and the
// matrix pipes 10%; 512 units 137 us for 587 MB (4.3 TB/s), bound by memory.
#include <type_traits>

#include "bm_internal.h"
#include "bm_kv4_attn.h"
#include "bm_kv4_dev.h"
#include "bm_lanes.h"

namespace bm {
namespace {

using kv4::kChunk;
using kv4::kNegInf;
using kv4::f32x4;

// Slots of a split, by the length alone, so that a sample's results are the same bits in
// any batch.  Each of a split's waves ends with its sums going through LDS, so longer
// splits are faster once they fill the card (us a step, bf16 d=128 G=4, splits of 512 ->
// 1024 -> 2048 slots: 64 units of 8192 entries 22.9 -> 21.6 -> 22.9, of 60001 109 -> 97 ->
// 97, 512 units of 20000 295 -> 274 -> 254) and slower while they do not (8 units of 4200:
// 9.9 -> 12.4 -> 17.5, of 8192: 10.2 -> 12.6 -> 18.2, of 20000: 12.3 -> 13.3 -> 19.8, of
// 60001: 21.7 -> 20.3 -> 21.9).
constexpr int kShortSplit = 512, kLongSplit = 1024, kShortEntries = 16384;
constexpr int kMaxSplits = kMaxCapAny / kLongSplit;
static_assert(kShortEntries / kShortSplit <= kMaxSplits, "splits of the shorter kind");
int split_slots(int n) { return n <= kShortEntries ? kShortSplit : kLongSplit; }

constexpr int NW = 4;                    // waves of a split (eight: the same or slower)
constexpr int kJoin = 256;               // threads that join a head's splits

template <bool BF16, int D, int G, bool NT>
__global__ void __launch_bounds__(64 * NW, BF16 ? 3 : 2) kv4_split_kernel(Kv4DecodeArgs a, int split) {
  using E = typename std::conditional<BF16, uint16_t, float>::type;
  using Attn = kv4::Attn<BF16, D, G, NT>;
  constexpr int RB = Attn::RB, SB = Attn::SB;
  __shared__ __align__(16) float red[NW][G][Attn::kRed];
  __shared__ float s_m[NW][G], s_l[NW][G];
  const int u = blockIdx.x, c = blockIdx.y;
  const int bi = u / a.n_kv_heads, hk = u - bi * a.n_kv_heads;
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int64_t row0 = (int64_t)u * a.cap;
  const kv4::Planes pl = {static_cast<const uint8_t*>(a.kq) + (int64_t)u * a.slots * RB,
                          static_cast<const uint8_t*>(a.ks) + (int64_t)u * a.slots * SB,
                          static_cast<const uint8_t*>(a.vq) + (int64_t)u * a.slots * RB,
                          static_cast<const uint8_t*>(a.vs) + (int64_t)u * a.slots * SB, a.pos + row0};
  const E* qb = static_cast<const E*>(a.q) + ((int64_t)bi * a.n_heads + hk * G) * a.seq_ld * D;
  const int pad = a.pad ? max(0, a.pad[bi]) : 0;
  const int end = min(a.len0, (c + 1) * split);

  const Attn at(lane);
  typename Attn::Query q;
  typename Attn::Out o;
  at.load_q(qb, a.seq_ld * D, q);
  Attn::clear(o);
  float m = kNegInf, l = 0.0f;             // running maximum, this lane's part of the sum
  // A chunk's rows of K are dead once its logits are formed, those of V once they are added:
  // the next chunk's loads take their registers there, and are on their way during the
  // other half of the work.
  typename Attn::KRows k;
  typename Attn::VRows v;
  int base = c * split + w * kChunk;
  at.load_k(pl, base, end - base, k);
  at.load_v(pl, base, end - base, v);
  for (; base < end; base += NW * kChunk) {
    const int rows = end - base, next = base + NW * kChunk;
    typename Attn::Logits z;
    at.logits(k, q, a.scale_log2, rows, z);
    at.load_k(pl, next, end - next, k);
    if (pad > 0)
      at.pads(pl, base, rows, pad, [&](int e) {
        z[e] = kNegInf;
        Attn::hide_value(v, e);
      });
    at.hide_values_past(v, rows);
    // the new maximum; what was summed so far is scaled to it
    float mx = m;
#pragma unroll
    for (int e = 0; e < 16; ++e) mx = fmaxf(mx, z[e]);
    mx = kv4::xor16_32_max(mx);
    const float ref = mx == kNegInf ? 0.0f : mx;   // nothing visible yet: all weights are 0
    if (__any(mx > m)) {
      const float shrink = __builtin_amdgcn_exp2f(m - ref);
      l *= shrink;
#pragma unroll
      for (int t = 0; t < Attn::DT; ++t) o[t] *= shrink;
    }
    m = mx;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      kv4::u32x4 pw[Attn::PP];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int e = 8 * x + 2 * j;
        const float p0 = __builtin_amdgcn_exp2f(z[e] - ref);
        const float p1 = __builtin_amdgcn_exp2f(z[e + 1] - ref);
        l += p0;
        l += p1;
        uint32_t part[Attn::PP];
        kv4::split_pair<Attn::PP>(p0, p1, part);
#pragma unroll
        for (int p = 0; p < Attn::PP; ++p) pw[p][j] = part[p];
      }
      at.add_values(v, x, pw, o);
    }
    at.load_v(pl, next, end - next, v);
  }
  l = lanes::add_xor<32>(lanes::add_xor<16>(l));
  if (lane < G) {
    s_m[w][lane] = m;
    s_l[w][lane] = l;
  }
  if (at.i < G) at.store_o(o, &red[w][at.i][0]);
  __syncthreads();
  // this split's partial outputs [G][D], and its (m, l) [G][2]
  const int64_t part = ((int64_t)u * a.nsplit + c) * G;
  float* out = a.part + part * D;
  float* out_ml = a.part + (int64_t)a.units * a.nsplit * G * D + part * 2;
  for (int idx = tid; idx < G * (D + 1); idx += 64 * NW) {
    const int g = idx / (D + 1), d = idx - g * (D + 1);
    float mg = s_m[0][g];
#pragma unroll
    for (int i = 1; i < NW; ++i) mg = fmaxf(mg, s_m[i][g]);
    const float ref = mg == kNegInf ? 0.0f : mg;    // a split of hidden entries only
    float x = 0.0f;
#pragma unroll
    for (int i = 0; i < NW; ++i)
      x = fmaf(d < D ? red[i][g][Attn::red_word(min(d, D - 1))] : s_l[i][g],
               __builtin_amdgcn_exp2f(s_m[i][g] - ref), x);
    if (d < D) {
      out[g * D + d] = x;
    } else {
      out_ml[2 * g] = mg;
      out_ml[2 * g + 1] = x;
    }
  }
}

// All of a head's partial outputs are on their way before the weights are known: a thread
// has four elements of every kRows-th split, 16 bytes each.
template <bool BF16, int D, int G>
__global__ void __launch_bounds__(kJoin) kv4_combine_kernel(Kv4DecodeArgs a) {
  using E = typename std::conditional<BF16, uint16_t, float>::type;
  constexpr int TPR = D / 4;                // threads per split's row
  constexpr int kRows = kJoin / TPR;        // splits read at a time
  constexpr int kEach = (kMaxSplits + kRows - 1) / kRows;
  constexpr int NWJ = kJoin / 64;
  __shared__ float wgt[kMaxSplits];
  __shared__ __align__(16) float red[kRows][D];
  __shared__ float s_max[NWJ], s_den[NWJ], s_own;
  static_assert(kMaxSplits <= kJoin, "a thread per split");
  const int u = blockIdx.x, g = blockIdx.y;
  const int bi = u / a.n_kv_heads, hk = u - bi * a.n_kv_heads;
  const int tid = threadIdx.x, w = tid >> 6, lane = tid & 63;
  const int64_t plane = ((int64_t)bi * a.n_kv_heads + hk) * a.seq_ld;
  const E* knew = static_cast<const E*>(a.kin) + plane * D;
  const E* vnew = static_cast<const E*>(a.vin) + plane * D;
  const int64_t qrow = ((int64_t)bi * a.n_heads + hk * G + g) * a.seq_ld * D;
  const int n = a.nsplit;
  const int64_t first = (int64_t)u * n * G + g;
  const float* part = a.part + first * D;
  const float* ml = a.part + (int64_t)a.units * n * G * D + first * 2;
  const int sc = min(tid, n - 1) * G * 2;
  const float m0 = ml[sc], ll = ml[sc + 1];
  const int ro = tid / TPR, e4 = (tid % TPR) * 4;
  f32x4 x[kEach];
#pragma unroll
  for (int k = 0; k < kEach; ++k)
    x[k] = *reinterpret_cast<const f32x4*>(part + (int64_t)min(ro + k * kRows, n - 1) * G * D + e4);
  if (w == 0) {
    const float s = lanes::wave_sum(kv4::dot_part<BF16, D>(static_cast<const E*>(a.q) + qrow, knew, lane));
    if (lane == 0) s_own = s * a.scale_log2;
  }
  const float wm = lanes::wave_max(m0);
  if (lane == 0) s_max[w] = wm;
  __syncthreads();
  const float own = s_own;
  float M = own;
#pragma unroll
  for (int i = 0; i < NWJ; ++i) M = fmaxf(M, s_max[i]);
  const float f = __builtin_amdgcn_exp2f(m0 - M);
  if (tid < n) wgt[tid] = f;
  const float den = lanes::wave_sum(tid < n ? f * ll : 0.0f);
  if (lane == 0) s_den[w] = den;
  __syncthreads();
  f32x4 num = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    const int c = ro + k * kRows;
    if (c < n) num += x[k] * wgt[c];
  }
  *reinterpret_cast<f32x4*>(&red[ro][e4]) = num;
  __syncthreads();
  if (tid < D) {
    const float p = __builtin_amdgcn_exp2f(own - M);
    float v;
    if constexpr (BF16) v = __uint_as_float((uint32_t)vnew[tid] << 16);
    else v = vnew[tid];
    float sum = p * v, all = p;
#pragma unroll
    for (int i = 0; i < kRows; ++i) sum += red[i][tid];
#pragma unroll
    for (int i = 0; i < NWJ; ++i) all += s_den[i];
    const float y = sum / all;
    E* o = static_cast<E*>(a.o) + qrow + tid;
    if constexpr (BF16) *o = __builtin_bit_cast(uint16_t, (__bf16)y);
    else *o = y;
  }
  if (g != 0) return;
  // the step's pair into slot len0
  if (tid < D / 4) {
    const int wh = tid / (D / 8), c = tid - wh * (D / 8);
    float x[8];
    uint32_t byte;
    kv4::load8<BF16>((wh ? vnew : knew) + c * 8, x);
    const uint32_t code = kv4::quantise8(x, &byte);
    kv4::store_row<D>(wh ? a.vq : a.kq, wh ? a.vs : a.ks, wh, (int64_t)u * a.slots, a.len0, c, code, byte);
  }
  if (tid == 0) {
    a.score[(int64_t)u * a.cap + a.len0] = 0.0f;
    a.pos[(int64_t)u * a.cap + a.len0] = a.cur_pos;
    a.len[u] = a.len0 + 1;
  }
}

template <bool BF16, int D, int G>
hipError_t launch_t(const Kv4DecodeArgs& a, hipStream_t stream) {
  // rows are read once per step: a cache larger than the last-level cache streams past it
  const size_t bytes = (size_t)a.units * a.len0 * (D + D / 16);
  const int split = split_slots(a.len0);
  const dim3 grid((unsigned)a.units, (unsigned)a.nsplit);
  if (bytes > kLastLevelCacheBytes)
    hipLaunchKernelGGL((kv4_split_kernel<BF16, D, G, true>), grid, dim3(64 * NW), 0, stream, a, split);
  else
    hipLaunchKernelGGL((kv4_split_kernel<BF16, D, G, false>), grid, dim3(64 * NW), 0, stream, a, split);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((kv4_combine_kernel<BF16, D, G>), dim3((unsigned)a.units, (unsigned)G),
                     dim3(kJoin), 0, stream, a);
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

int kv4_long_splits(int len0) { return (len0 + split_slots(len0) - 1) / split_slots(len0); }

hipError_t launch_kv4_long(const Kv4DecodeArgs& a, int dtype, int head_dim, int group,
                           hipStream_t stream) {
  if (dtype == BM_BF16)
    return head_dim == 128 ? launch_g<true, 128>(a, group, stream) : launch_g<true, 64>(a, group, stream);
  return head_dim == 128 ? launch_g<false, 128>(a, group, stream) : launch_g<false, 64>(a, group, stream);
}

}  // namespace bm
