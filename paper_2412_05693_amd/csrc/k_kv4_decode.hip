// K9: one decode step per unit over a cache held in 4 bits (include/bm_kv4.h): K4's
// step -- attention over the cached entries and the step's own pair, score
// update, ranking, one removal, in-place write -- with the cached rows as 4-bit
// floats (bm_kv4_attn.h) and the step's pair quantised into the slot it gets.
//
// One workgroup per unit:
//   1. logits of all cached entries into LDS, a wave at a time on 64 slots;
//   2. the exact softmax: sums per head, then every entry's probabilities, scores
//      and ranking; the probabilities stay in LDS as the parts that the next
//      product takes;
//   3. outputs: 64 slots a wave, chunk c into stream c % kStreams, the streams' sums
//      added in order; the step's own pair (as given, float32) joins at the end.
// The next chunk's rows are on their way while one is computed.
//
// HBM-bound: 4.25 bits an element and 12 bytes an entry for its score and position.
// 8192 units of 512 entries (d=128, G=4): 619 MB read and 30 written in 119 us where two
// steps over a layer make a pass (kernel trace: 121), 5.4 TB/s (a copy: 5.2); steps replayed
// from a graph over codes of random bits take 128-130.  The same loads without conversions
// and products take 111 us, 107 without the scores and positions too; an earlier layout
// whose rows came from the cache took 91.  The vector pipes are busy 46% of the time, the
// matrix pipes 17%.  Few units are bound by the chain of a workgroup: 8 units 8.7 us, and an
// earlier form with four waves took 7.7 without conversions and products.  A unit has one
// workgroup whatever its length, so few units leave most of the card idle: 8 units of 4096
// entries 31 us for 1 us of bytes.  Splitting a unit, as the split step over longer caches
// does, was not tried here: the scores need the unit's normaliser.
#include <type_traits>

#include "bm_internal.h"
#include "bm_kv4_attn.h"
#include "bm_kv4_dev.h"
#include "bm_lanes.h"

namespace bm {
namespace {

using kv4::f32x4;
using kv4::kChunk;
using kv4::kNegInf;
using kv4::u32x4;

// rows of scores and positions begin anywhere
typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
typedef int32_t i32x4u __attribute__((ext_vector_type(4), aligned(4)));

// Chunks of 64 slots are spread over so many partial output sums whatever the number of
// waves, so that a launch can choose it and a sample's results stay the same bits.
constexpr int kStreams = 4;

constexpr int kRing = 2;                   // chunks of K, and of V, in registers

// words of a head's plane of logits: 16 more than slots, so that the 16 words that a wave
// takes of each of four heads spread over all banks
__host__ __device__ __forceinline__ int plane_words(int nz) { return nz + 16; }

// a probability: rounded once, never fused into the sum that uses it
__device__ __forceinline__ float prob(float z, float m, float inv) {
#pragma clang fp contract(off)
  return __builtin_amdgcn_exp2f(z - m) * inv;
}

template <bool BF16, int D, int G, int NW, bool NT>
__global__ void __launch_bounds__(64 * NW, BF16 ? 3 : 2) kv4_decode_kernel(Kv4DecodeArgs a) {
  using E = typename std::conditional<BF16, uint16_t, float>::type;
  using Attn = kv4::Attn<BF16, D, G, NT>;
  constexpr int NTH = 64 * NW;
  constexpr int RB = Attn::RB, SB = Attn::SB, DT = Attn::DT;
  static_assert(NW <= kStreams, "a wave has whole streams");
  extern __shared__ __attribute__((aligned(16))) float dsm[];
  __shared__ float s_m[NW][G], s_own[G];
  __shared__ uint64_t s_wkey[NW];
  __shared__ int s_wslot[NW];

  const int u = blockIdx.x;
  const int bi = u / a.n_kv_heads, hk = u - bi * a.n_kv_heads;
  const int tid = threadIdx.x, w = NW == 1 ? 0 : __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int n = a.len0;
  const int nz = (n + kChunk - 1) & ~(kChunk - 1);
  const int chunks = nz / kChunk;
  const int zs = plane_words(nz);
  float* z = dsm;                          // [G][zs] logits, then probabilities
  float* red = z + G * zs;                 // [kStreams][G][kRed] partial outputs (NW > 1)
  const int64_t row0 = (int64_t)u * a.cap, slot0 = (int64_t)u * a.slots;
  const kv4::Planes pl = {static_cast<const uint8_t*>(a.kq) + slot0 * RB,
                          static_cast<const uint8_t*>(a.ks) + slot0 * SB,
                          static_cast<const uint8_t*>(a.vq) + slot0 * RB,
                          static_cast<const uint8_t*>(a.vs) + slot0 * SB, a.pos + row0};
  float* score = a.score + row0;
  int32_t* pos = a.pos + row0;
  float* lw = a.lastw ? a.lastw + row0 : nullptr;
  const int64_t plane = ((int64_t)bi * a.n_kv_heads + hk) * a.seq_ld;
  const E* knew = static_cast<const E*>(a.kin) + plane * D;
  const E* vnew = static_cast<const E*>(a.vin) + plane * D;
  const E* qb = static_cast<const E*>(a.q) + ((int64_t)bi * a.n_heads + hk * G) * a.seq_ld * D;
  E* ob = static_cast<E*>(a.o) + ((int64_t)bi * a.n_heads + hk * G) * a.seq_ld * D;
  const int64_t head_stride = a.seq_ld * D;
  const int pad = a.pad ? max(0, a.pad[bi]) : 0;
  const Attn at(lane);
  auto as_float = [](E x) -> float {
    if constexpr (BF16) return __uint_as_float((uint32_t)x << 16);
    else return x;
  };
  auto rounded = [](float x) -> E {
    if constexpr (BF16) return __builtin_bit_cast(uint16_t, (__bf16)x);
    else return x;
  };
  // a wave's chunks of V in order: every kStreams-th from its first, then its next stream's
  auto next_chunk = [&](int c) {
    if (c + kStreams < chunks) return c + kStreams;
    return (c % kStreams) + NW < kStreams ? (c % kStreams) + NW : chunks;
  };
  auto load_k = [&](int base, typename Attn::KRows& rows) { at.load_k(pl, base, n - base, rows); };
  auto load_v = [&](int c, typename Attn::VRows& rows) {
    c = min(c, chunks);
    at.load_v(pl, c * kChunk, n - c * kChunk, rows);
  };
  auto load_quad = [&](int qd, f32x4& sc, i32x4u& ps) {
    if (4 * qd + 3 < n) {
      sc = *reinterpret_cast<const f32x4u*>(score + 4 * qd);
      ps = *reinterpret_cast<const i32x4u*>(pos + 4 * qd);
    } else {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int j = min(4 * qd + r, max(n - 1, 0));   // slot 0 exists even when empty
        sc[r] = score[j];
        ps[r] = pos[j];
      }
    }
  };

  // The first rows of K and V, the queries, the step's own pair and the first scores are
  // all on their way before any is used.
  constexpr int kStep = NW * kChunk;
  constexpr int GW = (G + NW - 1) / NW;    // heads of this wave in what waves share out
  constexpr int NSP = NW == 1 ? 2 : 1;     // quads of slots per thread loaded ahead
  typedef E own_t __attribute__((ext_vector_type(D / 64)));
  typename Attn::Query q;
  typename Attn::KRows k[kRing];
  typename Attn::VRows v[kRing];
#pragma unroll
  for (int r = 0; r + 1 < kRing; ++r) load_k(w * kChunk + r * kStep, k[r]);
  at.load_q(qb, head_stride, q);
  own_t own_q[GW];
  const own_t own_k = reinterpret_cast<const own_t*>(knew)[lane];
#pragma unroll
  for (int x = 0; x < GW; ++x)
    own_q[x] = reinterpret_cast<const own_t*>(qb + min(w + x * NW, G - 1) * head_stride)[lane];
  float pair[8] = {};                      // D / 8 lanes for each of the step's two rows
  if (tid < D / 4) kv4::load8<BF16>((tid < D / 8 ? knew : vnew) + (tid % (D / 8)) * 8, pair);
  const E v_out = vnew[tid % D];           // (NW > 1: of this thread's outputs)
  int ahead = w;
#pragma unroll
  for (int r = 0; r + 1 < kRing; ++r) {
    load_v(ahead, v[r]);
    ahead = next_chunk(ahead);
  }
  f32x4 sp_score[NSP];
  i32x4u sp_pos[NSP];
#pragma unroll
  for (int e = 0; e < NSP; ++e) load_quad(tid + NTH * e, sp_score[e], sp_pos[e]);

  // ---------------- 1. logits ----------------
  {
    float m = kNegInf;
    auto take = [&](const typename Attn::KRows& rows, int base) {
      typename Attn::Logits zt;
      at.logits(rows, q, a.scale_log2, n - base, zt);
      if (pad > 0) at.pads(pl, base, n - base, pad, [&](int e) { zt[e] = kNegInf; });
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const f32x4 x = {zt[4 * t], zt[4 * t + 1], zt[4 * t + 2], zt[4 * t + 3]};
#pragma unroll
        for (int r = 0; r < 4; ++r) m = fmaxf(m, x[r]);
        if (at.i < G) *reinterpret_cast<f32x4*>(z + at.i * zs + base + 16 * t + 4 * at.h) = x;
      }
    };
    for (int base = w * kChunk; base < n;) {
#pragma unroll
      for (int r = 0; r < kRing; ++r) {
        if (base >= n) break;
        load_k(base + (kRing - 1) * kStep, k[(r + kRing - 1) % kRing]);
        take(k[r], base);
        base += kStep;
      }
    }
    m = kv4::xor16_32_max(m);
    if (lane < G) s_m[w][lane] = m;
#pragma unroll
    for (int x = 0; x < GW; ++x) {
      float s = 0.0f;
#pragma unroll
      for (int e = 0; e < D / 64; ++e) s = fmaf(as_float(own_q[x][e]), as_float(own_k[e]), s);
      s = lanes::wave_sum(s);
      if (lane == 0 && w + x * NW < G) s_own[w + x * NW] = s * a.scale_log2;
    }
  }
  uint32_t byte;
  const uint32_t code = kv4::quantise8(pair, &byte);
  __syncthreads();

  // ---------------- 2. softmax, scores, ranking ----------------
  // Each wave forms every head's maximum and sum by itself: 64 / G lanes a head.
  float mg[G], inv[G], p_own[G], w_own = 0.0f;
#pragma unroll
  for (int g = 0; g < G; ++g) {
    float m = s_own[g];
#pragma unroll
    for (int i = 0; i < NW; ++i) m = fmaxf(m, s_m[i][g]);
    mg[g] = m;
  }
  {
    constexpr int L = 64 / G;
    const int hg = lane / L;
    float m = mg[0];
#pragma unroll
    for (int g = 1; g < G; ++g)
      if (hg == g) m = mg[g];
    float s = 0.0f;
    const float* zh = z + hg * zs;
#pragma unroll 2
    for (int qd = lane % L; qd < nz / 4; qd += L) {
      const f32x4 x = *reinterpret_cast<const f32x4*>(zh + 4 * qd);
      float e[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) e[r] = __builtin_amdgcn_exp2f(x[r] - m);
      s += (e[0] + e[1]) + (e[2] + e[3]);
    }
    if constexpr (G == 1) s = lanes::wave_sum(s);
    else s = lanes::group_sum<L>(s);
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const float all = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(s), g * L));
      inv[g] = 1.0f / (all + __builtin_amdgcn_exp2f(s_own[g] - mg[g]));
    }
  }
  if constexpr (NW > 1) __syncthreads();   // every wave has read the logits
#pragma unroll
  for (int g = 0; g < G; ++g) {
    p_own[g] = prob(s_own[g], mg[g], inv[g]);
    w_own += p_own[g];
  }
  const bool evict = n + 1 > a.kv_max;
  uint64_t best = ~0ull;
  int bslot = n;                           // entry n is the step's own
  auto rank_quad = [&](int qd, const f32x4& sc, const i32x4u& ps) {
    float gain[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int g = 0; g < G; ++g) {
      u32x4* at_z = reinterpret_cast<u32x4*>(z + g * zs + 4 * qd);
      const f32x4 x = __builtin_bit_cast(f32x4, *at_z);
      float p[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        p[r] = prob(x[r], mg[g], inv[g]);
        gain[r] += p[r];
      }
      u32x4 y;
      if constexpr (BF16) {                // {part 0 of two pairs, part 1 of the same}
        uint32_t lo[2], hi[2];
        kv4::split_pair<2>(p[0], p[1], lo);
        kv4::split_pair<2>(p[2], p[3], hi);
        y = u32x4{lo[0], hi[0], lo[1], hi[1]};
      } else {
#pragma unroll
        for (int r = 0; r < 4; ++r) y[r] = __float_as_uint(p[r]);
      }
      *at_z = y;
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int j = 4 * qd + r;
      if (j >= n) continue;
      const float s = sc[r] + gain[r];
      score[j] = s;
      if (lw) lw[j] = gain[r];
      const uint64_t key = rank_key(a.rule, s, gain[r], ps[r], a.cur_pos);
      const bool less = key < best;
      best = less ? key : best;
      bslot = less ? j : bslot;
    }
  };
#pragma unroll
  for (int e = 0; e < NSP; ++e)
    if (tid + NTH * e < nz / 4) rank_quad(tid + NTH * e, sp_score[e], sp_pos[e]);
  for (int qd = tid + NTH * NSP; qd < nz / 4; qd += NTH) {
    f32x4 sc;
    i32x4u ps;
    load_quad(qd, sc, ps);
    rank_quad(qd, sc, ps);
  }
  if (tid == 0) {
    const uint64_t key = rank_key(a.rule, w_own, w_own, a.cur_pos, a.cur_pos);
    if (key < best) {
      best = key;
      bslot = n;
    }
  }
  if (evict) {
    const uint64_t wmin = lanes::wave_min_u64(best);
    const uint64_t holders = __ballot(best == wmin);
    bslot = __builtin_amdgcn_readlane(bslot, (int)__builtin_ctzll(holders));
    if (lane == 0) {
      s_wkey[w] = wmin;
      s_wslot[w] = bslot;
    }
  }
  __syncthreads();

  // ---------------- 3. outputs ----------------
  auto add_chunk = [&](typename Attn::VRows& rows, int base, typename Attn::Out& o) {
    if (pad > 0) at.pads(pl, base, n - base, pad, [&](int e) { Attn::hide_value(rows, e); });
    at.hide_values_past(rows, n - base);
    const float* pz = z + min(at.i, G - 1) * zs + base + 4 * at.h;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const u32x4 t0 = *reinterpret_cast<const u32x4*>(pz + 32 * x);
      const u32x4 t1 = *reinterpret_cast<const u32x4*>(pz + 32 * x + 16);
      u32x4 pw[Attn::PP];
      if constexpr (BF16) {
        pw[0] = u32x4{t0[0], t0[1], t1[0], t1[1]};
        pw[1] = u32x4{t0[2], t0[3], t1[2], t1[3]};
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const u32x4 t = j < 2 ? t0 : t1;
          uint32_t part[Attn::PP];
          kv4::split_pair<Attn::PP>(__uint_as_float(t[2 * (j & 1)]), __uint_as_float(t[2 * (j & 1) + 1]), part);
#pragma unroll
          for (int p = 0; p < Attn::PP; ++p) pw[p][j] = part[p];
        }
      }
      at.add_values(rows, x, pw, o);
    }
  };
  typename Attn::Out o, total;             // (total: NW = 1)
  Attn::clear(total);
  for (int c = w; c < chunks;) {
#pragma unroll
    for (int r = 0; r < kRing; ++r) {
      if (c >= chunks) break;
      load_v(ahead, v[(r + kRing - 1) % kRing]);
      ahead = next_chunk(ahead);
      if (c < kStreams) Attn::clear(o);    // a stream's first chunk
      add_chunk(v[r], c * kChunk, o);
      const int s = c % kStreams;
      c = next_chunk(c);
      if (c < chunks && c % kStreams == s) continue;
      // the stream's last chunk
      if constexpr (NW == 1) {
#pragma unroll
        for (int t = 0; t < DT; ++t) total[t] += o[t];
      } else {
        if (at.i < G) at.store_o(o, red + (s * G + at.i) * Attn::kRed);
      }
    }
  }
  if constexpr (NW == 1) {
    if (at.i < G) {
      float p = p_own[0];
#pragma unroll
      for (int g = 1; g < G; ++g)
        if (at.i == g) p = p_own[g];
      typedef E vec __attribute__((ext_vector_type(DT)));
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int d = DT * (4 * at.h + r);
        const vec y = *reinterpret_cast<const vec*>(vnew + d);
        vec x;
#pragma unroll
        for (int t = 0; t < DT; ++t) x[t] = rounded(fmaf(p, as_float(y[t]), total[t][r]));
        *reinterpret_cast<vec*>(ob + at.i * head_stride + d) = x;
      }
    }
  } else {
    static_assert(NTH % D == 0, "a thread's outputs are one element of several heads");
    __syncthreads();
    for (int idx = tid; idx < G * D; idx += NTH) {
      const int g = idx / D, d = idx - g * D;
      float p = p_own[0];
#pragma unroll
      for (int e = 1; e < G; ++e)
        if (g == e) p = p_own[e];
      float x = 0.0f;
#pragma unroll
      for (int s = 0; s < kStreams; ++s)
        if (s < chunks) x += red[(s * G + g) * Attn::kRed + Attn::red_word(d)];
      ob[g * head_stride + d] = rounded(fmaf(p, as_float(v_out), x));
    }
  }

  // ---------------- 4. the step's pair ----------------
  int dst = n;                             // the slot that receives it
  if (evict) {
    uint64_t k0 = s_wkey[0];
    dst = s_wslot[0];
#pragma unroll
    for (int i = 1; i < NW; ++i)
      if (s_wkey[i] < k0) {
        k0 = s_wkey[i];
        dst = s_wslot[i];
      }
  }
  if (tid == 0) a.len[u] = evict ? n : n + 1;
  // unless it is the one removed (entry n of a full cache)
  if (evict && dst == n) return;
  // its score, by the thread that wrote the slot's before (or the first, behind the last)
  const int owner = dst < n ? (dst >> 2) % NTH : 0;
  if (tid == owner) {
    score[dst] = w_own;
    if (lw) lw[dst] = w_own;
    pos[dst] = a.cur_pos;
  }
  if (tid < D / 4) {
    const int wh = tid / (D / 8), c8 = tid - wh * (D / 8);
    kv4::store_row<D>(wh ? a.vq : a.kq, wh ? a.vs : a.ks, wh, slot0, dst, c8, code, byte);
  }
}

template <bool BF16, int D, int G, int NW>
hipError_t launch_w(const Kv4DecodeArgs& a, hipStream_t stream) {
  const int nz = (a.len0 + kChunk - 1) & ~(kChunk - 1);
  const size_t lds = sizeof(float) * ((size_t)G * plane_words(nz) +
                                      (NW > 1 ? kStreams * G * kv4::Attn<BF16, D, G, false>::kRed : 0));
  // rows are read once per step: a cache larger than the last-level cache streams past it
  const size_t bytes = (size_t)a.units * a.len0 * (D + D / 16 + 8);
  const dim3 grid((unsigned)a.units), block(64 * NW);
  if (bytes > kLastLevelCacheBytes)
    hipLaunchKernelGGL((kv4_decode_kernel<BF16, D, G, NW, true>), grid, block, lds, stream, a);
  else
    hipLaunchKernelGGL((kv4_decode_kernel<BF16, D, G, NW, false>), grid, block, lds, stream, a);
  return hipGetLastError();
}

// One wave per unit or four.  One has no partial outputs to join and waits for no other
// wave, which is fastest once every compute unit has several units; four shorten a unit's
// chain of loads where it has few, and share the LDS that a long unit's logits fill.
// us a step with one -> with four, 16 steps replayed from a graph over one full cache, bf16
// d=128 G=4, entries by units (512 entries at 768 units 19.2 -> 18.7, at 896 19.9 -> 22.7):
//   entries  8             512            1024           2048           8192
//   64       6.8 -> 6.9    7.9 -> 8.5     8.7 -> 14.0    10.7 -> 21.5   31.8 -> 72.3
//   128      8.0 -> 7.1    9.1 -> 9.2     10.2 -> 14.8   14.7 -> 24.0   40.4 -> 76.1
//   512      15.7 -> 8.7   18.6 -> 13.8   20.9 -> 23.5   32.1 -> 39.7   129 -> 150
//   1024     26.9 -> 11.5  31.3 -> 20.4   34.9 -> 34.4   65.2 -> 72.2   252 -> 249
//   2048     48.9 -> 17.9  55.0 -> 32.9   70.9 -> 69.9   163 -> 128
//   4096     93.2 -> 30.4  112 -> 68.1    224 -> 129     447 -> 247
// The rule misses 1024 entries of 2048 units.  The other forms, measured the same way
// afterwards, part at about the same places:
//                      bf16 d=128 G=1   bf16 d=64 G=1    f32 d=128 G=4    f32 d=64 G=1
//   512 x 512          17.6 -> 12.0     13.6 -> 8.6      23.8 -> 15.5     16.4 -> 10.1
//   512 x 1024         19.4 -> 20.5     15.6 -> 13.5     26.1 -> 28.2     19.0 -> 17.9
//   512 x 8192         121 -> 135       71.6 -> 89.8     165 -> 213       95.7 -> 115
//   1000 x 1024        33.3 -> 31.0     25.7 -> 20.3     45.0 -> 40.6     32.2 -> 26.2
//   1024 x 8192        229 -> 232       134 -> 146       295 -> 321       169 -> 188
//   2048 x 1024        68.1 -> 62.7     44.5 -> 34.4     95.8 -> 83.1     60.5 -> 47.6
//   2048 x 8192        416 -> 436       250 -> 258       758 -> 593       323 -> 335
// (what it costs most there: 26% at 1000 entries x 1024 units of bf16 d=64, 15% at 1024 x 8192
// of f32 d=64).
// (Two waves are between the two, eight slower than four but for 5% at 8 units of 2048
// entries.  A third chunk of K or V on its way changes nothing: 129 -> 127-145.)
constexpr int kManyUnits = 768;          // three for every compute unit
constexpr int kFewEntries = 1024;

template <bool BF16, int D, int G>
hipError_t launch_t(const Kv4DecodeArgs& a, hipStream_t stream) {
  if (a.len0 <= kChunk || (a.units > kManyUnits && a.len0 < kFewEntries))
    return launch_w<BF16, D, G, 1>(a, stream);
  return launch_w<BF16, D, G, 4>(a, stream);
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
