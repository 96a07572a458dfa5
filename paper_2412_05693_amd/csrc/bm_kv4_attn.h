// Attention of one unit's G query heads over cached entries held in 4 bits: what
// a wave does with 64 consecutive slots (shared by the scoring decode kernel and
// the split decode over long caches).
//
// Both products run on the matrix cores with the cached rows converted in
// registers (exactly: a 4-bit float times a power of two is a bfloat16).  S^T = K
// Q^T takes K rows as the A operand of a 16x16x32 MFMA: lane (i = lane % 16, h =
// lane / 16) loads one quarter of a row, which lies in one scale group, and the
// query operand is loaded with the same order of elements.  Lane (i, h) of S^T
// then holds four keys of query head i per tile of 16, and those keys are the
// contraction indices of O^T += V^T P^T that the lane stands for: its V operand
// needs the same keys, eight per MFMA, at one element of the head.  A lane loads
// 8 (head_dim 64: 4) consecutive elements of each key's V row, converts them in
// pairs and interleaves two keys with byte permutes; MFMA t of a head_dim then
// takes element 8 i + t (4 i + t) of every lane.  Nothing goes through LDS.
//
// Query rows are one bfloat16 (float32: three bfloat16 parts, 24 bits) and
// probabilities two (three) parts, so the products are as exact as float32
// accumulation; queries of the batch in bfloat16 are exact as they are.
#pragma once

#include <type_traits>

#include "bm_internal.h"
#include "bm_kv4_dev.h"

namespace bm {
namespace kv4 {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;

constexpr float kNegInf = -__builtin_huge_valf();
constexpr int kChunk = 64;                 // slots a wave takes at a time

// Position of slot j among its 64: four lane groups of a tile hold every fourth
// slot, so a lane's four logits of a tile lie together.
__device__ __forceinline__ int z_place(int j) {
  return (j & ~15) | ((j & 3) << 2) | ((j >> 2) & 3);
}

__device__ __forceinline__ float xor16_32_max(float v) {
  const uint32_t x = __float_as_uint(v);
  const auto a = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  const uint32_t y = __float_as_uint(fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1])));
  const auto b = __builtin_amdgcn_permlane32_swap(y, y, false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// x as the sum of N bfloat16 parts, pairs (x0, x1) packed into one word per part
template <int N>
__device__ __forceinline__ void split_pair(float x0, float x1, uint32_t (&part)[N]) {
#pragma unroll
  for (int p = 0; p < N; ++p) {
    bf16x2 b;
    b[0] = (__bf16)x0;
    b[1] = (__bf16)x1;
    part[p] = __builtin_bit_cast(uint32_t, b);
    x0 -= __uint_as_float(part[p] << 16);
    x1 -= __uint_as_float(part[p] & 0xFFFF0000u);
  }
}

// one unit's cache
struct Planes {
  const uint8_t *kq, *ks, *vq, *vs;
  const int32_t* pos;
};

__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(const void* p, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, bytes, 0x00020000);
}

template <bool BF16, int D, int G>
struct Attn {
  static constexpr int QP = BF16 ? 1 : 3;      // bfloat16 parts of a query element
  static constexpr int PP = BF16 ? 2 : 3;      // ... of a probability
  static constexpr int KM = D / 32;            // MFMAs (of 32 elements) per key tile
  static constexpr int DT = D / 16;            // output tiles of 16 elements
  static constexpr int KW = D / 32;            // words of a K row per lane
  static constexpr int RB = D / 2, SB = D / 32;   // bytes of a row's codes and scales

  bf16x8 q[QP][KM];
  f32x4 o[DT];       // O^T: row 4 h + r of tile t is element DT (4 h + r) + t of head i
  float m, l;        // running maximum (log2 units), and this lane's part of the sum
  int i, h;

  // query head min(i, G - 1) of the unit (columns past G repeat it, unused)
  template <typename E>
  __device__ __forceinline__ void init(const E* qb, int64_t head_stride, int lane) {
    i = lane & 15;
    h = lane >> 4;
    const E* row = qb + min(i, G - 1) * head_stride + h * (D / 4);
#pragma unroll
    for (int k = 0; k < KM; ++k) {
      if constexpr (BF16) {
        q[0][k] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(row + 8 * k));
      } else {
        float x[8];
        load8<false>(row + 8 * k, x);
        u32x4 w[QP];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          uint32_t part[QP];
          split_pair<QP>(x[2 * e], x[2 * e + 1], part);
#pragma unroll
          for (int p = 0; p < QP; ++p) w[p][e] = part[p];
        }
#pragma unroll
        for (int p = 0; p < QP; ++p) q[p][k] = __builtin_bit_cast(bf16x8, w[p]);
      }
    }
#pragma unroll
    for (int t = 0; t < DT; ++t) o[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    m = kNegInf;
    l = 0.0f;
  }

  // One chunk: slots base .. base + 63 of the unit's planes, base the same in every lane.
  // Slots from `end` on are not there (the buffer resources end before them, so their
  // loads return zeros), and entries whose position is below `pad` are visible to no
  // query.  Hidden entries weigh nothing whatever their rows hold.  store(t, z): the
  // lane's logits z (log2 units) of slots base + 16 t + 4 r + h, r = 0..3.
  template <typename Store>
  __device__ __forceinline__ void chunk(const Planes& pl, int base, int end, int pad, float c2,
                                        Store store) {
    const int rows = end - base;
    const auto kb = buffer(pl.kq + (int64_t)base * RB, rows * RB);
    const auto vb = buffer(pl.vq + (int64_t)base * RB, rows * RB);
    const auto ksb = buffer(pl.ks + (int64_t)base * SB, rows * SB);
    const auto vsb = buffer(pl.vs + (int64_t)base * SB, rows * SB);
    // K by tiles of 16 rows, lane i on row 4 (i % 4) + i / 4 of the tile; V row by row.
    // The rest of an address is an immediate.
    const int ki = 4 * (i & 3) + (i >> 2);
    const int k_at = ki * RB + h * (D / 8), ks_at = ki * SB + (D == 128 ? h : h >> 1);
    const int v_at = h * RB + (D == 128 ? 4 * i : 4 * (i >> 1)), vs_at = h * SB + (D == 128 ? i >> 2 : i >> 3);
    uint32_t kw[4][KW], vw[16];
    float ksc[4], vsc[16];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      if constexpr (KW == 4) {
        const u32x4 x = __builtin_amdgcn_raw_buffer_load_b128(kb, k_at + 16 * t * RB, 0, 0);
#pragma unroll
        for (int e = 0; e < 4; ++e) kw[t][e] = x[e];
      } else {
        const u32x2 x = __builtin_amdgcn_raw_buffer_load_b64(kb, k_at + 16 * t * RB, 0, 0);
        kw[t][0] = x[0];
        kw[t][1] = x[1];
      }
      ksc[t] = scale_of(__builtin_amdgcn_raw_buffer_load_b8(ksb, ks_at + 16 * t * SB, 0, 0));
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      vw[e] = __builtin_amdgcn_raw_buffer_load_b32(vb, v_at + 4 * e * RB, 0, 0);
      vsc[e] = scale_of(__builtin_amdgcn_raw_buffer_load_b8(vsb, vs_at + 4 * e * SB, 0, 0));
    }
    // bit e: slot 4 e + h of the chunk is hidden; pads among them (the others are zeros)
    uint32_t hide = 0, pads = 0;
    if (pad > 0) {
      const auto pb = buffer(pl.pos + base, rows * 4);
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if ((int)__builtin_amdgcn_raw_buffer_load_b32(pb, (h + 4 * e) * 4, 0, 0) < pad) pads |= 1u << e;
      hide = pads;
    }
    if (rows < kChunk) {
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (4 * e + h >= rows) hide |= 1u << e;
    }

    // logits
    f32x4 z[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < KM; ++k) {
        const bf16x8 a = __builtin_bit_cast(bf16x8, bf16x8_of(kw[t][k], ksc[t]));
#pragma unroll
        for (int p = QP - 1; p >= 0; --p)
          acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, q[p][k], acc, 0, 0, 0);
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) z[t][r] = acc[r] * c2;
    }
    if (pad > 0 || rows < kChunk) {
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (hide & (1u << e)) z[e >> 2][e & 3] = kNegInf;
      if (pad > 0) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (pads & (1u << e)) {
            vw[e] = 0;
            vsc[e] = 1.0f;
          }
      }
    }
#pragma unroll
    for (int t = 0; t < 4; ++t) store(t, z[t]);

    // the new maximum; what was summed so far is scaled to it
    float mx = m;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) mx = fmaxf(mx, z[t][r]);
    mx = xor16_32_max(mx);
    const float ref = mx == kNegInf ? 0.0f : mx;   // nothing visible yet: all weights are 0
    const float shrink = __builtin_amdgcn_exp2f(m - ref);
    m = mx;
    l *= shrink;
#pragma unroll
    for (int t = 0; t < DT; ++t) o[t] *= shrink;

    // probabilities and O^T += V^T P^T, 32 keys at a time
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      u32x4 pw[PP];
#pragma unroll
      for (int j = 0; j < 4; ++j) {          // key pairs (2 j, 2 j + 1) of the eight
        const int t = 2 * u + (j >> 1), r = 2 * (j & 1);
        const float p0 = __builtin_amdgcn_exp2f(z[t][r] - ref);
        const float p1 = __builtin_amdgcn_exp2f(z[t][r + 1] - ref);
        l += p0;
        l += p1;
        uint32_t part[PP];
        split_pair<PP>(p0, p1, part);
#pragma unroll
        for (int p = 0; p < PP; ++p) pw[p][j] = part[p];
      }
      uint32_t* const c = vw + 8 * u;
      float* const f = vsc + 8 * u;
      if constexpr (D == 64) {               // this lane's four of eight elements
#pragma unroll
        for (int e = 0; e < 8; ++e) c[e] >>= 16 * (i & 1);
      }
      // output tiles two at a time: one code pair of each key feeds both
      auto tiles = [&](auto sel) {
        constexpr int S = decltype(sel)::value;
        u32x4 v0, v1;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t x = bf16_pair<S>(c[2 * j], f[2 * j]), y = bf16_pair<S>(c[2 * j + 1], f[2 * j + 1]);
          v0[j] = __builtin_amdgcn_perm(y, x, 0x05040100u);
          v1[j] = __builtin_amdgcn_perm(y, x, 0x07060302u);
        }
#pragma unroll
        for (int p = PP - 1; p >= 0; --p) {
          const bf16x8 b = __builtin_bit_cast(bf16x8, pw[p]);
          o[2 * S] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v0), b, o[2 * S], 0, 0, 0);
          o[2 * S + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v1), b, o[2 * S + 1], 0, 0, 0);
        }
      };
      tiles(std::integral_constant<int, 0>{});
      tiles(std::integral_constant<int, 1>{});
      if constexpr (D == 128) {
        tiles(std::integral_constant<int, 2>{});
        tiles(std::integral_constant<int, 3>{});
      }
    }
  }

  // the sum over the wave's lanes of one head
  __device__ __forceinline__ float sum() const {
    return lanes::add_xor<32>(lanes::add_xor<16>(l));
  }

  // outputs of head i < G into red[D] of that head
  __device__ __forceinline__ void store_o(float* red) const {
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int t = 0; t < DT; ++t) red[DT * (4 * h + r) + t] = o[t][r];
  }
};

// this lane's part of a row pair's dot product: elements lane, lane + 64, ...
template <bool BF16, int D, typename E>
__device__ __forceinline__ float dot_part(const E* x, const E* y, int lane) {
  float s = 0.0f;
#pragma unroll
  for (int e = 0; e < D / 64; ++e) {
    if constexpr (BF16) {
      s = fmaf(__uint_as_float((uint32_t)x[lane + 64 * e] << 16),
               __uint_as_float((uint32_t)y[lane + 64 * e] << 16), s);
    } else {
      s = fmaf(x[lane + 64 * e], y[lane + 64 * e], s);
    }
  }
  return s;
}

}  // namespace kv4
}  // namespace bm
