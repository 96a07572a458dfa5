// Attention of one unit's G query heads over cached entries held in 4 bits: what
// a wave does with 64 consecutive slots (shared by the scoring decode kernel and
// the split decode over long caches).
//
// Both products run on the matrix cores with the cached rows converted in
// registers (exactly: a 4-bit float times a power of two is a bfloat16).  S^T = K
// Q^T takes K rows as the A operand of a 16x16x32 MFMA: lane (i = lane % 16, h =
// lane / 16) loads one quarter of a row, which lies in one scale group, and the
// query operand is loaded with the same order of elements.  Lane (i, h) of S^T then
// holds the logits of slots 16 t + 4 h + r (tiles t = 0..3 of a chunk, r = 0..3) under
// query head i, and those slots are the contraction indices of O^T += V^T P^T that the
// lane stands for: its V operand needs the same slots, eight per MFMA, at one element
// of the head.  A lane loads 8 (head_dim 64: 4) consecutive elements of each of its
// slots' V rows, converts them in pairs and interleaves two slots with byte permutes;
// MFMA t of a head_dim then takes element 8 i + t (4 i + t) of every lane.  Nothing of
// this goes through LDS.
//
// The planes' layouts (include/bm_kv4.h) are made for these loads: V words of four
// consecutive slots, and the scales of a lane's slots, lie side by side, so a lane reads
// a chunk with ten loads of 4 or 16 bytes, each a whole run of memory per wave.
//
// Query rows are one bfloat16, which holds a bfloat16 row exactly; float32 rows are three
// bfloat16 parts (24 bits).  Probabilities are two parts over a bfloat16 batch: each weight
// loses at most 2^-16 of itself, where the output's own rounding to bfloat16 is 2^-8; over
// a float32 batch three parts, 2^-24.  Sums are float32.
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

// NT: rows are loaded past the caches (not read again before they would have left them).
template <bool BF16, int D, int G, bool NT>
struct Attn {
  static constexpr int kAux = NT ? 2 : 0;      // a load's non-temporal bit
  static constexpr int QP = BF16 ? 1 : 3;      // bfloat16 parts of a query element
  static constexpr int PP = BF16 ? 2 : 3;      // ... of a probability
  static constexpr int KM = D / 32;            // MFMAs (of 32 elements) per key tile
  static constexpr int DT = D / 16;            // output tiles of 16 elements
  static constexpr int KW = D / 32;            // words of a K row per lane
  static constexpr int RB = D / 2, SB = D / 32;   // bytes of a row's codes and scales

  // What a lane loads of a chunk of 64 slots.
  struct KRows {
    uint32_t w[4][KW];     // quarter h of slots 16 t + i
    uint32_t s;            // their scales, a byte each
  };
  struct VRows {
    u32x4 w[4];            // eight elements of slots 16 t + 4 h + r, [t][r]
    u32x4 s;               // their scales, a byte each
  };
  typedef bf16x8 Query[QP][KM];
  typedef f32x4 Out[DT];   // O^T: row 4 h + r of tile t: element DT (4 h + r) + t of head i
  typedef float Logits[16];   // slots 16 t + 4 h + r of the chunk, [4 t + r], head i

  int i, h;
  int k_at, ks_at, v_at, vs_at;   // byte offsets of the lane's first loads in a chunk

  __device__ __forceinline__ explicit Attn(int lane) {
    i = lane & 15;
    h = lane >> 4;
    k_at = i * RB + h * (D / 8);
    ks_at = k_scale_at<D>(i, D == 128 ? h : h >> 1);
    v_at = 4 * v_word<D>(4 * h, D == 128 ? i : i >> 1);
    vs_at = v_scale_at<D>(4 * h, D == 128 ? i >> 2 : i >> 3);
  }

  // query head min(i, G - 1) of the unit (columns past G repeat it, unused)
  template <typename E>
  __device__ __forceinline__ void load_q(const E* qb, int64_t head_stride, Query& q) const {
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
  }

  // Loads of the chunk at slot `base`, the same in every lane, of which `rows` slots are
  // there: the buffer resources end with them (V and the scales: with the layout's last
  // group of slots), loads past them return zeros.  What
  // differs between a lane's loads is an immediate; its offsets are made opaque here, or
  // the compiler keeps each of the sums in a register of its own.
  __device__ __forceinline__ void load_k(const Planes& pl, int base, int rows, KRows& k) const {
    rows = max(rows, 0);
    const auto kb = buffer(pl.kq + (int64_t)base * RB, rows * RB);
    const auto sb = buffer(pl.ks + (int64_t)base * SB, ((rows + 63) & ~63) * SB);
    int at = k_at, sat = ks_at;
    asm volatile("" : "+v"(at), "+v"(sat));
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      if constexpr (KW == 4) {
        const u32x4 x = __builtin_amdgcn_raw_buffer_load_b128(kb, at + 16 * t * RB, 0, kAux);
#pragma unroll
        for (int e = 0; e < 4; ++e) k.w[t][e] = x[e];
      } else {
        const u32x2 x = __builtin_amdgcn_raw_buffer_load_b64(kb, at + 16 * t * RB, 0, kAux);
        k.w[t][0] = x[0];
        k.w[t][1] = x[1];
      }
    }
    k.s = __builtin_amdgcn_raw_buffer_load_b32(sb, sat, 0, kAux);
  }

  __device__ __forceinline__ void load_v(const Planes& pl, int base, int rows, VRows& v) const {
    rows = max(rows, 0);
    const auto vb = buffer(pl.vq + (int64_t)base * RB, ((rows + 3) & ~3) * RB);
    const auto sb = buffer(pl.vs + (int64_t)base * SB, ((rows + 63) & ~63) * SB);
    int at = v_at, sat = vs_at;
    asm volatile("" : "+v"(at), "+v"(sat));
#pragma unroll
    for (int x = 0; x < 4; ++x) v.w[x] = __builtin_amdgcn_raw_buffer_load_b128(vb, at + 16 * x * RB, 0, kAux);
    v.s = __builtin_amdgcn_raw_buffer_load_b128(sb, sat, 0, kAux);
  }

  // The lane's slot e = 4 t + r of a chunk counts nowhere, whatever its row holds (a scale byte of 0 is a
  // power of two like any other).
  static __device__ __forceinline__ void hide_value(VRows& v, int e) {
    v.w[e >> 2][e & 3] = 0;
    v.s[e >> 2] &= ~(0xFFu << (8 * (e & 3)));
  }
  __device__ __forceinline__ void hide_values_past(VRows& v, int rows) const {
    if (rows < kChunk) {
      asm volatile("");                      // a branch, not 16 selects in every chunk
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (rows - 4 * h <= 16 * (e >> 2) + (e & 3)) hide_value(v, e);
    }
  }

  // logits of a chunk in log2 units; slots that are not there are -infinity
  __device__ __forceinline__ void logits(const KRows& k, const Query& q, float c2, int rows, Logits& z) const {
    f32x4 acc[4] = {};
    float s[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) s[t] = scale_in(k.s, t);
    // the four tiles in turn: an MFMA does not wait for the one before it
#pragma unroll
    for (int m = 0; m < KM; ++m) {
      bf16x8 a[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) a[t] = __builtin_bit_cast(bf16x8, bf16x8_of(k.w[t][m], s[t]));
#pragma unroll
      for (int p = QP - 1; p >= 0; --p)
#pragma unroll
        for (int t = 0; t < 4; ++t) acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[t], q[p][m], acc[t], 0, 0, 0);
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) z[e] = acc[e >> 2][e & 3] * c2;
    if (rows < kChunk) {
      asm volatile("");
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (rows - 4 * h <= 16 * (e >> 2) + (e & 3)) z[e] = kNegInf;
    }
  }

  // Left padding: calls hide(e) for the lane's slots e = 4 t + r whose position is below
  // `pad` (those that are not there count as position 0).
  template <typename Hide>
  __device__ __forceinline__ void pads(const Planes& pl, int base, int rows, int pad, Hide hide) const {
    const auto pb = buffer(pl.pos + base, max(rows, 0) * 4);
    int at = 16 * h;
    asm volatile("" : "+v"(at));
    int p[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) p[e] = (int)__builtin_amdgcn_raw_buffer_load_b32(pb, at + 64 * (e >> 2) + 4 * (e & 3), 0, 0);
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if (p[e] < pad) hide(e);
  }

  // O^T += V^T P^T over the lane's slots 8 u .. 8 u + 7 of its 16 in a chunk.  pw: the
  // bfloat16 parts of their probabilities, in order.
  __device__ __forceinline__ void add_values(const VRows& v, int u, const u32x4 (&pw)[PP], Out& o) const {
    uint32_t c[8];
    float s[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      c[e] = v.w[2 * u + (e >> 2)][e & 3];
      if constexpr (D == 64) c[e] >>= 16 * (i & 1);   // this lane's four of the eight elements
      s[e] = scale_in(v.s[2 * u + (e >> 2)], e & 3);
    }
    // output tiles two at a time: one code pair of each slot feeds both
    auto tiles = [&](auto sel) {
      constexpr int S = decltype(sel)::value;
      u32x4 v0, v1;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t x = bf16_pair<S>(c[2 * j], s[2 * j]), y = bf16_pair<S>(c[2 * j + 1], s[2 * j + 1]);
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

  static __device__ __forceinline__ void clear(Out& o) {
#pragma unroll
    for (int t = 0; t < DT; ++t) o[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  // Outputs of head i < G into that head's kRed words.  Element DT (4 h + r) + t goes to
  // word DT (4 r + h) + t, and a head's words are half the banks longer than its elements,
  // so that the lanes of a wave spread over the banks.
  static constexpr int kRed = D + 32;
  __device__ __forceinline__ void store_o(const Out& o, float* red) const {
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int t = 0; t < DT; t += 4)
        *reinterpret_cast<f32x4*>(red + DT * (4 * r + h) + t) = f32x4{o[t][r], o[t + 1][r], o[t + 2][r], o[t + 3][r]};
  }
  static __device__ __forceinline__ int red_word(int d) {
    const int row = d / DT;
    return DT * (((row & 3) << 2) | (row >> 2)) + d % DT;
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
