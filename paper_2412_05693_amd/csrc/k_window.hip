// Tokens through a window cache (bm_window.h): a prompt's attention, and the storing of
// its rows behind it.
#include <type_traits>
#include <utility>

#include "bm_internal.h"
#include "bm_lanes.h"
#include "bm_window_dev.h"

// a lambda of the kernel, always part of it
#define BM_LAMBDA __device__ __attribute__((always_inline))

namespace bm {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __bf16 __attribute__((vector_size(8))) bf16v4;   // operand type of the LDS transpose read
typedef __attribute__((address_space(3))) bf16v4 lds_bf16v4;
typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
// the LDS object at byte `off` (an address kept as a number, so that it takes one register
// and an immediate offset)
template <typename T>
__device__ __forceinline__ T* lds_at(uint32_t off) { return (T*)(uintptr_t)off; }

constexpr float kNegInf = -__builtin_huge_valf();

// ---- bfloat16: tiles of 64 keys in LDS, 256 query rows a workgroup ----
//
// A workgroup is one unit and 256 / G tokens in all its G heads; a wave owns 64 rows of one
// head (two tiles of 32).  The keys that some row sees are numbered v = 0, 1, ..: the sinks
// before the first row's window, then everything from there to the last row.  With the row's
// index i and `shift` = what an index has more than its number behind the sinks, key v is
// visible iff  v <= i - shift  and  (v < sinks  or  v > i - shift - window).
//
// In halves of 32 keys, three stages at a time, so that matrix and vector work is there
// for each other: the logits of half t + 1 (S^T = K Q^T), the weights of half t, and
// O^T += V^T P^T of half t - 1.  LDS row order and operand layouts are those of the
// prefill kernel: K rows with bits 2 and 3 of their number swapped, so that a lane's
// logits are the second product's operand, V through the transposing LDS read.
// A wave of 64 rows reads every tile once for two products, which halves the LDS traffic
// of one with 32 rows.
//
// A weight is one bfloat16, off by at most 2^-8 of it, the row's sum takes it unrounded:
// outputs are off by 2.3e-3 (relative, root mean square) where exact ones rounded to
// bfloat16 are by 1.6e-3.  Two parts would be half as much matrix work again.
//
// MFMA-bound in principle; measured, the vector unit and the matrix unit take turns (39% of
// the waves' cycles are products, 9 vector instructions each).  32 heads, 8 KV heads,
// d = 128: 8 x 4096 tokens over a window of 1024 take 660 us (731 TFLOP/s, at 16 tiles a
// workgroup 9 of 42 us are its beginning and end), 2 x 32768 over 4096 4.1 ms (1.0 PFLOP/s);
// at d = 64 512 us and 3.0 ms (539 and 728 TFLOP/s).
// The loop's products alone run at 1.5 PFLOP/s.
constexpr int kPromptRows = 64;              // of a wave
constexpr int kPromptWaves = 4;
constexpr int kPromptTile = 64;              // keys
// A row's weights are taken against a maximum that moves once a logit is 2^24 beyond it: they
// stay below 2^24 and their sums below 2^40, which float32 and bfloat16 hold as exactly as
// smaller ones, and O is rescaled next to never (2^8: 15% of the halves of random rows).
constexpr float kRescaleLog2 = 24.0f;

__device__ __forceinline__ int kappa(int m) { return (m & ~12) | ((m & 4) << 1) | ((m & 8) >> 1); }

// chunk c of an LDS row r lies at position c ^ swz(r): no bank conflicts
template <int RB>
__device__ __forceinline__ constexpr int swz_k(int r) { return RB >= 256 ? r & 15 : (r >> 1) & 7; }
template <int RB>
__device__ __forceinline__ constexpr int swz_v(int r) { return RB >= 256 ? (r & 3) << 2 : ((r >> 1) & 1) << 2; }

__device__ __forceinline__ float xhalf_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  bf16x2 r = {(__bf16)lo, (__bf16)hi};
  return __builtin_bit_cast(uint32_t, r);
}
// logit register r of lane half h within a half tile: its key
__device__ __forceinline__ constexpr int key_of(int r, int h) {
  return 16 * (r >> 3) + 8 * h + 4 * ((r >> 2) & 1) + (r & 3);
}

// z = or += K Q^T of a 32 x 32 tile.  As assembly because z has to be in the registers that
// vector instructions work on: for a kernel of more than 256 registers the compiler puts
// every product's result into the accumulation registers, from which each of the
// logits would have to be copied first (622 TFLOP/s like that).  Operands of a product
// have arrived before it is issued (waits are the compiler's, for assembly too); what it
// does not count are the 19 wait states until a vector instruction may read the result:
// see z_settled and the steps' order.
template <bool FIRST>
__device__ __forceinline__ void mfma_z(f32x16& z, u32x4 k, u32x4 q) {
  if constexpr (FIRST)
    asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(z) : "v"(k), "a"(q));
  else
    asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+&v"(z) : "v"(k), "a"(q));
}
__device__ __forceinline__ void z_settled(f32x16 (&z)[2]) {
  asm volatile("s_nop 15\n\ts_nop 3" : "+v"(z[0]), "+v"(z[1]));
}

// x = max(x, y, z): one instruction (of values that assembly made the compiler first makes
// quiet numbers)
__device__ __forceinline__ void max3(float& x, float y, float z) {
  asm volatile("v_max3_f32 %0, %0, %1, %2" : "+v"(x) : "v"(y), "v"(z));
}

// a barrier for what the workgroup wrote to LDS (__syncthreads would also wait for the rows
// on their way into registers)
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// f(0), f(1), .. with numbers that are constants
template <typename F, int... I>
__device__ __forceinline__ void each(F f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}

// What a workgroup over a part of the keys leaves of a row: O without its division, m and l
// (none: -inf, 0), for launch_nodes_join.
__device__ __forceinline__ int64_t part_row(const PromptArgs& a, int u, int group, int g, int t) {
  return (((int64_t)u * a.nsplit + blockIdx.y) * group + g) * a.n_tok + t;
}
__device__ __forceinline__ void put_sums(const PromptArgs& a, int group, int d, int64_t at, float m, float l) {
  float* ml = a.part + (int64_t)a.units * a.nsplit * group * a.n_tok * d + at * 2;
  ml[0] = m;
  ml[1] = l;
}

// SPLIT: blockIdx.y is one of a.nsplit workgroups over the keys
template <int D, int G, bool SPLIT>
__global__ void __launch_bounds__(64 * kPromptWaves, 1) window_prompt_kernel(PromptArgs a, int tiles_per_unit) {
  constexpr int RB = 2 * D, CPR = RB / 16, KK = D / 16, MT = D / 32;
  constexpr int TILE = kPromptTile * RB;                     // bytes
  constexpr int NCOPY = kPromptTile * CPR / (64 * kPromptWaves);   // 16-byte chunks of a thread and tile
  constexpr int RPC = kPromptTile / NCOPY;                   // rows of a round of copies
  constexpr int PT = kPromptWaves * kPromptRows / G;         // tokens of a workgroup
  // two K tiles (t, t + 1) and three V tiles (t - 1, t, t + 1)
  __shared__ __attribute__((aligned(2 * TILE))) char lds[5 * TILE];
  char* const vbuf = lds + 2 * TILE;

  // workgroups of a unit on one XCD (they share keys): ids go round-robin over the 8 XCDs
  const int nwg = gridDim.x, L = blockIdx.x, q8 = nwg >> 3, r8 = nwg & 7, xcd = L & 7;
  const int lin = xcd * q8 + min(xcd, r8) + (L >> 3);
  const int u = lin / tiles_per_unit, pt = lin - u * tiles_per_unit;
  const int bi = u / a.n_kv_heads, hk = u - bi * a.n_kv_heads;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int n = lane & 31, h = lane >> 5;
  const int pad = a.pad ? max(0, __builtin_amdgcn_readfirstlane(a.pad[bi])) : 0;
  const int r0 = index_of(a.t0, pad);                        // the index of the call's first token
  const int p0 = pt * PT, tw = p0 + (w / G) * kPromptRows;   // first token of the workgroup, the wave
  const int p1 = min(p0 + PT, a.n_tok);
  const int64_t head = (int64_t)bi * a.n_heads + hk * G + w % G;

  // ---- the keys' numbers ----
  const int first = max(r0 + p0, 0), last = r0 + p1 - 1;     // indices of real rows
  const int lo = max(0, first - a.window + 1);
  const int lead = min(a.sinks, lo), shift = lo - lead;
  const int nv = lead + last - lo + 1;
  const int nt = (nv + kPromptTile - 1) / kPromptTile;
  // the workgroup's tiles: t0 to t1
  const int per = SPLIT ? (nt + a.nsplit - 1) / a.nsplit : nt;
  const int t0 = SPLIT ? min((int)blockIdx.y * per, nt) : 0, t1 = SPLIT ? min(t0 + per, nt) : nt;
  if (SPLIT && (last < 0 || t0 == t1)) {
    // pad tokens alone, or no keys left
    for (int c = lane; c < kPromptRows * CPR; c += 64) {
      const int t = tw + c / CPR;
      if (t >= a.n_tok) break;
      const int64_t at = part_row(a, u, G, w % G, t);
      float* y = a.part + at * D + c % CPR * 8;
      *reinterpret_cast<f32x4*>(y) = *reinterpret_cast<f32x4*>(y + 4) = f32x4{0, 0, 0, 0};
      if (c % CPR == 0) put_sums(a, G, D, at, kNegInf, 0.0f);
    }
    return;
  }
  if (last < 0) {
    // pad tokens alone
    for (int c = lane; c < kPromptRows * CPR; c += 64) {
      const int t = tw + c / CPR;
      if (t < a.n_tok)
        *reinterpret_cast<u32x4*>(static_cast<char*>(a.o) + (head * a.seq_ld + t) * RB + (c % CPR) * 16) = u32x4{0, 0, 0, 0};
    }
    return;
  }

  // ring places of the cached keys: number v lies at place0 + v (less the window at its end)
  const int ring0 = max(lo, a.sinks) - a.sinks;
  const int place0 = ring0 % a.window - (ring0 + a.sinks - shift);
  const char* kc = static_cast<const char*>(a.kc) + (int64_t)u * (a.window + a.sinks) * RB;
  const char* vc = static_cast<const char*>(a.vc) + (int64_t)u * (a.window + a.sinks) * RB;
  const char* ki = static_cast<const char*>(a.kin) + (int64_t)u * a.seq_ld * RB;
  const char* vi = static_cast<const char*>(a.vin) + (int64_t)u * a.seq_ld * RB;

  // ---- copies: the thread's 16-byte chunk of rows crow, crow + RPC, .. of tile t's K and V,
  //      through registers ----
  const int crow = threadIdx.x / CPR, cch = threadIdx.x % CPR;
  const int coff = crow * RB + cch * 16;
  u32x4 ks[NCOPY], vs[NCOPY];
  // a tile of the call's own rows alone is one run: no address arithmetic in vector registers
  struct Run {
    __amdgpu_buffer_rsrc_t k, v;
    bool is;
  };
  auto run_of = [&](int t) BM_LAMBDA {
    const int v0 = t * kPromptTile;
    const int64_t row = (int64_t)v0 + shift - r0;
    Run r;
    r.is = v0 >= lead && row >= 0 && v0 + kPromptTile <= nv;
    r.k = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(ki + row * RB), 0, TILE, 0x00020000);
    r.v = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(vi + row * RB), 0, TILE, 0x00020000);
    return r;
  };
  auto load_k = [&](const Run& r, int i) BM_LAMBDA { ks[i] = __builtin_amdgcn_raw_buffer_load_b128(r.k, coff, i * RPC * RB, 0); };
  auto load_v = [&](const Run& r, int i) BM_LAMBDA { vs[i] = __builtin_amdgcn_raw_buffer_load_b128(r.v, coff, i * RPC * RB, 0); };
  auto load_mixed = [&](u32x4 (&ks)[NCOPY], u32x4 (&vs)[NCOPY], int t) BM_LAMBDA {
    int v0 = t * kPromptTile + crow;
    asm volatile("" : "+v"(v0));      // (nothing of it outside the branch that it is in)
#pragma unroll
    for (int i = 0; i < NCOPY; ++i) {
      const int v = min(v0 + i * RPC, nv - 1);
      const int j = v < lead ? v : v + shift;
      int slot = place0 + v;
      slot = j < a.sinks ? j : a.sinks + (slot >= a.window ? slot - a.window : slot);
      const bool old = j < r0;
      const int64_t off = (int64_t)(old ? slot : j - r0) * RB + cch * 16;
      ks[i] = *reinterpret_cast<const u32x4*>((old ? kc : ki) + off);
      vs[i] = *reinterpret_cast<const u32x4*>((old ? vc : vi) + off);
    }
  };
  // (rows RPC apart have the same order of bits and chunks)
  const int kat = (crow & ~31) + kappa(crow & 31);
  const int kst = kat * RB + (cch ^ swz_k<RB>(kat)) * 16, vst = crow * RB + (cch ^ swz_v<RB>(crow)) * 16;
  auto store_k = [&](int i, int t) BM_LAMBDA {
    *reinterpret_cast<u32x4*>(lds + (t & 1) * TILE + kst + i * RPC * RB) = ks[i];
  };
  auto store_v = [&](int i, int at) BM_LAMBDA {
    *reinterpret_cast<u32x4*>(vbuf + at + vst + i * RPC * RB) = vs[i];
  };
  // (three tiles' rows and the queries on their way at once: one wait for memory)
  u32x4 k1[NCOPY], v1[NCOPY], k2[NCOPY], v2[NCOPY];
  load_mixed(ks, vs, t0);
  load_mixed(k1, v1, min(t0 + 1, t1 - 1));
  load_mixed(k2, v2, min(t0 + 2, t1 - 1));

  // ---- queries: lane (n, h) holds row n, chunks 2 kk + h ----
  u32x4 qf[2][KK];
#pragma unroll
  for (int rt = 0; rt < 2; ++rt) {
    const int t = min(tw + 32 * rt + n, a.n_tok - 1);
    const char* q = static_cast<const char*>(a.q) + (head * a.seq_ld + t) * RB;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
      qf[rt][kk] = *reinterpret_cast<const u32x4*>(q + 16 * (2 * kk + h));
  }
  auto store_tile = [&](int t) BM_LAMBDA {
#pragma unroll
    for (int i = 0; i < NCOPY; ++i) {
      store_k(i, t);
      store_v(i, t * TILE);
    }
  };
  store_tile(0);
#pragma unroll
  for (int i = 0; i < NCOPY; ++i) {
    ks[i] = k1[i];
    vs[i] = v1[i];
  }
  store_tile(1);
#pragma unroll
  for (int i = 0; i < NCOPY; ++i) {
    ks[i] = k2[i];
    vs[i] = v2[i];
  }

  // what a row sees, in key numbers (rows that are no tokens take the nearest one's)
  int vhi[2];
#pragma unroll
  for (int rt = 0; rt < 2; ++rt)
    vhi[rt] = max(min(r0 + tw + 32 * rt + n, last), first) - shift;
  const int wfirst = max(min(r0 + tw, last), first) - shift;
  const int wlast = max(min(r0 + tw + kPromptRows - 1, last), first) - shift;
  // a half whose keys every row of the wave sees
  auto plain = [&](int t) BM_LAMBDA {
    const int v0 = 32 * t;
    return v0 + 31 <= wfirst && (v0 + 31 < a.sinks || v0 > wlast - a.window);
  };

  const int frag0 = n * RB + (h ^ swz_k<RB>(n)) * 16;
  const int j16 = lane & 15, vrow = 8 * h + (j16 >> 2);
  const int vbase = vrow * RB + 16 * swz_v<RB>(vrow) + (16 * ((lane >> 4) & 1) + 4 * (j16 & 3)) * 2;
  const float c2 = a.scale_log2;

  f32x16 o[2][MT];
  float m[2] = {kNegInf, kNegInf}, l[2] = {0.0f, 0.0f};
#pragma unroll
  for (int rt = 0; rt < 2; ++rt)
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) o[rt][mt] = f32x16{};

  // operand addresses in LDS: K of tile t + 1 or t, V of the half before
  uint32_t ka[KK], va[MT];
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_void*)lds;
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) ka[kk] = lds0 + (uint32_t)(frag0 ^ (32 * kk));
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) va[mt] = lds0 + 4 * TILE + (uint32_t)(vbase ^ (64 * mt));

  // hide what rows do not see of half t: the row's keys as bits, then two instructions a logit
  auto hide = [&](f32x16 (&z)[2], float (&top)[2], int t) BM_LAMBDA {
    const int v0 = 32 * t;
    auto below = [](int x) BM_LAMBDA { return x <= 0 ? 0u : x >= 32 ? ~0u : (1u << x) - 1; };   // keys < x
    const uint32_t sinks = below(a.sinks - v0);
#pragma unroll
    for (int rt = 0; rt < 2; ++rt) {
      const uint32_t in = below(vhi[rt] + 1 - v0), old = below(vhi[rt] + 1 - a.window - v0);
      const uint32_t seen = in & (~old | sinks);
      const int bits = (int)(seen >> (8 * h));       // lane half h's keys all have 8 h
      top[rt] = kNegInf;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const uint32_t keep = (uint32_t)__builtin_amdgcn_sbfe(bits, key_of(r, 0), 1);   // ~0 or 0
        z[rt][r] = __uint_as_float((__float_as_uint(z[rt][r]) & keep) | (0xFF800000u & ~keep));
        if (r & 1) max3(top[rt], z[rt][r - 1], z[rt][r]);
      }
    }
  };

  // One half: zo holds half t's logits (what nobody sees is hidden), top their maxima, po half
  // t - 1's weights, kpre the first operands of half t + 1's logits, raised whether some row's
  // maximum has to move.  KH: which half of its tile t + 1, and t - 1, is; side(j): what
  // else goes behind product j.
  u32x4 kpre[2];
  bool raised;
  float top[2] = {kNegInf, kNegInf};
  auto exceeds = [&]() BM_LAMBDA {
    return __ballot(top[0] * c2 > m[0] + kRescaleLog2 || top[1] * c2 > m[1] + kRescaleLog2) != 0;
  };
  auto step = [&](auto kh_tag, auto side, f32x16 (&zn)[2], f32x16 (&zo)[2], u32x4 (&pn)[2][2],
                  const u32x4 (&po)[2][2], int t) BM_LAMBDA {
    constexpr int KH = decltype(kh_tag)::value;
    // the maximum a row's weights are taken against; O follows behind this step's product
    float f[2] = {1.0f, 1.0f};
    const bool raise = raised;
    if (__builtin_expect(raise, 0)) {
#pragma unroll
      for (int rt = 0; rt < 2; ++rt) {
        const float mn = fmaxf(m[rt], xhalf_max(top[rt]) * c2);
        f[rt] = mn == kNegInf ? 1.0f : __builtin_amdgcn_exp2f(m[rt] - mn);
        m[rt] = mn;
        l[rt] *= f[rt];
      }
    }
    float ref[2];
#pragma unroll
    for (int rt = 0; rt < 2; ++rt) ref[rt] = m[rt] == kNegInf ? 0.0f : m[rt];

    // 2 KK logit products, then 4 MT value products, each with its share of the weights behind
    // it: about as many cycles as the product takes
    constexpr int NQ = 2 * KK, NP = 4 * MT, NS = NQ + NP, kAhead = 2, NB = kAhead + 1;
    u32x4 kf[NB], vf[NB];
    kf[0] = kpre[0];
    kf[1] = kpre[1];
    auto k_fetch = [&](int j) BM_LAMBDA { kf[j % NB] = *lds_at<lds_u32x4>(ka[j] + KH * 32 * RB); };
    auto v_fetch = [&](int j) BM_LAMBDA {
      const uint32_t x = va[j % MT] + (KH * 32 + 16 * (j / MT)) * RB;
      const bf16v4 x0 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(lds_at<lds_bf16v4>(x));
      const bf16v4 x1 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(lds_at<lds_bf16v4>(x + 4 * RB));
      const u32x2 y0 = __builtin_bit_cast(u32x2, x0), y1 = __builtin_bit_cast(u32x2, x1);
      vf[j % NB] = u32x4{y0.x, y0.y, y1.x, y1.y};
    };
    float x[2], e[2];
    float sum[2] = {0.0f, 0.0f};
    // weight i of the lane's 32, in three stages (argument, exp2, sum and packing) so that
    // none waits for the one before
    auto args = [&](int i) BM_LAMBDA { x[i & 1] = fmaf(zo[i / 16][i % 16], c2, -ref[i / 16]); };
    float even;
    auto sums = [&](int i) BM_LAMBDA {
      sum[i / 16] += e[i & 1];
      if (i & 1) {
        uint32_t y = pack2(even, e[1]);
        asm volatile("" : "+v"(y), "+v"(sum[i / 16]));   // (made here, not where the next step uses it)
        pn[i / 16][(i / 8) & 1][(i / 2) & 3] = y;
      } else {
        asm volatile("" : "+v"(sum[i / 16]));
        even = e[0];
      }
    };
    auto weight = [&](int i) BM_LAMBDA {
      const float y = __builtin_amdgcn_exp2f(x[i & 1]);
      if (i > 0) sums(i - 1);
      e[i & 1] = y;
      if (i + 1 < 32) args(i + 1);
    };
    args(0);
    float nt0[2] = {kNegInf, kNegInf};
    each([&](auto jc) BM_LAMBDA {
      constexpr int j = decltype(jc)::value;
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (j < NQ) {
        constexpr int kk = j / 2, rt = j % 2;
        if constexpr (kk == 0) mfma_z<true>(zn[rt], kf[kk % NB], qf[rt][kk]);
        else mfma_z<false>(zn[rt], kf[kk % NB], qf[rt][kk]);
      } else {
        constexpr int q = (j - NQ) / 2, rt = j % 2, mt = q % MT, s = q / MT;
        o[rt][mt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vf[q % NB]),
                                                            __builtin_bit_cast(bf16x8, po[rt][s]), o[rt][mt], 0, 0, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (j % 2 == 0) {
        constexpr int next = j / 2 + kAhead;         // the operand that comes kAhead pairs on
        if constexpr (next < KK) k_fetch(next);
        else if constexpr (next < NS / 2) v_fetch(next - KK);
        else {
          // (the next tile's first rows, which all waves wrote: behind the barrier, when this
          // step's own operands have been read)
          if constexpr (KH == 1 && next == NS / 2) lds_barrier();
          kpre[next - NS / 2] = *lds_at<lds_u32x4>(KH ? ka[next - NS / 2] ^ TILE : ka[next - NS / 2] + 32 * RB);
        }
      }
#pragma unroll
      for (int i = j * 32 / NS; i < (j + 1) * 32 / NS; ++i) weight(i);
      // maxima of the new logits (the last of their products is kWait value products and the
      // weights between them away), and whether they matter
      constexpr int kWait = NP / 4, kMax = NP - kWait - 2;
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (NQ + kWait + i * kMax / 16 == j) max3(nt0[i / 8], zn[i / 8][2 * (i % 8)], zn[i / 8][2 * (i % 8) + 1]);
      side(jc);
      if constexpr (j == NS - 2) {
        top[0] = nt0[0];
        top[1] = nt0[1];
        raised = exceeds();
      }
    }, std::make_integer_sequence<int, NS>{});
    sums(31);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int rt = 0; rt < 2; ++rt) l[rt] += sum[rt];
    if (__builtin_expect(raise, 0)) {
      asm volatile("" : "+v"(f[0]), "+v"(f[1]));    // (not multiplied by 1 every time)
#pragma unroll
      for (int rt = 0; rt < 2; ++rt)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          o[rt][mt] *= f[rt];
          asm volatile("" : "+a"(o[rt][mt]));       // (back in its registers on this path)
        }
    }
    if (!plain(t + 1)) {
      hide(zn, top, t + 1);
      raised = exceeds();
    }
  };

  f32x16 za[2], zb[2];
  u32x4 pa[2][2], pb[2][2];
  // nothing comes before the first half: weights and values of zero
#pragma unroll
  for (int rt = 0; rt < 2; ++rt)
#pragma unroll
    for (int s = 0; s < 2; ++s) pb[rt][s] = u32x4{0, 0, 0, 0};
  for (int c = threadIdx.x; c < 32 * CPR; c += 64 * kPromptWaves)
    *reinterpret_cast<u32x4*>(vbuf + 2 * TILE + 32 * RB + c * 16) = u32x4{0, 0, 0, 0};
  __syncthreads();
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) {
    const u32x4 kf = *lds_at<lds_u32x4>(ka[kk]);
#pragma unroll
    for (int rt = 0; rt < 2; ++rt) {
      if (kk == 0) mfma_z<true>(za[rt], kf, qf[rt][kk]);
      else mfma_z<false>(za[rt], kf, qf[rt][kk]);
    }
  }
  z_settled(za);
#pragma unroll
  for (int rt = 0; rt < 2; ++rt)
#pragma unroll
    for (int r = 0; r < 16; r += 2) max3(top[rt], za[rt][r], za[rt][r + 1]);
  if (!plain(2 * t0)) hide(za, top, 2 * t0);
  raised = exceeds();
#pragma unroll
  for (int i = 0; i < 2; ++i) kpre[i] = *lds_at<lds_u32x4>(ka[i] + 32 * RB);
  // Tile t's halves: once the first one has read its operands K(t) and V(t - 1) are done with,
  // and K(t + 2) and V(t + 2) take their places, copy by copy between the second one's
  // products.  The barrier in every tile's first half, behind its last operands and before
  // the first ones of the next tile, keeps both apart: it lets no wave overwrite what
  // another one still reads, and shows what all of them wrote a tile before.  (Past the
  // last tile the copies are of it, into places that nobody reads any more.)
  uint32_t v_at = 4 * TILE;                    // V of tile t - 1
  auto keep_o = [&]() BM_LAMBDA {
    // (O stays in the accumulation registers over the loop)
#pragma unroll
    for (int rt = 0; rt < 2; ++rt)
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) asm volatile("" : "+a"(o[rt][mt]));
  };
  keep_o();
  for (int t = 0; t < t1 - t0; ++t) {
    step(std::integral_constant<int, 1>{}, [](auto) BM_LAMBDA {}, zb, za, pa, pb, 2 * (t0 + t));
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) ka[kk] ^= TILE;
    keep_o();
    const uint32_t v_new = v_at - 2 * TILE;
    const int next = v_at == 4 * TILE ? -2 * TILE : TILE;
    v_at += next;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) va[mt] += next;
    const Run run = run_of(min(t0 + t + 3, t1 - 1));
    step(std::integral_constant<int, 0>{},
         [&](auto jc) BM_LAMBDA {
           constexpr int j = decltype(jc)::value, EVERY = (2 * KK + 4 * MT) / 16, c = j / EVERY;
           if constexpr (j % EVERY == 0) {
             if constexpr (c < NCOPY) store_k(c, t);
             if constexpr (c >= NCOPY && c < 2 * NCOPY) store_v(c - NCOPY, v_new);
             if constexpr (c == 2 * NCOPY) {
               if (__builtin_expect(!run.is, 0)) load_mixed(ks, vs, min(t0 + t + 3, t1 - 1));
             }
             if constexpr (c >= 2 * NCOPY && c < 4 * NCOPY) {
               if (run.is) {
                 if constexpr (c < 3 * NCOPY) load_k(run, c - 2 * NCOPY);
                 else load_v(run, c - 3 * NCOPY);
               }
             }
           }
         },
         za, zb, pb, pa, 2 * (t0 + t) + 1);
    keep_o();
  }
  // the last half's values
#pragma unroll
  for (int q = 0; q < 2 * MT; ++q) {
    const uint32_t x = va[q % MT] + (32 + 16 * (q / MT)) * RB;
    const bf16v4 x0 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(lds_at<lds_bf16v4>(x));
    const bf16v4 x1 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(lds_at<lds_bf16v4>(x + 4 * RB));
    const u32x2 y0 = __builtin_bit_cast(u32x2, x0), y1 = __builtin_bit_cast(u32x2, x1);
#pragma unroll
    for (int rt = 0; rt < 2; ++rt)
      o[rt][q % MT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, u32x4{y0.x, y0.y, y1.x, y1.y}),
                                                              __builtin_bit_cast(bf16x8, pb[rt][q / MT]), o[rt][q % MT], 0, 0, 0);
  }
  if constexpr (SPLIT) {
#pragma unroll
    for (int rt = 0; rt < 2; ++rt) {
      const float sum = lanes::add_xor<32>(l[rt]);
      const int t = tw + 32 * rt + n;
      if (t >= a.n_tok) continue;
      const bool real = r0 + t >= 0;                       // (a pad token sees nothing)
      const int64_t at = part_row(a, u, G, w % G, t);
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const f32x16 x = o[rt][mt];
          *reinterpret_cast<f32x4*>(a.part + at * D + 32 * mt + 8 * i + 4 * h) =
              f32x4{x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]};
        }
      if (h == 0) put_sums(a, G, D, at, real ? m[rt] : kNegInf, real ? sum : 0.0f);
    }
    return;
  }
  __syncthreads();

  // ---- outputs, through the wave's part of LDS into whole rows ----
#pragma unroll
  for (int rt = 0; rt < 2; ++rt) {
    const float sum = lanes::add_xor<32>(l[rt]);
    // (a pad token sees nothing)
    const bool real = r0 + tw + 32 * rt + n >= 0;
    const float inv = real ? 1.0f / sum : 0.0f;
    char* ost = lds + w * (32 * RB);
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f32x16 x = o[rt][mt];
        const int d0 = 32 * mt + 8 * i + 4 * h;
        const u32x2 y = {pack2(x[4 * i] * inv, x[4 * i + 1] * inv), pack2(x[4 * i + 2] * inv, x[4 * i + 3] * inv)};
        *reinterpret_cast<u32x2*>(ost + n * RB + ((d0 * 2) ^ (16 * swz_k<RB>(n)))) = real ? y : u32x2{0, 0};
      }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int j = 0; j < 32 * CPR / 64; ++j) {
      const int r = j * (64 / CPR) + lane / CPR, c = lane % CPR, t = tw + 32 * rt + r;
      const u32x4 y = *reinterpret_cast<const u32x4*>(ost + r * RB + 16 * (c ^ swz_k<RB>(r)));
      if (t < a.n_tok) *reinterpret_cast<u32x4*>(static_cast<char*>(a.o) + (head * a.seq_ld + t) * RB + c * 16) = y;
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// ---- float32: 16 query rows a wave, operands straight from the rows ----
//
// A sixteenth of bfloat16's matrix rate (4096 cycles a tile of 32 keys at d = 128, where a
// wave loads 32 KB), so nothing is staged; 8 x 1024 tokens over a window of 1024 take 1.42 ms
// (97 of 154 TFLOP/s), with the L2 at 12 TB/s.  Lane (i, h) of a tile: S^T = K Q^T takes 16
// bytes of key row 16 s + i a step, contracting their four elements one after the other; a
// lane then holds 8 logits of row i, keys 16 t + 4 h + r, and O^T += V^T P^T takes the keys in
// that order: elements EPL i .. of V rows 16 t + 4 h + r, M-tile e standing for EPL i + e.
// Every wave has its own keys: its rows' sinks and window.
constexpr int kF32Rows = 16, kF32Tile = 32;

template <int D>
__global__ void __launch_bounds__(256, 2) window_prompt_f32_kernel(PromptArgs a, int blocks) {
  const bool split = a.nsplit > 1;             // blockIdx.y: one of the workgroups over the keys
  constexpr int RB = 4 * D, KL = D / 16, EPL = D / 16;
  const int group = a.n_heads / a.n_kv_heads;
  const int64_t wave = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, i16 = lane & 15, h = lane >> 4;
  if (wave >= (int64_t)a.units * group * blocks) return;
  // the heads of a unit next to each other: they share keys
  const int g = (int)(wave % group), blk = (int)(wave / group % blocks), u = (int)(wave / group / blocks);
  const int bi = u / a.n_kv_heads, hk = u - bi * a.n_kv_heads;
  const int64_t head = (int64_t)bi * a.n_heads + hk * group + g;
  const int pad = a.pad ? max(0, __builtin_amdgcn_readfirstlane(a.pad[bi])) : 0;
  const int r0 = index_of(a.t0, pad), tw = blk * kF32Rows, t_own = tw + i16;
  const int p1 = min(tw + kF32Rows, a.n_tok);
  float* o = static_cast<float*>(a.o) + (head * a.seq_ld + t_own) * D + 4 * EPL * h;
  const int first = max(r0 + tw, 0), last = r0 + p1 - 1;
  const int lo = max(0, first - a.window + 1), lead = min(a.sinks, lo), shift = lo - lead;
  const int nv = lead + last - lo + 1, nt = (nv + kF32Tile - 1) / kF32Tile;
  const int64_t at = split ? part_row(a, u, group, g, t_own) : 0;
  if (split) o = a.part + at * D + 4 * EPL * h;
  const int per = (nt + a.nsplit - 1) / a.nsplit, t0 = min((int)blockIdx.y * per, nt), t1 = min(t0 + per, nt);
  if (last < 0 || t0 == t1) {
    // pad tokens alone, or no keys left
    if (t_own < a.n_tok) {
      for (int e = 0; e < 4 * EPL; e += 4) *reinterpret_cast<f32x4*>(o + e) = f32x4{0, 0, 0, 0};
      if (split && h == 0) put_sums(a, group, D, at, kNegInf, 0.0f);
    }
    return;
  }
  const int ring0 = max(lo, a.sinks) - a.sinks;
  const int place0 = ring0 % a.window - (ring0 + a.sinks - shift);
  const char* kc = static_cast<const char*>(a.kc) + (int64_t)u * (a.window + a.sinks) * RB;
  const char* vc = static_cast<const char*>(a.vc) + (int64_t)u * (a.window + a.sinks) * RB;
  const char* ki = static_cast<const char*>(a.kin) + (int64_t)u * a.seq_ld * RB;
  const char* vi = static_cast<const char*>(a.vin) + (int64_t)u * a.seq_ld * RB;
  // the row of key number v (past the last one: the last)
  auto row_of = [&](int v, const char* cached, const char* input) BM_LAMBDA {
    v = min(v, nv - 1);
    const int j = v < lead ? v : v + shift;
    int slot = place0 + v;
    slot = j < a.sinks ? j : a.sinks + (slot >= a.window ? slot - a.window : slot);
    return j < r0 ? cached + (int64_t)slot * RB : input + (int64_t)(j - r0) * RB;
  };
  f32x4 kf[2][KL], vf[8][EPL / 4], qf[KL];
  auto load_k = [&](int t) BM_LAMBDA {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const char* p = row_of(t * kF32Tile + 16 * s + i16, kc, ki) + 16 * h;
#pragma unroll
      for (int kk = 0; kk < KL; ++kk) kf[s][kk] = *reinterpret_cast<const f32x4*>(p + 64 * kk);
    }
  };
  auto load_v = [&](int t) BM_LAMBDA {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const char* p = row_of(t * kF32Tile + 16 * (i >> 2) + 4 * h + (i & 3), vc, vi) + i16 * (4 * EPL);
#pragma unroll
      for (int e = 0; e < EPL / 4; ++e) vf[i][e] = *reinterpret_cast<const f32x4*>(p + 16 * e);
    }
  };
  load_k(t0);
  load_v(t0);
  {
    const char* q = static_cast<const char*>(a.q) + (head * a.seq_ld + min(t_own, a.n_tok - 1)) * RB + 16 * h;
#pragma unroll
    for (int kk = 0; kk < KL; ++kk) qf[kk] = *reinterpret_cast<const f32x4*>(q + 64 * kk);
  }
  const int vhi = max(min(r0 + t_own, last), first) - shift;      // what the lane's row sees
  const int wfirst = first - shift, wlast = last - shift;
  f32x4 acc[EPL];
  float m = kNegInf, l = 0.0f;
#pragma unroll
  for (int e = 0; e < EPL; ++e) acc[e] = f32x4{0, 0, 0, 0};
  const float c2 = a.scale_log2;
  for (int t = t0; t < t1; ++t) {
    f32x4 s[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
#pragma unroll
    for (int kk = 0; kk < KL; ++kk)
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int x = 0; x < 2; ++x)
          s[x] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[x][kk][j], qf[kk][j], s[x], 0, 0, 0);
    load_k(t + 1);
    const int v0 = t * kF32Tile;
    if (!(v0 + 31 <= wfirst && (v0 + 31 < a.sinks || v0 > wlast - a.window))) {
      auto below = [](int x) BM_LAMBDA { return x <= 0 ? 0u : x >= 32 ? ~0u : (1u << x) - 1; };   // keys < x
      const uint32_t seen = below(vhi + 1 - v0) & (~below(vhi + 1 - a.window - v0) | below(a.sinks - v0));
#pragma unroll
      for (int i = 0; i < 8; ++i)
        s[i >> 2][i & 3] = (seen >> (16 * (i >> 2) + 4 * h + (i & 3))) & 1 ? s[i >> 2][i & 3] : kNegInf;
    }
    float top = kNegInf;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = fmaxf(top, s[i >> 2][i & 3]);
    if (__ballot(top * c2 > m + kRescaleLog2) != 0) {
      float x = lanes::max_xor16_32(top) * c2;
      const float mn = fmaxf(m, x), f = mn == kNegInf ? 1.0f : __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      l *= f;
#pragma unroll
      for (int e = 0; e < EPL; ++e) acc[e] *= f;
    }
    const float ref = m == kNegInf ? 0.0f : m;
    float p[8], sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      p[i] = __builtin_amdgcn_exp2f(fmaf(s[i >> 2][i & 3], c2, -ref));
      sum += p[i];
    }
    l += sum;
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int e = 0; e < EPL; ++e)
        acc[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[i][e / 4][e % 4], p[i], acc[e], 0, 0, 0);
    load_v(t + 1);
  }
  if (t_own >= a.n_tok) return;
  l = lanes::add_xor<32>(lanes::add_xor<16>(l));
  const bool real = r0 + t_own >= 0;                              // (a pad token sees nothing)
  const float inv = split ? 1.0f : 1.0f / l;
  if (split && h == 0) put_sums(a, group, D, at, real ? m : kNegInf, real ? l : 0.0f);
#pragma unroll
  for (int x = 0; x < 4; ++x)
#pragma unroll
    for (int e = 0; e < EPL; e += 4) {
      const f32x4 y = {acc[e][x] * inv, acc[e + 1][x] * inv, acc[e + 2][x] * inv, acc[e + 3][x] * inv};
      *reinterpret_cast<f32x4*>(o + EPL * x + e) = real ? y : f32x4{0, 0, 0, 0};
    }
}

// Rows of the tokens that the cache keeps, 16 bytes a thread: token t of the call's last
// min(n_tok, window), and the sinks among the others.  Grid (units, chunks of rows).
template <int RB>
__global__ void __launch_bounds__(256) window_store_kernel(PromptArgs a, int rows) {
  constexpr int CPR = RB / 16;
  const int u = blockIdx.x;
  const int pad = a.pad ? max(0, a.pad[u / a.n_kv_heads]) : 0;
  const int c = blockIdx.y * 256 + threadIdx.x;
  const int r = c / CPR, ch = c % CPR;
  if (r >= rows) return;
  const int kept = min(a.n_tok, a.window), r0 = index_of(a.t0, pad);
  const int t = kept_token(r, rows - kept, a.n_tok, a.window, a.sinks, r0);
  if (t < 0) return;
  const int i = r0 + t;
  const int64_t src = ((int64_t)u * a.seq_ld + t) * RB + ch * 16;
  const int64_t dst =
      ((int64_t)u * (a.window + a.sinks) + window_slot(i, a.sinks, a.window)) * RB + ch * 16;
  *reinterpret_cast<uint4*>(static_cast<char*>(a.kc) + dst) =
      *reinterpret_cast<const uint4*>(static_cast<const char*>(a.kin) + src);
  *reinterpret_cast<uint4*>(static_cast<char*>(a.vc) + dst) =
      *reinterpret_cast<const uint4*>(static_cast<const char*>(a.vin) + src);
}

template <int RB>
hipError_t launch_store(const PromptArgs& a, hipStream_t stream) {
  const int kept = a.n_tok < a.window ? a.n_tok : a.window;
  const int lead = a.sinks < a.n_tok - kept ? a.sinks : a.n_tok - kept;
  const unsigned chunks = (unsigned)(((int64_t)(kept + lead) * (RB / 16) + 255) / 256);
  hipLaunchKernelGGL((window_store_kernel<RB>), dim3((unsigned)a.units, chunks), dim3(256), 0, stream, a,
                     kept + lead);
  return hipGetLastError();
}

// A launch of fewer workgroups than compute units gives each row block's keys to several, as
// many as the measured times of their work make worth it: 1.9 us a tile of 64 keys, 2.7 us
// one of 32 in float32, against 5 us for a join and 14 (4) us for the parts of 256
// workgroups.  us without -> with, samples x tokens of 8 KV heads, four query heads each,
// d = 128:
//   window  1 x 128      1 x 512      2 x 256      8 x 256      float32, 1 x 128
//   512     31 -> 25     32 -> 32     32 -> 32     39 -> 39     54 -> 28
//   1024    45 -> 29     45 -> 41     47 -> 41     56 -> 56     96 -> 39
//   4096    132 -> 37    138 -> 61    143 -> 61    164 -> 152   351 -> 102
constexpr int kPromptWorkgroups = 256, kMaxPromptSplits = 64;
int most_prompt_splits(int64_t workgroups) {
  const int64_t s = kPromptWorkgroups / workgroups;
  return s < 1 ? 1 : s > kMaxPromptSplits ? kMaxPromptSplits : (int)s;
}
int prompt_splits(int64_t workgroups, int tiles, bool bf16) {
  // tenths of us
  const int most = most_prompt_splits(workgroups), tile = bf16 ? 19 : 27, parts = bf16 ? 140 : 40;
  int best = 1, least = tiles * tile;
  for (int s = 2; s <= most; ++s) {
    const int cost = (tiles + s - 1) / s * tile + 50 + (int)(parts * workgroups * s / kPromptWorkgroups);
    if (cost < least) {
      best = s;
      least = cost;
    }
  }
  return best;
}
// tokens of a row block, and workgroups
int block_tokens(bool bf16, int group) { return bf16 ? kPromptWaves * kPromptRows / group : kF32Rows; }
int64_t prompt_workgroups(int units, int group, int n_tok, bool bf16) {
  const int pt = block_tokens(bf16, group);
  const int64_t blocks = ((int64_t)n_tok + pt - 1) / pt;
  return bf16 ? units * blocks : (units * group * blocks + 3) / 4;
}

// behind the workgroups: the join of their parts, the rows to store
hipError_t finish(const PromptArgs& a, int dtype, int head_dim, hipStream_t stream) {
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (a.nsplit > 1) {
    NodesArgs n{};
    n.o = a.o;
    n.part = a.part;
    n.seq_ld = a.seq_ld;
    n.n_heads = a.n_heads;
    n.n_kv_heads = a.n_kv_heads;
    n.units = a.units;
    n.n = a.n_tok;
    n.nsplit = a.nsplit;
    e = launch_nodes_join(n, dtype, head_dim, stream);
    if (e != hipSuccess) return e;
  }
  const int rb = head_dim * (dtype == BM_BF16 ? 2 : 4);
  return rb == 128 ? launch_store<128>(a, stream) : rb == 256 ? launch_store<256>(a, stream) : launch_store<512>(a, stream);
}

template <int D, int G>
hipError_t launch_bf16(const PromptArgs& a, hipStream_t stream) {
  const int tiles = (int)prompt_workgroups(1, G, a.n_tok, true);
  const dim3 grid((unsigned)(a.units * tiles), (unsigned)a.nsplit);
  if (a.nsplit > 1)
    hipLaunchKernelGGL((window_prompt_kernel<D, G, true>), grid, dim3(64 * kPromptWaves), 0, stream, a, tiles);
  else
    hipLaunchKernelGGL((window_prompt_kernel<D, G, false>), grid, dim3(64 * kPromptWaves), 0, stream, a, tiles);
  return finish(a, BM_BF16, D, stream);
}

template <int D>
hipError_t launch_f32(const PromptArgs& a, int group, hipStream_t stream) {
  hipLaunchKernelGGL((window_prompt_f32_kernel<D>),
                     dim3((unsigned)prompt_workgroups(a.units, group, a.n_tok, false), (unsigned)a.nsplit), dim3(256), 0,
                     stream, a, (a.n_tok + kF32Rows - 1) / kF32Rows);
  return finish(a, BM_F32, D, stream);
}

template <int D>
hipError_t launch_d(const PromptArgs& a, int dtype, int group, hipStream_t stream) {
  if (dtype == BM_F32) return launch_f32<D>(a, group, stream);
  switch (group) {
    case 1: return launch_bf16<D, 1>(a, stream);
    case 2: return launch_bf16<D, 2>(a, stream);
    case 4: return launch_bf16<D, 4>(a, stream);
    default: return hipErrorInvalidValue;
  }
}

// A few tokens are the nodes of a chain: their waves have fewer rows, and take keys each.  us
// as nodes and as a prompt, samples x tokens of 8 KV heads, four query heads each, d = 128,
// over a window of 4096: bfloat16 1 x 16 22 and 24, 32 x 16 107 and 181, 1 x 32 28 and 26,
// 32 x 32 144 and 183, 1 x 64 35 and 32, 32 x 64 267 and 192; float32 8 x 8 64 and 110,
// 32 x 16 389 and 392, 32 x 32 761 and 712.
bool is_short(const PromptArgs& a, int dtype, int group) {
  return a.n_tok <= kShortPrompt && a.n_tok * group <= (dtype == BM_BF16 ? 128 : 64);
}

}  // namespace

bool prompt_fits(int units, int group, int n_tok) {
  return (int64_t)units * group * n_tok / 4 < 0x7FFFFFFF;
}

size_t prompt_work_bytes(int units, int head_dim, int group, int n, bool bf16) {
  size_t most = nodes_work_bytes(units, head_dim, group, n < kShortPrompt ? n : kShortPrompt);
  // (every number of row blocks that is split; the last block full, or what n has of it)
  const int pt = block_tokens(bf16, group);
  for (int64_t t = pt;; t += pt) {
    const int tokens = (int)(t < n ? t : n), s = most_prompt_splits(prompt_workgroups(units, group, tokens, bf16));
    if (s == 1) break;
    const size_t bytes = (size_t)units * group * tokens * s * (head_dim + 2) * sizeof(float);
    if (bytes > most) most = bytes;
    if (t >= n) break;
  }
  return most;
}

hipError_t launch_prompt(PromptArgs a, int dtype, int head_dim, int group, hipStream_t stream) {
  if (is_short(a, dtype, group)) {
    NodesArgs n{};
    n.q = a.q;
    n.kin = a.kin;
    n.vin = a.vin;
    n.o = a.o;
    n.kc = a.kc;
    n.vc = a.vc;
    n.pad = a.pad;
    n.part = a.part;
    n.seq_ld = a.seq_ld;
    n.n_heads = a.n_heads;
    n.n_kv_heads = a.n_kv_heads;
    n.units = a.units;
    n.slots = a.window + a.sinks;
    n.len0 = a.t0 < n.slots ? a.t0 : n.slots;
    n.n = a.n_tok;
    n.next_pos = a.t0;
    n.window = a.window;
    n.sinks = a.sinks;
    n.chain = 1;
    n.store = a.n_tok == 1;
    n.scale_log2 = a.scale_log2;
    const hipError_t e = launch_nodes(n, dtype, head_dim, group, stream);
    if (e != hipSuccess || n.store) return e;
    a.nsplit = 1;
    return finish(a, dtype, head_dim, stream);
  }
  const bool bf16 = dtype == BM_BF16;
  // (a row block sees the sinks, the window before it and itself, and no more than there is)
  const int64_t end = (int64_t)a.t0 + a.n_tok, seen = (int64_t)a.sinks + a.window + block_tokens(bf16, group);
  const int tile = bf16 ? kPromptTile : kF32Tile;
  a.nsplit = prompt_splits(prompt_workgroups(a.units, group, a.n_tok, bf16), (int)(((end < seen ? end : seen) + tile - 1) / tile), bf16);
  return head_dim == 128 ? launch_d<128>(a, dtype, group, stream) : launch_d<64>(a, dtype, group, stream);
}

}  // namespace bm
