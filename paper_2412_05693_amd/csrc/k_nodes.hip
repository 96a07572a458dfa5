// The nodes of a tree of drafted tokens (or one generated token) over a cache: a bounded
// one or a window cache (bm_draft.h, bm_window.h).
//
// A unit's rows are its G n (query head, node) pairs.  Every row is an online softmax over
// the cached entries and over the nodes: a running maximum m (log2 units), the sum l of
// exp2(z - m), and o = sum exp2(z - m) v; parts of the keys are joined by
// o = sum_c 2^(m_c - M) o_c / sum_c 2^(m_c - M) l_c with M the largest m_c.
//
// A wave works on 16 RT rows and on tiles of 32 keys, and needs no LDS for it:
//   S^T = K Q^T  (16 x 16 MFMA tiles, keys x rows): lane (i, h) loads 16 bytes of key row i
//                a step, a row's chunk 4 kk + h in step kk; Q lies in registers alike.
//   a lane then holds 8 logits of one row, keys 16 t + 4 h + r (t < 2, r < 4), which is the
//   layout that P^T has to have as the next product's operand if that one takes its keys in
//   the order (t, r) within lane quarter h:
//   O^T += V^T P^T: lane (i, h) loads elements EPL i .. of V's rows 16 t + 4 h + r (whole
//                rows a wave load) and, for bfloat16, transposes its 8 x EPL block with byte
//                permutes.  M-tile e then stands for the elements EPL i + e.
// bfloat16 weights go in two parts, the nearest bfloat16 and that of the rest (2^-16 in
// all), so the outputs carry little more than their own rounding.
//
// The workgroup's waves share the rows (up to 8 blocks of them) and then the key tiles; waves
// over the same rows join through LDS, workgroups over the same unit through the workspace
// and a second launch.
#include <type_traits>

#include "bm_internal.h"
#include "bm_lanes.h"
#include "bm_window_dev.h"

// a lambda of the kernel, always part of it
#define BM_LAMBDA __device__ __attribute__((always_inline))

namespace bm {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;

constexpr float kNegInf = -__builtin_huge_valf();
constexpr float kRescaleLog2 = 8.0f;   // the maximum moves once a logit is 2^8 beyond it
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kTile = 32;              // keys
constexpr int kNodeWaves = 8;
constexpr int kMaxNodeSplits = 64;     // a lane of the joining wave each
constexpr int kNoWindow = 0x7FFFFFFF;

template <bool BF16, int D>
struct NodeCfg {
  using E = typename std::conditional<BF16, uint16_t, float>::type;
  static constexpr int RB = D * (int)sizeof(E);        // bytes of a row
  static constexpr int KL = RB / 64;                   // 16-byte loads of a lane a key row
  static constexpr int EPL = D / 16;                   // elements of a lane a V row
  static constexpr int VW = EPL * (int)sizeof(E) / 4;  // ... and words
};

__device__ __forceinline__ float xmax4(float x) {   // over the lanes 16 apart
  uint32_t y = __float_as_uint(x);
  const auto a = __builtin_amdgcn_permlane16_swap(y, y, false, false);
  y = __float_as_uint(fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1])));
  const auto b = __builtin_amdgcn_permlane32_swap(y, y, false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float xsum4(float x) { return lanes::add_xor<32>(lanes::add_xor<16>(x)); }

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  bf16x2 r = {(__bf16)lo, (__bf16)hi};
  return __builtin_bit_cast(uint32_t, r);
}

// a buffer of whole rows: reads behind its end give zeros
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_of(const void* p, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, bytes, 0x00020000);
}

// What the tree is to one wave: lane a stands for node a.
struct Tree {
  uint64_t sees;   // the nodes that node a sees, itself included
  int depth;
};

__device__ __forceinline__ uint64_t shfl64(uint64_t x, int lane) {
  const uint32_t lo = __shfl((uint32_t)x, lane), hi = __shfl((uint32_t)(x >> 32), lane);
  return (uint64_t)hi << 32 | lo;
}

// Ancestors by doubling the step up the tree; then the nodes that a window or a left pad
// hides (r0: the index of a root, below 0 where the sample has not begun).
__device__ __forceinline__ Tree make_tree(const int32_t* parent, int n, int r0, int sinks, int window) {
  const int a = threadIdx.x & 63;
  int up = -1;
  if (parent && a < n) {
    up = parent[a];
    if (up < 0 || up >= a) up = -1;
  }
  Tree t;
  t.sees = 1ull << a;
  while (__ballot(up >= 0) != 0) {
    const uint64_t more = shfl64(t.sees, max(up, 0));
    const int next = __shfl(up, max(up, 0));
    if (up >= 0) {
      t.sees |= more;
      up = next;
    }
  }
  t.depth = __popcll(t.sees) - 1;
  if (r0 < 0 || __ballot(t.depth >= window) != 0) {
    for (int c = 0; c < n; ++c) {
      const int dc = __shfl(t.depth, c), j = r0 + dc;
      if (j < 0 || (j >= sinks && t.depth - dc >= window)) t.sees &= ~(1ull << c);
    }
  }
  return t;
}

// Work of a launch over the waves: rows of 16 RT, and what is left over the keys.
struct NodePlan {
  int rt;          // row tiles of a wave
  int row_waves;   // waves of a workgroup over different rows
  int row_groups;  // workgroups over different rows of a unit
  int key_waves() const { return kNodeWaves / row_waves; }
};

NodePlan plan_of(int rows, bool bf16) {
  NodePlan p;
  p.rt = bf16 && rows > 16 ? 2 : 1;
  const int blocks = (rows + 16 * p.rt - 1) / (16 * p.rt);
  p.row_waves = 1;
  while (p.row_waves < blocks && p.row_waves < kNodeWaves) p.row_waves *= 2;
  p.row_groups = (blocks + p.row_waves - 1) / p.row_waves;
  return p;
}

template <bool BF16, int D, int RT>
__global__ void __launch_bounds__(64 * kNodeWaves, 1) nodes_kernel(NodesArgs a, int row_waves) {
  using C = NodeCfg<BF16, D>;
  using E = typename C::E;
  constexpr int RB = C::RB, KL = C::KL, EPL = C::EPL, VW = C::VW;
  constexpr int OREGS = 4 * EPL;                       // output values of a lane and row tile
  // joins: half of the waves hand over O, m and l; rows of a wave's weights (see patch)
  constexpr int JOIN = RT * (OREGS + 2) * 64;
  __shared__ float lds[(kNodeWaves / 2) * JOIN > kNodeWaves * 512 * RT ? (kNodeWaves / 2) * JOIN
                                                                     : kNodeWaves * 512 * RT];
  const int group = a.n_heads / a.n_kv_heads, rows = group * a.n;
  const int u = blockIdx.x, split = blockIdx.y;
  const int bi = u / a.n_kv_heads, hk = u - bi * a.n_kv_heads;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int i16 = lane & 15, h = lane >> 4;
  const int key_waves = kNodeWaves / row_waves, rw = wave / key_waves, kw = wave - rw * key_waves;
  const int row0 = ((int)blockIdx.z * row_waves + rw) * 16 * RT;     // the wave's first row
  const int pad = a.pad ? max(0, __builtin_amdgcn_readfirstlane(a.pad[bi])) : 0;
  const int r0 = a.next_pos - pad;                                   // a root's index
  const Ring ring(r0, a.sinks, max(a.window, 1));
  const int entries = a.window ? ring.filled() : a.len0;

  // ---- the workgroup's tiles: its share of the cached ones and, in the last share, the nodes' ----
  const int tiles = (entries + kTile - 1) / kTile;
  const int per = (tiles + a.nsplit - 1) / a.nsplit;
  const int lo = min(split * per, tiles), cached = min(tiles - lo, per);
  const int total = cached + (split == a.nsplit - 1 ? (a.n + kTile - 1) / kTile : 0);

  const char* kc = static_cast<const char*>(a.kc) + (int64_t)u * a.slots * RB;
  const char* vc = static_cast<const char*>(a.vc) + (int64_t)u * a.slots * RB;
  const char* kin = static_cast<const char*>(a.kin) + (int64_t)u * a.seq_ld * RB;
  const char* vin = static_cast<const char*>(a.vin) + (int64_t)u * a.seq_ld * RB;
  const int32_t* pos = a.window ? nullptr : a.pos + (int64_t)u * a.slots;

  u32x4 kf[2][KL];
  uint32_t vf[8][VW];
  int pk = 0;           // the position of key (lane & 31) of the tile (left padding)
  auto load_k = [&](int t) BM_LAMBDA {
    const bool node = t >= cached;
    const int base = (node ? t - cached : lo + t) * kTile;
    const auto r = rows_of(node ? kin : kc, (node ? a.n : entries) * RB);
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int kk = 0; kk < KL; ++kk)
        kf[s][kk] = __builtin_amdgcn_raw_buffer_load_b128(r, (base + 16 * s + i16) * RB + 16 * h + 64 * kk, 0, 0);
    if (pos && pad > 0 && !node) pk = pos[min(base + (lane & 31), entries - 1)];
  };
  auto load_v = [&](int t) BM_LAMBDA {
    const bool node = t >= cached;
    const int base = (node ? t - cached : lo + t) * kTile;
    const auto r = rows_of(node ? vin : vc, (node ? a.n : entries) * RB);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int off = (base + 16 * (i >> 2) + 4 * h + (i & 3)) * RB + i16 * (4 * VW);
      if constexpr (VW == 2) {
        const u32x2 x = __builtin_amdgcn_raw_buffer_load_b64(r, off, 0, 0);
        vf[i][0] = x.x;
        vf[i][1] = x.y;
      } else {
#pragma unroll
        for (int w = 0; w < VW; w += 4) {
          const u32x4 x = __builtin_amdgcn_raw_buffer_load_b128(r, off + 4 * w, 0, 0);
          vf[i][w] = x.x;
          vf[i][w + 1] = x.y;
          vf[i][w + 2] = x.z;
          vf[i][w + 3] = x.w;
        }
      }
    }
  };
  load_k(kw);
  load_v(kw);

  // ---- the rows' queries, and what the tree shows them ----
  u32x4 qf[RT][KL];
  int row[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    row[rt] = row0 + 16 * rt + i16;
    const int x = min(row[rt], rows - 1), g = x / a.n, node = x - g * a.n;
    const char* q = static_cast<const char*>(a.q) +
                    (((int64_t)bi * a.n_heads + hk * group + g) * a.seq_ld + node) * RB;
#pragma unroll
    for (int kk = 0; kk < KL; ++kk)
      qf[rt][kk] = *reinterpret_cast<const u32x4*>(q + 16 * h + 64 * kk);
  }
  const Tree tree = make_tree(a.parent ? a.parent + (int64_t)bi * a.n : nullptr, a.n, r0, a.sinks,
                              a.window ? a.window : kNoWindow);
  uint64_t sees[RT];
  int depth[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int node = min(row[rt], rows - 1) % a.n;
    sees[rt] = shfl64(tree.sees, node);
    depth[rt] = __shfl(tree.depth, node);
  }
  // entries that the window hides from the deepest node: those of index <= edge
  const bool nested = __ballot((threadIdx.x & 63) < a.n && tree.depth > 0) != 0;
  int deepest = 0;
  if (a.window) {
    deepest = (threadIdx.x & 63) < a.n ? tree.depth : 0;
#pragma unroll
    for (int off = 32; off; off >>= 1) deepest = max(deepest, __shfl_xor(deepest, off));
  }

  if (a.store && split == 0 && blockIdx.z == 0 && r0 >= 0) {
    // the token's own rows into its slot, which nobody sees in this call
    constexpr int CPR = RB / 16;
    if (threadIdx.x < 2 * CPR) {
      const bool v = threadIdx.x >= CPR;
      const int c = (threadIdx.x - (v ? CPR : 0)) * 16;
      char* dst = static_cast<char*>(v ? a.vc : a.kc) +
                  ((int64_t)u * a.slots + window_slot(r0, a.sinks, a.window)) * RB + c;
      *reinterpret_cast<u32x4*>(dst) = *reinterpret_cast<const u32x4*>((v ? vin : kin) + c);
    }
  }

  f32x4 acc[RT][EPL];
  float m[RT], l[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    m[rt] = kNegInf;
    l[rt] = 0.0f;
#pragma unroll
    for (int e = 0; e < EPL; ++e) acc[rt][e] = f32x4{0, 0, 0, 0};
  }
  const float c2 = a.scale_log2;

  for (int t = kw; t < total; t += key_waves) {
    const bool node = t >= cached;
    const int base = (node ? t - cached : lo + t) * kTile;
    // ---- logits ----
    f32x4 s[RT][2];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
      for (int x = 0; x < 2; ++x) s[rt][x] = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int kk = 0; kk < KL; ++kk)
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          if constexpr (BF16) {
            s[rt][x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf[x][kk]),
                                                               __builtin_bit_cast(bf16x8, qf[rt][kk]), s[rt][x], 0, 0, 0);
          } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
              s[rt][x] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kf[x][kk][j]),
                                                              __uint_as_float(qf[rt][kk][j]), s[rt][x], 0, 0, 0);
          }
        }

    // ---- who sees what.  Keys that nobody sees: bit k of `gone`; keys that some rows see
    //      and others do not (`mixed`): dist, their index less that of the oldest one a
    //      root does not see, against the row's depth, or the tree's bits ----
    uint32_t gone = 0;
    bool mixed = node;
    int dist[8];
    if (!node) {
      const int k32 = lane & 31, slot = base + k32;
      bool out = slot >= entries;
      if (pos && pad > 0) out = out || pk < pad;
      if (a.window) {
        const int j = ring.index(min(slot, a.slots - 1));
        const bool old = slot >= a.sinks && j - (r0 - a.window) <= deepest;
        if (nested)
          mixed = __ballot(old && !out) != 0;
        else
          out = out || old;
      }
      gone = (uint32_t)__ballot(out);
      if (mixed) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int sl = base + 16 * (i >> 2) + 4 * h + (i & 3);
          dist[i] = sl < a.sinks ? kNoWindow : ring.index(min(sl, a.slots - 1)) - (r0 - a.window);
        }
      }
    } else {
      gone = base + kTile > a.n ? ~0u << (a.n - base) : 0;
    }
    const uint32_t hide = gone >> (4 * h);               // bit 16 t + r: this lane's key (t, r)
    uint32_t mask[RT];                                   // ... as each row sees it
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      mask[rt] = hide;
      if (mixed) {
        if (node) {
          mask[rt] |= (uint32_t)~(sees[rt] >> base) >> (4 * h);
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (dist[i] <= depth[rt]) mask[rt] |= 1u << (16 * (i >> 2) + (i & 3));
        }
      }
    }

    // (float32 rows of 128: K and V together leave no registers to load ahead)
    constexpr bool kAhead = BF16 || D == 64;
    if constexpr (kAhead) load_k(t + key_waves);

    // ---- softmax ----
    uint32_t phi[RT][4], plo[RT][4];                     // bfloat16 weights, two parts
    float pw[RT][8];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      float z[8], top = kNegInf;
#pragma unroll
      for (int i = 0; i < 8; ++i) z[i] = s[rt][i >> 2][i & 3];
      if (gone != 0 || mixed) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if ((mask[rt] >> (16 * (i >> 2) + (i & 3))) & 1) z[i] = kNegInf;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) top = fmaxf(top, z[i]);
      if (__ballot(top * c2 > m[rt] + kRescaleLog2) != 0) {
        const float mn = fmaxf(m[rt], xmax4(top) * c2);
        // (a row that has seen no key yet: nothing to scale)
        const float f = mn == kNegInf ? 1.0f : __builtin_amdgcn_exp2f(m[rt] - mn);
        m[rt] = mn;
        l[rt] *= f;
#pragma unroll
        for (int e = 0; e < EPL; ++e) acc[rt][e] *= f;
      }
      const float ref = m[rt] == kNegInf ? 0.0f : m[rt];
      float sum = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        pw[rt][i] = __builtin_amdgcn_exp2f(fmaf(z[i], c2, -ref));
        sum += pw[rt][i];
      }
      l[rt] += sum;
      if constexpr (BF16) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t hi = pack2(pw[rt][2 * i], pw[rt][2 * i + 1]);
          phi[rt][i] = hi;
          plo[rt][i] = pack2(pw[rt][2 * i] - __uint_as_float(hi << 16),
                             pw[rt][2 * i + 1] - __uint_as_float(hi & 0xFFFF0000u));
        }
      }
    }

    // ---- V rows that weigh nothing for a row must not reach it, NaN and infinities
    //      included: those nobody sees become zeros; where rows differ, a row with such a
    //      value becomes zeros too and is added to the rows that see it one by one ----
    uint32_t bad = 0;
    if (gone != 0) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const bool z = (hide >> (16 * (i >> 2) + (i & 3))) & 1;
#pragma unroll
        for (int w = 0; w < VW; ++w) vf[i][w] = z ? 0u : vf[i][w];
      }
    }
    if (mixed) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        bool b = false;
#pragma unroll
        for (int w = 0; w < VW; ++w) {
          const uint32_t x = vf[i][w];
          if constexpr (BF16)
            b = b || (x & 0x7F80u) == 0x7F80u || (x & 0x7F800000u) == 0x7F800000u;
          else
            b = b || (x & 0x7F800000u) == 0x7F800000u;
        }
        const uint64_t any = __ballot(b);
        if (any != 0) {
#pragma unroll
          for (int q = 0; q < 4; ++q)
            if ((any >> (16 * q)) & 0xFFFF) bad |= 1u << (16 * (i >> 2) + 4 * q + (i & 3));
          const bool z = (any >> (16 * h)) & 0xFFFF;
#pragma unroll
          for (int w = 0; w < VW; ++w) vf[i][w] = z ? 0u : vf[i][w];
        }
      }
    }

    // ---- O^T += V^T P^T ----
    if constexpr (BF16) {
      u32x4 vt[EPL];
#pragma unroll
      for (int w = 0; w < VW; ++w)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          vt[2 * w][j] = __builtin_amdgcn_perm(vf[2 * j + 1][w], vf[2 * j][w], 0x05040100);
          vt[2 * w + 1][j] = __builtin_amdgcn_perm(vf[2 * j + 1][w], vf[2 * j][w], 0x07060302);
        }
      load_v(t + key_waves);
#pragma unroll
      for (int e = 0; e < EPL; ++e)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          const bf16x8 v8 = __builtin_bit_cast(bf16x8, vt[e]);
          const u32x4 ph = {phi[rt][0], phi[rt][1], phi[rt][2], phi[rt][3]};
          const u32x4 pl = {plo[rt][0], plo[rt][1], plo[rt][2], plo[rt][3]};
          acc[rt][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v8, __builtin_bit_cast(bf16x8, ph), acc[rt][e], 0, 0, 0);
          acc[rt][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v8, __builtin_bit_cast(bf16x8, pl), acc[rt][e], 0, 0, 0);
        }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < EPL; ++e)
#pragma unroll
          for (int rt = 0; rt < RT; ++rt)
            acc[rt][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vf[i][e]), pw[rt][i], acc[rt][e], 0, 0, 0);
      load_v(t + key_waves);
    }

    // ---- the rows taken out above, for those that see them ----
    if (bad != 0) {
      float* w = lds + wave * 512 * RT;                  // weights [RT][32 keys][16 rows], < 0: hidden
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int key = 16 * (i >> 2) + 4 * h + (i & 3);
          w[(rt * 32 + key) * 16 + i16] = (mask[rt] >> (16 * (i >> 2) + (i & 3))) & 1 ? -1.0f : pw[rt][i];
        }
      // (a wave's own LDS writes are in order with its reads)
      __builtin_amdgcn_wave_barrier();
      const E* src = reinterpret_cast<const E*>(node ? vin : vc);
      for (uint32_t left = bad; left != 0; left &= left - 1) {
        const int key = __builtin_ctz(left);
        const E* v = src + (int64_t)(base + key) * D + 4 * EPL * h;
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          const float p = w[(rt * 32 + key) * 16 + i16];
          if (p >= 0.0f) {
#pragma unroll
            for (int x = 0; x < 4; ++x)
#pragma unroll
              for (int e = 0; e < EPL; ++e) {
                float f;
                if constexpr (BF16) f = __uint_as_float((uint32_t)v[EPL * x + e] << 16);
                else f = v[EPL * x + e];
                acc[rt][e][x] += p * f;
              }
          }
        }
      }
      __builtin_amdgcn_wave_barrier();
    }
    if constexpr (!kAhead) load_k(t + key_waves);
  }
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) l[rt] = xsum4(l[rt]);

  // ---- join the waves over the same rows, half of them handing over at a time ----
  for (int half = key_waves >> 1; half > 0; half >>= 1) {
    __syncthreads();
    float* x = lds + (rw * half + (kw & (half - 1))) * JOIN + lane;
    if (kw >= half && kw < 2 * half) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        float* y = x + rt * (OREGS + 2) * 64;
#pragma unroll
        for (int i = 0; i < OREGS; ++i) y[i * 64] = acc[rt][i >> 2][i & 3];
        y[OREGS * 64] = m[rt];
        y[(OREGS + 1) * 64] = l[rt];
      }
    }
    __syncthreads();
    if (kw < half) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        const float* y = x + rt * (OREGS + 2) * 64;
        const float mo = y[OREGS * 64], mn = fmaxf(m[rt], mo);
        const float f = m[rt] == kNegInf ? 0.0f : __builtin_amdgcn_exp2f(m[rt] - mn);
        const float fo = mo == kNegInf ? 0.0f : __builtin_amdgcn_exp2f(mo - mn);
        m[rt] = mn;
        l[rt] = l[rt] * f + y[(OREGS + 1) * 64] * fo;
#pragma unroll
        for (int i = 0; i < OREGS; ++i) acc[rt][i >> 2][i & 3] = acc[rt][i >> 2][i & 3] * f + y[i * 64] * fo;
      }
    }
  }
  if (kw != 0) return;

  // ---- results: lane (i16, h) holds elements 4 EPL h .. of row i16 ----
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    if (row[rt] >= rows) continue;
    if (a.nsplit > 1) {
      const int64_t at = ((int64_t)u * a.nsplit + split) * rows + row[rt];
      float* o = a.part + at * D + 4 * EPL * h;
#pragma unroll
      for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int e = 0; e < EPL; e += 4)
          *reinterpret_cast<f32x4*>(o + EPL * x + e) =
              f32x4{acc[rt][e][x], acc[rt][e + 1][x], acc[rt][e + 2][x], acc[rt][e + 3][x]};
      if (h == 0) {
        float* ml = a.part + (int64_t)a.units * a.nsplit * rows * D + at * 2;
        ml[0] = m[rt];
        ml[1] = l[rt];
      }
      continue;
    }
    const int g = row[rt] / a.n, node = row[rt] - g * a.n;
    const int64_t head = (int64_t)bi * a.n_heads + hk * group + g;
    const bool none = r0 + depth[rt] < 0;                // a pad token: it sees nothing
    const float inv = none ? 0.0f : 1.0f / l[rt];
    E* o = static_cast<E*>(a.o) + (head * a.seq_ld + node) * D + 4 * EPL * h;
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
      for (int e = 0; e < EPL; e += 4) {
        f32x4 y = {acc[rt][e][x], acc[rt][e + 1][x], acc[rt][e + 2][x], acc[rt][e + 3][x]};
        y = none ? f32x4{0, 0, 0, 0} : y * inv;
        if constexpr (BF16)
          *reinterpret_cast<u32x2*>(o + EPL * x + e) = u32x2{pack2(y.x, y.y), pack2(y.z, y.w)};
        else
          *reinterpret_cast<f32x4*>(o + EPL * x + e) = y;
      }
    if (a.lse && h == 0)
      a.lse[head * a.n + node] = none ? kNegInf : (m[rt] + __builtin_amdgcn_logf(l[rt])) * kLn2;
  }
}

// Join the parts of a unit's keys: a wave a row, lane c holding part c's m and l.
template <typename E, int D>
__global__ void __launch_bounds__(256) nodes_join_kernel(NodesArgs a) {
  constexpr int P = D / 64;
  const int group = a.n_heads / a.n_kv_heads, rows = group * a.n;
  const int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (w >= (int64_t)a.units * rows) return;
  const int u = (int)(w / rows), row = (int)(w - (int64_t)u * rows);
  const int g = row / a.n, node = row - g * a.n;
  const int64_t first = (int64_t)u * a.nsplit * rows + row;
  const float* ml = a.part + (int64_t)a.units * a.nsplit * rows * D;
  float m = kNegInf, l = 0.0f;
  if (lane < a.nsplit) {
    const float* x = ml + (first + (int64_t)lane * rows) * 2;
    m = x[0];
    l = x[1];
  }
  const float top = lanes::wave_max(m);
  const bool none = top == kNegInf;                      // a pad token: it sees nothing
  const float f = m == kNegInf ? 0.0f : __builtin_amdgcn_exp2f(m - top);
  const float sum = lanes::wave_sum(f * l);
  float o[P] = {};
  for (int c = 0; c < a.nsplit; ++c) {
    const float fc = __shfl(f, c);
    const float* x = a.part + (first + (int64_t)c * rows) * D + lane * P;
#pragma unroll
    for (int e = 0; e < P; ++e) o[e] = fmaf(fc, x[e], o[e]);
  }
  const int64_t head = (int64_t)(u / a.n_kv_heads) * a.n_heads + (u % a.n_kv_heads) * group + g;
  E* dst = static_cast<E*>(a.o) + (head * a.seq_ld + node) * D + lane * P;
#pragma unroll
  for (int e = 0; e < P; ++e) {
    const float y = none ? 0.0f : o[e] / sum;
    if constexpr (sizeof(E) == 2) *reinterpret_cast<__bf16*>(dst + e) = (__bf16)y;
    else dst[e] = y;
  }
  if (a.lse && lane == 0)
    a.lse[head * a.n + node] = none ? kNegInf : (top + __builtin_amdgcn_logf(sum)) * kLn2;
}

// Workgroups over a unit's entries: as many as there are compute units for, each with at
// least kMinTiles tiles a wave (with fewer the joining launch costs more than it spares).
constexpr int kNodeWorkgroups = 512;
constexpr int kMinTiles = 1;
int most_splits(int units, const NodePlan& p) {
  const int64_t base = (int64_t)units * p.row_groups;
  const int64_t s = kNodeWorkgroups / base;
  return s < 1 ? 1 : s > kMaxNodeSplits ? kMaxNodeSplits : (int)s;
}

template <bool BF16, int D, int RT>
hipError_t launch_t(NodesArgs a, const NodePlan& p, hipStream_t stream) {
  const int tiles = (a.len0 + kTile - 1) / kTile, least = kMinTiles * p.key_waves();
  a.nsplit = most_splits(a.units, p);
  if (a.nsplit > tiles / least) a.nsplit = tiles / least > 1 ? tiles / least : 1;
  hipLaunchKernelGGL((nodes_kernel<BF16, D, RT>), dim3((unsigned)a.units, (unsigned)a.nsplit, (unsigned)p.row_groups),
                     dim3(64 * kNodeWaves), 0, stream, a, p.row_waves);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.nsplit == 1) return e;
  const int64_t rows = (int64_t)a.units * (a.n_heads / a.n_kv_heads) * a.n;
  hipLaunchKernelGGL((nodes_join_kernel<typename NodeCfg<BF16, D>::E, D>), dim3((unsigned)((rows + 3) / 4)), dim3(256),
                     0, stream, a);
  return hipGetLastError();
}

}  // namespace

size_t nodes_work_bytes(int units, int head_dim, int group, int n) {
  const size_t rows = (size_t)units * group * n;
  size_t most = 16;
  for (int bf16 = 0; bf16 < 2; ++bf16) {
    const int s = most_splits(units, plan_of(group * n, bf16 != 0));
    const size_t bytes = s > 1 ? rows * s * (head_dim + 2) * sizeof(float) : 0;
    if (bytes > most) most = bytes;
  }
  return most;
}

hipError_t launch_nodes(const NodesArgs& a, int dtype, int head_dim, int group, hipStream_t stream) {
  const NodePlan p = plan_of(group * a.n, dtype == BM_BF16);
  if (dtype == BM_F32)
    return head_dim == 128 ? launch_t<false, 128, 1>(a, p, stream) : launch_t<false, 64, 1>(a, p, stream);
  if (head_dim == 128)
    return p.rt == 1 ? launch_t<true, 128, 1>(a, p, stream) : launch_t<true, 128, 2>(a, p, stream);
  return p.rt == 1 ? launch_t<true, 64, 1>(a, p, stream) : launch_t<true, 64, 2>(a, p, stream);
}

}  // namespace bm
