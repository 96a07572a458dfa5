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
// A token is HBM-bound: 64 samples' over windows of 4096 entries (8 KV heads, d = 128) take
// 162 us, 6.6 TB/s (d = 64 85, 6.3; float32 over 1024 entries 109, 4.9).  A tree of 64 nodes with four heads each (256 rows a unit) is bound by its
// waves' own instructions, one wave a SIMD: 512 units of 4096 entries take 505 us, 375 without
// their loads, of which the products are 186 (545 TFLOP/s; with the second parts 820).
// Short launches are a chain of latencies: 8 units of 64 rows and 512 entries take 10.5 us
// (11 with waves of 32 rows, of which arguments 1, queries and tree 2, tiles 3, the join 2).
//
// The workgroup's waves share the rows (up to 8 blocks of them) and then the key tiles; waves
// over the same rows join through LDS, workgroups over the same unit through the workspace
// and a second launch.
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
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;

constexpr float kNegInf = -__builtin_huge_valf();
constexpr float kRescaleLog2 = 24.0f;  // the maximum moves once a logit is 2^24 beyond it
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kTile = 32;              // keys
// Waves of a workgroup: two a SIMD where 256 registers hold one's tile, otherwise one.
constexpr bool big_wave(bool bf16, int d, int rt) { return bf16 ? rt > 1 : d == 128; }
constexpr int node_waves(bool bf16, int d, int rt) { return big_wave(bf16, d, rt) ? 4 : 8; }
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

__device__ __forceinline__ float xsum4(float x) { return lanes::add_xor<32>(lanes::add_xor<16>(x)); }

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  bf16x2 r = {(__bf16)lo, (__bf16)hi};
  return __builtin_bit_cast(uint32_t, r);
}

// a buffer of whole rows: reads behind its end give zeros
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_of(const void* p, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, bytes, 0x00020000);
}

// x = max(x, y, z) in one instruction (of values that assembly made the compiler first makes
// quiet numbers)
__device__ __forceinline__ void max3(float& x, float y, float z) {
  asm volatile("v_max3_f32 %0, %0, %1, %2" : "+v"(x) : "v"(y), "v"(z));
}

// f(0), f(1), .. with numbers that are constants
template <typename F, int... I>
__device__ __forceinline__ void each(F f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
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
__device__ __forceinline__ Tree make_tree(const int32_t* parent, bool chain, int n, int r0, int sinks, int window) {
  const int a = threadIdx.x & 63;
  int up = -1;
  if (parent && a < n) {
    up = parent[a];
    if (up < 0 || up >= a) up = -1;
  }
  Tree t;
  t.sees = chain ? (2ull << a) - 1 : 1ull << a;    // (2 << 63 is 0)
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
  int waves;       // of a workgroup
  int rt;          // row tiles of a wave
  int row_waves;   // waves of a workgroup over different rows
  int row_groups;  // workgroups over different rows of a unit
  int key_waves() const { return waves / row_waves; }
};

// Waves of 64 rows read the keys from the caches half as often as those of 32, and are half as
// many: they pay once the launch has work for all compute units.  us with 32 -> 64 rows,
// 64 nodes of one, two or four query heads a KV head:
//   units rows entries   d = 128         d = 64         units rows entries   d = 128         d = 64
//   64 256 512           32.3 -> 42.2    26.9 -> 32.8   256 128 512          34.3 -> 32.0    25.3 -> 22.3
//   128 256 1024         51.5 -> 60.3    39.7 -> 45.7   256 128 2048         93.6 -> 75.6    59.8 -> 55.3
//   64 256 4096          92.4 -> 84.2    74.1 -> 65.8   512 128 512          65.4 -> 60.5    33.8 -> 42.7
//   256 256 512          65.7 -> 52.5    33.7 -> 36.1   512 128 2048         190 -> 159      102 -> 109
//   256 256 2048         177 -> 137      96.6 -> 101    64 64 4096           33.6 -> 35.4    26.3 -> 24.6
//   512 256 2048         369 -> 272      194 -> 203     256 64 512           21.4 -> 24.3    16.4 -> 16.5
//   64 128 512           26.4 -> 30.3    20.3 -> 21.0   256 64 2048          55.0 -> 52.4    35.8 -> 33.2
//   64 128 4096          55.4 -> 51.2    39.7 -> 37.9   512 64 2048          123 -> 116      57.1 -> 65.0
// One number for all of them (2^25) is up to 17% off at d = 128 (128 units of 256 rows, whose
// half as many workgroups split the keys instead) and up to 26% at d = 64, where two
// workgroups of the smaller waves fit a compute unit.
constexpr int64_t kBigWork = 1 << 25;       // units x rows x entries
// Waves of 16 rows have the shorter chain where there is next to nothing to read; us with
// 32 -> 16 rows:
//   units rows entries  8 32 512      8 64 512      8 256 512     32 64 512     32 128 512
//                       12.5 -> 11.8  14.4 -> 13.8  24.6 -> 23.2  18.1 -> 17.5  24.4 -> 25.5
//                       8 32 4096     8 64 4096     64 64 512     64 128 4096
//                       15.5 -> 15.2  19.3 -> 19.8  18.9 -> 20.1  40.1 -> 55.3
constexpr int64_t kSmallWork = 1 << 20;
NodePlan plan_of(int rows, bool bf16, int d, int64_t work) {
  NodePlan p;
  p.rt = !bf16 || rows <= 16 || work <= kSmallWork ? 1 : rows <= 32 || work < kBigWork ? 2 : 4;
  p.waves = node_waves(bf16, d, p.rt);
  const int blocks = (rows + 16 * p.rt - 1) / (16 * p.rt);
  p.row_waves = 1;
  while (p.row_waves < blocks && p.row_waves < p.waves) p.row_waves *= 2;
  p.row_groups = (blocks + p.row_waves - 1) / p.row_waves;
  return p;
}

// z = or += K Q^T of a 16 x 16 tile of bfloat16, for waves of 32 and 64 rows.  As assembly: for a
// kernel of more than 256 registers the compiler puts every product's result into the
// accumulation registers, from which each logit would have to be copied before a vector
// instruction could use it.  The compiler does not count the wait states until such an
// instruction may read the result either: s_settled does.
template <bool FIRST>
__device__ __forceinline__ void mfma_s(f32x4& z, u32x4 k, u32x4 q) {
  if constexpr (FIRST)
    asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, 0" : "=&v"(z) : "v"(k), "a"(q));
  else
    asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+&v"(z) : "v"(k), "a"(q));
}
template <int RT>
__device__ __forceinline__ void s_settled(f32x4 (&s)[RT][2]) {
  asm volatile("s_nop 15" ::: "memory");
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) asm volatile("" : "+v"(s[rt][0]), "+v"(s[rt][1]));
}

// NT: the cached rows are read past the last-level cache
template <bool BF16, int D, int RT, bool NT>
__global__ void __launch_bounds__(64 * node_waves(BF16, D, RT), 1) nodes_kernel(NodesArgs a, int row_waves) {
  constexpr int kNodeWaves = node_waves(BF16, D, RT);
  constexpr bool kBig = big_wave(BF16, D, RT);
  using C = NodeCfg<BF16, D>;
  using E = typename C::E;
  constexpr int RB = C::RB, KL = C::KL, EPL = C::EPL, VW = C::VW;
  constexpr int kAux = NT ? 2 : 0;                     // a load's non-temporal bit
  // a wave's part of LDS: O in quads of elements, m and l, for the join; the weights of a tile
  // of 32 keys (see the end of a tile) for a moment before
  constexpr int QUADS = EPL, PART = RT * (QUADS * 256 + 128);
  static_assert(QUADS * 256 >= 512, "weights of 32 keys and 16 rows");
  __shared__ __attribute__((aligned(16))) float lds[kNodeWaves * PART];
  const int group = a.n_heads / a.n_kv_heads, rows = group * a.n;
  const int u = blockIdx.x, split = blockIdx.y;
  const int bi = u / a.n_kv_heads, hk = u - bi * a.n_kv_heads;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int i16 = lane & 15, h = lane >> 4;
  const int key_waves = kNodeWaves / row_waves, rw = wave / key_waves, kw = wave - rw * key_waves;
  const int row0 = ((int)blockIdx.z * row_waves + rw) * 16 * RT;     // the wave's first row
  const int pad = a.pad ? max(0, __builtin_amdgcn_readfirstlane(a.pad[bi])) : 0;
  const int r0 = index_of(a.next_pos, pad);                          // a root's index
  const Ring ring(r0, a.sinks, max(a.window, 1));
  const int entries = a.window ? ring.filled() : a.len0;

  // ---- the workgroup's tiles: its share of the cached ones with the nodes' behind them ----
  const int tiles = (entries + kTile - 1) / kTile, all = tiles + (a.n + kTile - 1) / kTile;
  const int per = (all + a.nsplit - 1) / a.nsplit;
  const int lo = min(split * per, all), total = min(per, all - lo);
  const int cached = min(max(tiles - lo, 0), total), node0 = tiles - lo;   // tile node0 is the first of the nodes

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
    const int base = (node ? t - node0 : lo + t) * kTile;
    const auto r = rows_of(node ? kin : kc, (node ? a.n : entries) * RB);
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int kk = 0; kk < KL; ++kk)
        kf[s][kk] = __builtin_amdgcn_raw_buffer_load_b128(r, (base + 16 * s + i16) * RB + 16 * h + 64 * kk, 0, kAux);
    if (pos && pad > 0 && !node) pk = pos[min(base + (lane & 31), entries - 1)];
  };
  auto load_v = [&](int t) BM_LAMBDA {
    const bool node = t >= cached;
    const int base = (node ? t - node0 : lo + t) * kTile;
    const auto r = rows_of(node ? vin : vc, (node ? a.n : entries) * RB);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int off = (base + 16 * (i >> 2) + 4 * h + (i & 3)) * RB + i16 * (4 * VW);
      if constexpr (VW == 2) {
        const u32x2 x = __builtin_amdgcn_raw_buffer_load_b64(r, off, 0, kAux);
        vf[i][0] = x.x;
        vf[i][1] = x.y;
      } else {
#pragma unroll
        for (int w = 0; w < VW; w += 4) {
          const u32x4 x = __builtin_amdgcn_raw_buffer_load_b128(r, off + 4 * w, 0, kAux);
          vf[i][w] = x.x;
          vf[i][w + 1] = x.y;
          vf[i][w + 2] = x.z;
          vf[i][w + 3] = x.w;
        }
      }
    }
  };
  load_k(kw);
  if constexpr (!(BF16 && kBig)) load_v(kw);

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
  const Tree tree = make_tree(a.parent ? a.parent + (int64_t)bi * a.n : nullptr, a.chain != 0, a.n, r0, a.sinks,
                              a.window ? a.window : kNoWindow);
  // (what a row's node sees and its depth come from that node's lane where they are needed)
  int own[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) own[rt] = min(row[rt], rows - 1) % a.n;

  // The entries that the window hides from the deepest node: `old` slots from `oldest` on, going
  // round behind the ring's last one.  Where all nodes are roots nobody sees them; otherwise
  // the deeper ones do not.
  const bool nested = __ballot(lane < a.n && tree.depth > 0) != 0;
  int oldest = 0, old = 0;
  if (a.window) {
    int deepest = 0;
    if (nested) {
      deepest = lane < a.n ? tree.depth : 0;
#pragma unroll
      for (int off = 32; off; off >>= 1) deepest = max(deepest, __shfl_xor(deepest, off));
      deepest = __builtin_amdgcn_readfirstlane(deepest);
    }
    const bool full = r0 >= a.sinks + a.window;
    oldest = a.sinks + (full ? (ring.last + 1) % a.window : 0);
    old = min(full ? deepest + 1 : max(r0 - a.window + deepest - a.sinks + 1, 0), a.window);
  }
  const int old_end = min(oldest + old, a.slots), wrapped = a.sinks + oldest + old - a.slots;   // slots behind the ring's start
  auto has_old = [&](int base) BM_LAMBDA {
    return old > 0 && ((base < old_end && base + kTile > oldest) || (base < wrapped && base + kTile > a.sinks));
  };
  auto is_old = [&](int slot) BM_LAMBDA {
    return (slot >= oldest && slot < old_end) || (slot >= a.sinks && slot < wrapped);
  };

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

  auto keep_acc = [&]() BM_LAMBDA {
    // (O stays in the accumulation registers over the loops)
    if constexpr (kBig) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int e = 0; e < EPL; ++e) asm volatile("" : "+a"(acc[rt][e]));
    }
  };
  // Tile t.  MIXED: rows see different keys of it (the nodes, and entries at the window's edge);
  // otherwise they all see the same ones.
  auto tile = [&](auto mixed_tag, int t) BM_LAMBDA {
    constexpr bool MIXED = decltype(mixed_tag)::value;
    const bool node = MIXED && t >= cached;
    const int base = (node ? t - node0 : lo + t) * kTile;
    // ---- logits ----
    f32x4 s[RT][2];
    if constexpr (!(BF16 && kBig)) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int x = 0; x < 2; ++x) s[rt][x] = f32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int kk = 0; kk < KL; ++kk)
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          if constexpr (BF16 && kBig) {
            if (kk == 0) mfma_s<true>(s[rt][x], kf[x][kk], qf[rt][kk]);
            else mfma_s<false>(s[rt][x], kf[x][kk], qf[rt][kk]);
          } else if constexpr (BF16) {
            s[rt][x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf[x][kk]),
                                                               __builtin_bit_cast(bf16x8, qf[rt][kk]), s[rt][x], 0, 0, 0);
          } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
              s[rt][x] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kf[x][kk][j]),
                                                              __uint_as_float(qf[rt][kk][j]), s[rt][x], 0, 0, 0);
          }
        }
    const int pk0 = pk;
    if constexpr (!kBig) load_k(t + key_waves);
    if constexpr (BF16 && kBig) s_settled(s);

    // ---- keys that nobody sees: bit k of `gone`; V rows of theirs become zeros, so that a
    //      NaN there does not count either ----
    uint32_t gone = 0;
    if (node) {
      gone = base + kTile > a.n ? ~0u << (a.n - base) : 0;
    } else if (base + kTile > entries || (pos && pad > 0) || (!nested && has_old(base))) {
      const int slot = base + (lane & 31);
      gone = (uint32_t)__ballot(slot >= entries || (pos && pad > 0 && pk0 < pad) || (!nested && is_old(slot)));
    }
    const uint32_t hide = gone >> (4 * h);               // bit 16 t + r: this lane's key (t, r)
    if (gone != 0) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const bool z = (hide >> (16 * (i >> 2) + (i & 3))) & 1;
#pragma unroll
        for (int w = 0; w < VW; ++w) vf[i][w] = z ? 0u : vf[i][w];
        if constexpr (!MIXED) {
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) s[rt][i >> 2][i & 3] = z ? kNegInf : s[rt][i >> 2][i & 3];
        }
      }
    }
    // ... and what each row does not see: by the tree, or by the index of an entry less that
    // of the oldest one a root does not see, against the row's depth
    uint32_t mask[RT];
    if constexpr (MIXED) {
      int dist[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int slot = base + 16 * (i >> 2) + 4 * h + (i & 3);
        dist[i] = node || slot < a.sinks ? kNoWindow : ring.index(min(slot, a.slots - 1)) - (r0 - a.window);
      }
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        const int depth = __shfl(tree.depth, own[rt]);
        const uint64_t sees = shfl64(tree.sees, own[rt]);
        mask[rt] = hide | (node ? (uint32_t)~(sees >> base) >> (4 * h) : 0u);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (dist[i] <= depth) mask[rt] |= 1u << (16 * (i >> 2) + (i & 3));
          if ((mask[rt] >> (16 * (i >> 2) + (i & 3))) & 1) s[rt][i >> 2][i & 3] = kNegInf;
        }
      }
    }

    // ---- softmax ----
    uint32_t phi[RT][4], plo[RT][4];                     // bfloat16 weights, two parts
    float pf[BF16 ? 1 : RT][8];                          // float32 weights
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      float top = kNegInf;
      float(&pw)[8] = pf[BF16 ? 0 : rt];
#pragma unroll
      for (int i = 0; i < 8; ++i) top = fmaxf(top, s[rt][i >> 2][i & 3]);
      if (__builtin_expect(__ballot(top * c2 > m[rt] + kRescaleLog2) != 0, 0)) {
        const float mn = fmaxf(m[rt], lanes::max_xor16_32(top) * c2);
        // (a row that has seen no key yet: nothing to scale)
        const float f = mn == kNegInf ? 1.0f : __builtin_amdgcn_exp2f(m[rt] - mn);
        m[rt] = mn;
        l[rt] *= f;
#pragma unroll
        for (int e = 0; e < EPL; ++e) {
          acc[rt][e] *= f;
          if constexpr (kBig) asm volatile("" : "+a"(acc[rt][e]));   // (back in its registers on this path)
        }
      }
      const float ref = m[rt] == kNegInf ? 0.0f : m[rt];
      float sum = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        pw[i] = __builtin_amdgcn_exp2f(fmaf(s[rt][i >> 2][i & 3], c2, -ref));
        sum += pw[i];
      }
      l[rt] += sum;
      if constexpr (BF16) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t hi = pack2(pw[2 * i], pw[2 * i + 1]);
          phi[rt][i] = hi;
          plo[rt][i] = pack2(pw[2 * i] - __uint_as_float(hi << 16), pw[2 * i + 1] - __uint_as_float(hi & 0xFFFF0000u));
        }
      }
    }

    // ---- MIXED: a V row with an infinity or a NaN becomes zeros too, and is added below to
    //      the rows that see it, one by one ----
    uint32_t bad = 0;
    if constexpr (MIXED) {
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
      if constexpr (kBig) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
          for (int w = 0; w < VW; ++w) vf[i][w] = 0;
      } else {
        load_v(t + key_waves);
      }
#pragma unroll
      for (int e = 0; e < EPL; ++e)
#pragma unroll
        for (int part = 0; part < 2; ++part)
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) {
            const uint32_t(&p)[4] = part ? plo[rt] : phi[rt];
            acc[rt][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vt[e]),
                                                                 __builtin_bit_cast(bf16x8, u32x4{p[0], p[1], p[2], p[3]}),
                                                                 acc[rt][e], 0, 0, 0);
          }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < EPL; ++e)
#pragma unroll
          for (int rt = 0; rt < RT; ++rt)
            acc[rt][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vf[i][e]), pf[rt][i], acc[rt][e], 0, 0, 0);
      load_v(t + key_waves);
    }

    // ---- the rows taken out above, for those that see them ----
    if constexpr (MIXED) {
      if (__builtin_expect(bad != 0, 0)) {
        float* w = lds + wave * PART;                // weights [RT][32 keys][16 rows], < 0: hidden
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int key = 16 * (i >> 2) + 4 * h + (i & 3);
            float p;
            if constexpr (BF16) {
              const uint32_t x = phi[rt][i >> 1], y = plo[rt][i >> 1];
              p = i & 1 ? __uint_as_float(x & 0xFFFF0000u) + __uint_as_float(y & 0xFFFF0000u)
                        : __uint_as_float(x << 16) + __uint_as_float(y << 16);
            } else {
              p = pf[rt][i];
            }
            w[(rt * 32 + key) * 16 + i16] = (mask[rt] >> (16 * (i >> 2) + (i & 3))) & 1 ? -1.0f : p;
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
      keep_acc();
    }
    if constexpr (kBig) load_k(t + key_waves);           // (before, there are no registers for it)
  };

  // Big waves, plain tiles: the values' product of tile t - 1 goes with the weights of tile t,
  // product by product, so that the matrix and the vector unit work at the same time (one
  // wave a SIMD: nobody else would use the one while the other works).  V is loaded a
  // tile later than K: vf holds tile t - 1's rows, of which nobody sees `late`.
  using weights_t = uint32_t[BF16 && kBig ? RT : 1][8];
  weights_t po = {};                                     // tile t - 1's: four words, four of the rest
  uint32_t late = 0;
  auto turn = [&](u32x4 (&vt)[EPL]) BM_LAMBDA {
    if (late != 0) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const bool z = ((late >> (4 * h)) >> (16 * (i >> 2) + (i & 3))) & 1;
#pragma unroll
        for (int w = 0; w < VW; ++w) vf[i][w] = z ? 0u : vf[i][w];
      }
    }
#pragma unroll
    for (int w = 0; w < VW; ++w)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        vt[2 * w][j] = __builtin_amdgcn_perm(vf[2 * j + 1][w], vf[2 * j][w], 0x05040100);
        vt[2 * w + 1][j] = __builtin_amdgcn_perm(vf[2 * j + 1][w], vf[2 * j][w], 0x07060302);
      }
  };
  auto product = [&](auto jc, const u32x4 (&vt)[EPL]) BM_LAMBDA {
    constexpr int j = decltype(jc)::value, e = j / (2 * RT), part = j / RT % 2, rt = j % RT;
    const uint32_t* p = po[rt] + 4 * part;
    acc[rt][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vt[e]),
                                                         __builtin_bit_cast(bf16x8, u32x4{p[0], p[1], p[2], p[3]}),
                                                         acc[rt][e], 0, 0, 0);
  };
  // what is left of the last plain tile
  auto flush = [&]() BM_LAMBDA {
    if constexpr (BF16 && kBig) {
      u32x4 vt[EPL];
      turn(vt);
      each([&](auto jc) BM_LAMBDA { product(jc, vt); }, std::make_integer_sequence<int, 2 * RT * EPL>{});
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int i = 0; i < 8; ++i) po[rt][i] = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int w = 0; w < VW; ++w) vf[i][w] = 0;
      late = 0;
      keep_acc();
    }
  };
  auto plain_tile = [&](int t) BM_LAMBDA {
    if constexpr (!(BF16 && kBig)) {
      tile(std::false_type{}, t);
    } else {
      const int base = (lo + t) * kTile;
      f32x4 s[RT][2];
#pragma unroll
      for (int kk = 0; kk < KL; ++kk)
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) {
            if (kk == 0) mfma_s<true>(s[rt][x], kf[x][kk], qf[rt][kk]);
            else mfma_s<false>(s[rt][x], kf[x][kk], qf[rt][kk]);
          }
      const int pk0 = pk;
      load_k(t + key_waves);
      u32x4 vt[EPL];
      turn(vt);
      load_v(t);
      s_settled(s);
      late = 0;
      if (base + kTile > entries || (pos && pad > 0) || (!nested && has_old(base))) {
        const int slot = base + (lane & 31);
        late = (uint32_t)__ballot(slot >= entries || (pos && pad > 0 && pk0 < pad) || (!nested && is_old(slot)));
        if (late != 0) {
          const uint32_t hide = late >> (4 * h);
#pragma unroll
          for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int i = 0; i < 8; ++i)
              s[rt][i >> 2][i & 3] = (hide >> (16 * (i >> 2) + (i & 3))) & 1 ? kNegInf : s[rt][i >> 2][i & 3];
        }
      }
      // the maxima; O follows behind the product of the tile before
      float top[RT], f[RT];
      bool over = false;
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        top[rt] = kNegInf;
        f[rt] = 1.0f;
#pragma unroll
        for (int i = 0; i < 8; i += 2) max3(top[rt], s[rt][i >> 2][i & 3], s[rt][i >> 2][(i & 3) + 1]);
        over = over || top[rt] * c2 > m[rt] + kRescaleLog2;
      }
      const bool raise = __ballot(over) != 0;
      if (__builtin_expect(raise, 0)) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          const float mn = fmaxf(m[rt], lanes::max_xor16_32(top[rt]) * c2);
          f[rt] = mn == kNegInf ? 1.0f : __builtin_amdgcn_exp2f(m[rt] - mn);
          m[rt] = mn;
          l[rt] *= f[rt];
        }
      }
      float ref[RT], sum[RT];
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        ref[rt] = m[rt] == kNegInf ? 0.0f : m[rt];
        sum[rt] = 0.0f;
      }
      // weight i of the lane's 8 RT: its argument a weight before, its sum and packing one behind
      weights_t pn;
      float x[2], y[2];
      auto args = [&](int i) BM_LAMBDA { x[i & 1] = fmaf(s[i / 8][(i >> 2) & 1][i & 3], c2, -ref[i / 8]); };
      auto pack = [&](int i) BM_LAMBDA {
        sum[i / 8] += y[i & 1];
        if (i & 1) {
          uint32_t hi = pack2(y[0], y[1]);
          uint32_t rest = pack2(y[0] - __uint_as_float(hi << 16), y[1] - __uint_as_float(hi & 0xFFFF0000u));
          asm volatile("" : "+v"(hi), "+v"(rest), "+v"(sum[i / 8]));   // (made here, not where they are used)
          pn[i / 8][(i & 7) >> 1] = hi;
          pn[i / 8][4 + ((i & 7) >> 1)] = rest;
        }
      };
      constexpr int NS = 2 * RT * EPL, NW = 8 * RT, EVERY = NS / NW;
      args(0);
      each([&](auto jc) BM_LAMBDA {
        constexpr int j = decltype(jc)::value, i = j / EVERY;
        __builtin_amdgcn_sched_barrier(0);
        product(jc, vt);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (j % EVERY == 0) {
          // (an even weight's packing waits for the odd one's: y holds both)
          const float e = __builtin_amdgcn_exp2f(x[i & 1]);
          if constexpr (i > 0) pack(i - 1);
          y[i & 1] = e;
          if constexpr (i + 1 < NW) args(i + 1);
        }
      }, std::make_integer_sequence<int, NS>{});
      pack(NW - 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        l[rt] += sum[rt];
#pragma unroll
        for (int i = 0; i < 8; ++i) po[rt][i] = pn[rt][i];
      }
      if (__builtin_expect(raise, 0)) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          asm volatile("" : "+v"(f[rt]));              // (not multiplied by 1 every time)
#pragma unroll
          for (int e = 0; e < EPL; ++e) {
            acc[rt][e] *= f[rt];
            asm volatile("" : "+a"(acc[rt][e]));
          }
        }
      }
    }
  };
  keep_acc();
  if constexpr (BF16 && kBig) {
    // nothing comes before the first plain tile
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int w = 0; w < VW; ++w) vf[i][w] = 0;
  }
  for (int t = kw; t < total;) {
    for (; t < cached && !(nested && has_old((lo + t) * kTile)); t += key_waves) {
      plain_tile(t);
      keep_acc();
    }
    flush();
    if (t < total) {
      if constexpr (BF16 && kBig) load_v(t);
      tile(std::true_type{}, t);
      t += key_waves;
    }
  }
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) l[rt] = xsum4(l[rt]);

  // ---- join the waves over the same rows, and the results: lane (i16, h) holds elements
  //      4 EPL h .. of row i16, EPL of them for each x; the waves take turns by (rt, x) ----
  float* part = lds + (wave - kw) * PART;                // of the first wave over these rows
  if (key_waves > 1) {
    float* mine = lds + wave * PART;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      float* y = mine + rt * (QUADS * 256 + 128);
#pragma unroll
      for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int e = 0; e < EPL; e += 4)
          *reinterpret_cast<f32x4*>(y + ((x * EPL + e) / 4 * 64 + lane) * 4) =
              f32x4{acc[rt][e][x], acc[rt][e + 1][x], acc[rt][e + 2][x], acc[rt][e + 3][x]};
      y[QUADS * 256 + lane] = m[rt];
      y[QUADS * 256 + 64 + lane] = l[rt];
    }
    __syncthreads();
  }
  // (their number is a constant here so that nothing waits for one LDS read after the other)
  auto join = [&](auto kw_tag) BM_LAMBDA {
    constexpr int KW = decltype(kw_tag)::value;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const bool none = r0 + __shfl(tree.depth, own[rt]) < 0;   // a pad token: it sees nothing
      if (row[rt] >= rows) continue;
      float f[KW], mx = m[rt], sum = l[rt];
      if constexpr (KW > 1) {
        const float* y = part + rt * (QUADS * 256 + 128) + QUADS * 256 + lane;
        float mj[KW], lj[KW];
#pragma unroll
        for (int j = 0; j < KW; ++j) {
          mj[j] = y[j * PART];
          lj[j] = y[j * PART + 64];
        }
        mx = mj[0];
#pragma unroll
        for (int j = 1; j < KW; ++j) mx = fmaxf(mx, mj[j]);
        sum = 0.0f;
#pragma unroll
        for (int j = 0; j < KW; ++j) {
          f[j] = mj[j] == kNegInf ? 0.0f : __builtin_amdgcn_exp2f(mj[j] - mx);
          sum = fmaf(f[j], lj[j], sum);
        }
      }
      const int g = row[rt] / a.n, node = own[rt];
      const int64_t head = (int64_t)bi * a.n_heads + hk * group + g;
      const int64_t at = ((int64_t)u * a.nsplit + split) * rows + row[rt];
      const float inv = a.nsplit > 1 ? 1.0f : none ? 0.0f : 1.0f / sum;
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        if (((4 * rt + x) & (KW - 1)) != kw) continue;
#pragma unroll
        for (int e = 0; e < EPL; e += 4) {
          f32x4 o = {acc[rt][e][x], acc[rt][e + 1][x], acc[rt][e + 2][x], acc[rt][e + 3][x]};
          if constexpr (KW > 1) {
            o = f32x4{0, 0, 0, 0};
            const float* y = part + rt * (QUADS * 256 + 128) + ((x * EPL + e) / 4 * 64 + lane) * 4;
#pragma unroll
            for (int j = 0; j < KW; ++j) o += f[j] * *reinterpret_cast<const f32x4*>(y + j * PART);
          }
          if (a.nsplit > 1) {
            *reinterpret_cast<f32x4*>(a.part + at * D + 4 * EPL * h + EPL * x + e) = o;
            continue;
          }
          o = none ? f32x4{0, 0, 0, 0} : o * inv;
          E* dst = static_cast<E*>(a.o) + (head * a.seq_ld + node) * D + 4 * EPL * h + EPL * x + e;
          if constexpr (BF16) *reinterpret_cast<u32x2*>(dst) = u32x2{pack2(o.x, o.y), pack2(o.z, o.w)};
          else *reinterpret_cast<f32x4*>(dst) = o;
        }
      }
      if (h == 0 && kw == 0) {
        if (a.nsplit > 1) {
          float* ml = a.part + (int64_t)a.units * a.nsplit * rows * D + at * 2;
          ml[0] = mx;
          ml[1] = sum;
        } else if (a.lse) {
          a.lse[head * a.n + node] = none ? kNegInf : (mx + __builtin_amdgcn_logf(sum)) * kLn2;
        }
      }
    }
  };
  if (key_waves == 1) join(std::integral_constant<int, 1>{});
  else if (key_waves == 2) join(std::integral_constant<int, 2>{});
  else if (key_waves == 4) join(std::integral_constant<int, 4>{});
  else if constexpr (kNodeWaves == 8) join(std::integral_constant<int, 8>{});
}

// Join the parts of a unit's keys: lane c holds part c's m and l of a row, C parts are on their
// way at a time (past the last one its own again, without weight), the first ones before
// their weights are known.  Latency-bound: a wave has one row, four where two parts say
// that there are many (32768 rows take 12.0 us, 14.5 with one a wave; one token's 32 rows
// of four parts the other way round: 10.0 us a step, 10.9 with two a wave).
template <int C>
constexpr int join_rows() { return C == 2 ? 4 : 1; }
template <typename E, int D, int C>
__global__ void __launch_bounds__(256) nodes_join_kernel(NodesArgs a) {
  constexpr int P = D / 64, R = join_rows<C>();
  const int group = a.n_heads / a.n_kv_heads, rows = group * a.n, all = a.units * rows;
  const int w0 = ((int)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * R;
  const int lane = threadIdx.x & 63;
  if (w0 >= all) return;
  const float* ml = a.part + (int64_t)a.nsplit * all * D;
  int u[R], row[R];
  int64_t first[R];
  float x[R][C][P], m[R], l[R], o[R][P];
  auto load = [&](int c0) BM_LAMBDA {
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const float* y = a.part + (first[r] + (int64_t)min(c0 + c, a.nsplit - 1) * rows) * D + lane * P;
#pragma unroll
        for (int e = 0; e < P; ++e) x[r][c][e] = y[e];
      }
  };
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int w = min(w0 + r, all - 1);
    u[r] = w / rows;
    row[r] = w - u[r] * rows;
    first[r] = (int64_t)u[r] * a.nsplit * rows + row[r];
    m[r] = kNegInf;
    l[r] = 0.0f;
    if (lane < a.nsplit) {
      const float* y = ml + (first[r] + (int64_t)lane * rows) * 2;
      m[r] = y[0];
      l[r] = y[1];
    }
#pragma unroll
    for (int e = 0; e < P; ++e) o[r][e] = 0.0f;
  }
  load(0);
  float top[R], f[R], sum[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    top[r] = lanes::wave_max(m[r]);
    f[r] = m[r] == kNegInf ? 0.0f : __builtin_amdgcn_exp2f(m[r] - top[r]);
    sum[r] = lanes::wave_sum(f[r] * l[r]);
  }
  for (int c0 = 0;;) {
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const float fc = c0 + c < a.nsplit ? __shfl(f[r], c0 + c) : 0.0f;
#pragma unroll
        for (int e = 0; e < P; ++e) o[r][e] = fmaf(fc, x[r][c][e], o[r][e]);
      }
    c0 += C;
    if (c0 >= a.nsplit) break;
    load(c0);
  }
#pragma unroll
  for (int r = 0; r < R; ++r) {
    if (w0 + r >= all) break;
    const bool none = top[r] == kNegInf;                 // a pad token: it sees nothing
    const int g = row[r] / a.n, node = row[r] - g * a.n;
    const int64_t head = (int64_t)(u[r] / a.n_kv_heads) * a.n_heads + (u[r] % a.n_kv_heads) * group + g;
    E* dst = static_cast<E*>(a.o) + (head * a.seq_ld + node) * D + lane * P;
#pragma unroll
    for (int e = 0; e < P; ++e) o[r][e] = none ? 0.0f : o[r][e] / sum[r];
    if constexpr (sizeof(E) == 4) {
#pragma unroll
      for (int e = 0; e < P; ++e) dst[e] = o[r][e];
    } else if constexpr (P == 2) {
      *reinterpret_cast<uint32_t*>(dst) = pack2(o[r][0], o[r][1]);
    } else {
      *reinterpret_cast<__bf16*>(dst) = (__bf16)o[r][0];
    }
    if (a.lse && lane == 0)
      a.lse[head * a.n + node] = none ? kNegInf : (top[r] + __builtin_amdgcn_logf(sum[r])) * kLn2;
  }
}

// Workgroups over a unit's entries: what fills the compute units, one workgroup each, with at
// least one tile a wave, and as many rows of partial results as the joining launch reads
// in a few microseconds.
constexpr int kNodeWorkgroups = 256;
constexpr int kMostPartialRows = 65536;
int most_splits(int units, int rows, const NodePlan& p) {
  const int64_t fill = kNodeWorkgroups / ((int64_t)units * p.row_groups);
  const int64_t room = kMostPartialRows / ((int64_t)units * rows);
  const int64_t s = fill < room ? fill : room;
  return s < 1 ? 1 : s > kMaxNodeSplits ? kMaxNodeSplits : (int)s;
}

// (split launches have at most kMostPartialRows rows: numbers of 32 bits)
template <bool BF16, int D>
hipError_t launch_join(const NodesArgs& a, hipStream_t stream) {
  using E = typename NodeCfg<BF16, D>::E;
  const int rows = a.units * (a.n_heads / a.n_kv_heads) * a.n;
  auto launch = [&](auto c) {
    constexpr int C = decltype(c)::value, in_block = 4 * join_rows<C>();
    hipLaunchKernelGGL((nodes_join_kernel<E, D, C>), dim3((unsigned)((rows + in_block - 1) / in_block)), dim3(256), 0, stream, a);
  };
  if (a.nsplit <= 2) launch(std::integral_constant<int, 2>{});
  else if (a.nsplit <= 4) launch(std::integral_constant<int, 4>{});
  else launch(std::integral_constant<int, 8>{});
  return hipGetLastError();
}

template <bool BF16, int D, int RT>
hipError_t launch_t(NodesArgs a, const NodePlan& p, hipStream_t stream) {
  const int tiles = (a.len0 + kTile - 1) / kTile + (a.n + kTile - 1) / kTile, most = tiles / p.key_waves();
  a.nsplit = most_splits(a.units, a.n_heads / a.n_kv_heads * a.n, p);
  if (a.nsplit > most) a.nsplit = most > 1 ? most : 1;
  const dim3 grid((unsigned)a.units, (unsigned)a.nsplit, (unsigned)p.row_groups), block(64 * p.waves);
  // Rows that one wave alone reads, once a step, stream past the last-level cache where it holds
  // less than half of them: 1.07 GB take 161 us instead of 176, while of 269 MB the next
  // step still finds enough there (45.7 us past it, 42.6 through it).
  const size_t bytes = (size_t)a.units * a.len0 * 2 * NodeCfg<BF16, D>::RB;
  const bool past = RT == 1 && p.row_waves == 1 && p.row_groups == 1 && bytes > 2 * kLastLevelCacheBytes;
  if (past)
    hipLaunchKernelGGL((nodes_kernel<BF16, D, RT, RT == 1>), grid, block, 0, stream, a, p.row_waves);
  else
    hipLaunchKernelGGL((nodes_kernel<BF16, D, RT, false>), grid, block, 0, stream, a, p.row_waves);
  hipError_t e = hipGetLastError();
  return e == hipSuccess && a.nsplit > 1 ? launch_join<BF16, D>(a, stream) : e;
}

}  // namespace

size_t nodes_work_bytes(int units, int head_dim, int group, int n) {
  // (no plan has more splits than one of a single row group; never less for more nodes)
  const int64_t fill = kNodeWorkgroups / units, s = fill > kMaxNodeSplits ? kMaxNodeSplits : fill;
  if (s < 2) return 16;
  const int64_t rows = (int64_t)units * group * n * s;
  return (size_t)(rows < kMostPartialRows ? rows : kMostPartialRows) * (head_dim + 2) * sizeof(float);
}

hipError_t launch_nodes(const NodesArgs& a, int dtype, int head_dim, int group, hipStream_t stream) {
  const int64_t work = (int64_t)a.units * group * a.n * a.len0;
  const NodePlan p = plan_of(group * a.n, dtype == BM_BF16, head_dim, work);
  if (dtype == BM_F32)
    return head_dim == 128 ? launch_t<false, 128, 1>(a, p, stream) : launch_t<false, 64, 1>(a, p, stream);
  if (head_dim == 128)
    return p.rt == 1 ? launch_t<true, 128, 1>(a, p, stream)
         : p.rt == 2 ? launch_t<true, 128, 2>(a, p, stream) : launch_t<true, 128, 4>(a, p, stream);
  return p.rt == 1 ? launch_t<true, 64, 1>(a, p, stream)
       : p.rt == 2 ? launch_t<true, 64, 2>(a, p, stream) : launch_t<true, 64, 4>(a, p, stream);
}

hipError_t launch_nodes_join(const NodesArgs& a, int dtype, int head_dim, hipStream_t stream) {
  if (dtype == BM_F32) return head_dim == 128 ? launch_join<false, 128>(a, stream) : launch_join<false, 64>(a, stream);
  return head_dim == 128 ? launch_join<true, 128>(a, stream) : launch_join<true, 64>(a, stream);
}

}  // namespace bm
