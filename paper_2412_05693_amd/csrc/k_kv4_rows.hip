// K8: rows into and out of a cache held in 4 bits (include/bm_kv4.h).
//
// A lane owns eight consecutive elements of a row, a quad of lanes one group of
// 32 and its scale; it moves the K row's and the V row's eight elements of the
// same slot.  The scale is an integer step on the float bits of the group's
// largest element, the codes come from gfx950's conversions.  HBM-bound: 16
// (float32: 32) bytes in for 4.25 bytes out, or the reverse, each read and
// written once.  512 units of 256 bf16 rows of 128 (84 MB): 14.7 us stored, 13.8
// read back (5.7 and 6.1 TB/s); 4096 units of 512 rows read back 1.36 GB in 251
// us (5.4 TB/s; a copy of that size runs at 5.2).
#include "bm_internal.h"
#include "bm_kv4_dev.h"

namespace bm {
namespace {

using kv4::u32x4;

// Item i of a launch is row i % n of unit i / n; a lane takes ITERS of them, the loads of
// all in flight.  A workgroup's first item is split with one 64-bit division, the rest
// with 32-bit ones (n <= 65536).
template <int D, int ITERS>
struct Items {
  static constexpr int kLanes = D / 8;              // lanes per row
  static constexpr int kRows = 256 / kLanes;        // rows a workgroup moves at a time
  int64_t u0, left;
  uint32_t r0, n;
  int lane, first;
  __device__ __forceinline__ Items(const Kv4RowsArgs& a, int64_t block) {
    const int64_t i0 = block * (kRows * ITERS);
    u0 = i0 / a.n;
    r0 = (uint32_t)(i0 - u0 * a.n);
    n = (uint32_t)a.n;
    left = (int64_t)a.units * a.n - i0;
    lane = threadIdx.x % kLanes;
    first = threadIdx.x / kLanes;
  }
  // unit and row of the lane's k-th item; false past the last (the unit and row are
  // then those of the workgroup's first item, so that a load stays in bounds)
  __device__ __forceinline__ bool at(int k, int64_t* u, uint32_t* r) const {
    const uint32_t off = (uint32_t)(first + k * kRows);
    const bool live = off < left;
    const uint32_t t = r0 + (live ? off : 0);
    const uint32_t q = t / n;
    *u = u0 + q;
    *r = t - q * n;
    return live;
  }
};

template <bool BF16, int D, int ITERS>
__device__ __forceinline__ void write_rows(const Kv4RowsArgs& a, int64_t block) {
  constexpr int EB = BF16 ? 2 : 4;
  const Items<D, ITERS> it(a, block);
  float x[ITERS][2][8];
  int64_t base[ITERS];                   // the unit's first slot in the planes
  uint32_t slot[ITERS];
  bool live[ITERS];
#pragma unroll
  for (int k = 0; k < ITERS; ++k) {
    int64_t u;
    uint32_t r;
    live[k] = it.at(k, &u, &r);
    base[k] = u * a.slots;
    slot[k] = a.slot0 + r;
    const int64_t src = ((u * a.seq_ld + r) * D + it.lane * 8) * EB;
    kv4::load8<BF16>(static_cast<const char*>(a.k) + src, x[k][0]);
    kv4::load8<BF16>(static_cast<const char*>(a.v) + src, x[k][1]);
  }
#pragma unroll
  for (int k = 0; k < ITERS; ++k) {
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      uint32_t byte;
      const uint32_t c = kv4::quantise8(x[k][w], &byte);
      if (live[k])
        kv4::store_row<D>(w ? a.vq : a.kq, w ? a.vs : a.ks, w, base[k], slot[k], it.lane, c, byte);
    }
  }
}

template <bool BF16, int D, int ITERS>
__device__ __forceinline__ void read_rows(const Kv4RowsArgs& a, int64_t block) {
  constexpr int EB = BF16 ? 2 : 4;
  const Items<D, ITERS> it(a, block);
  uint32_t c[ITERS][2], s[ITERS][2];
  int64_t dst[ITERS];
  bool live[ITERS];
#pragma unroll
  for (int k = 0; k < ITERS; ++k) {
    int64_t u;
    uint32_t r;
    live[k] = it.at(k, &u, &r);
    const int64_t base = u * a.slots;      // the unit's first slot in the planes
    const uint32_t slot = a.slot0 + r;
    dst[k] = ((u * a.seq_ld + r) * D + it.lane * 8) * EB;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      const uint32_t at = w ? kv4::v_word<D>(slot, it.lane) : kv4::k_word<D>(slot, it.lane);
      c[k][w] = (static_cast<const uint32_t*>(w ? a.vq : a.kq) + base * (D / 8))[at];
      const uint32_t g = it.lane / 4, sat = w ? kv4::v_scale_at<D>(slot, g) : kv4::k_scale_at<D>(slot, g);
      s[k][w] = (static_cast<const uint8_t*>(w ? a.vs : a.ks) + base * (D / 32))[sat];
    }
  }
#pragma unroll
  for (int k = 0; k < ITERS; ++k) {
    if (!live[k]) continue;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      u32x4* p = reinterpret_cast<u32x4*>(const_cast<char*>(static_cast<const char*>(w ? a.v : a.k)) + dst[k]);
      const u32x4 x = kv4::bf16x8_of(c[k][w], kv4::scale_of(s[k][w]));
      if constexpr (BF16) {
        *p = x;
      } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          u32x4 y;
          y[0] = x[2 * i] << 16;
          y[1] = x[2 * i] & 0xFFFF0000u;
          y[2] = x[2 * i + 1] << 16;
          y[3] = x[2 * i + 1] & 0xFFFF0000u;
          p[i] = y;
        }
      }
    }
  }
}

// Both directions in one launch: workgroups below `reads` read rows, the others write.
template <bool BF16, int D, int ITERS>
__global__ void __launch_bounds__(256) kv4_rows_kernel(Kv4RowsArgs r, Kv4RowsArgs w, int reads) {
  if ((int)blockIdx.x < reads)
    read_rows<BF16, D, ITERS>(r, blockIdx.x);
  else
    write_rows<BF16, D, ITERS>(w, (int)blockIdx.x - reads);
}

// Row pairs of a launch from which a lane takes four: fewer leave workgroups for every
// compute unit only if it takes one.
constexpr int64_t kManyRows = 1 << 16;

template <bool BF16, int D, int ITERS>
hipError_t launch_i(const Kv4RowsArgs& r, const Kv4RowsArgs& w, hipStream_t stream) {
  constexpr int64_t per = Items<D, ITERS>::kRows * ITERS;
  const int64_t reads = ((int64_t)r.units * r.n + per - 1) / per;
  const int64_t blocks = reads + ((int64_t)w.units * w.n + per - 1) / per;
  if (blocks > 0xFFFFFF) return hipErrorInvalidValue;   // 2^32 threads a launch
  hipLaunchKernelGGL((kv4_rows_kernel<BF16, D, ITERS>), dim3((unsigned)blocks), dim3(256), 0, stream, r, w,
                     (int)reads);
  return hipGetLastError();
}

template <bool BF16, int D>
hipError_t launch_t(const Kv4RowsArgs& r, const Kv4RowsArgs& w, hipStream_t stream) {
  const bool many = (int64_t)r.units * r.n + (int64_t)w.units * w.n >= kManyRows;
  return many ? launch_i<BF16, D, 4>(r, w, stream) : launch_i<BF16, D, 1>(r, w, stream);
}

}  // namespace

hipError_t launch_kv4_rows(const Kv4RowsArgs& r, const Kv4RowsArgs& w, int dtype, int head_dim,
                           hipStream_t stream) {
  if (dtype == BM_BF16)
    return head_dim == 128 ? launch_t<true, 128>(r, w, stream) : launch_t<true, 64>(r, w, stream);
  return head_dim == 128 ? launch_t<false, 128>(r, w, stream) : launch_t<false, 64>(r, w, stream);
}

}  // namespace bm
