// Where the tokens of a window cache lie (bm_window.h), and who sees them.  An index is a
// token's position less its sample's left pad.
#pragma once

#include <hip/hip_runtime.h>

namespace bm {

// the slot of the token at index i >= 0
__device__ __forceinline__ int window_slot(int i, int sinks, int window) {
  return i < sinks ? i : sinks + (i - sinks) % window;
}

// What lies in a window cache before the token at index `end`.
struct Ring {
  int end, sinks, window;
  int last;    // the place of the last token behind the sinks, counted from the first such slot
  __device__ __forceinline__ Ring(int end, int sinks, int window)
      : end(end), sinks(sinks), window(window), last(end > sinks ? (end - sinks - 1) % window : 0) {}
  // slots that hold a token
  __device__ __forceinline__ int filled() const { return min(max(end, 0), sinks + window); }
  // index of the token in a slot, -1 if there is none
  __device__ __forceinline__ int index(int slot) const {
    if (slot < sinks) return slot < end ? slot : -1;
    const int back = last - (slot - sinks);      // tokens between that one and the last
    const int i = end - 1 - (back < 0 ? back + window : back);
    return i >= sinks ? i : -1;
  }
};

// whether the token at index i >= 0 sees the one at index j
__device__ __forceinline__ bool window_sees(int i, int j, int sinks, int window) {
  return j >= 0 && j <= i && (j < sinks || i - j < window);
}

}  // namespace bm
