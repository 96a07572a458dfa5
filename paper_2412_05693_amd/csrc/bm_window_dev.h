// Where the tokens of a window cache lie (bm_window.h), and who sees them.  An index is a
// token's position less its sample's left pad.
#pragma once

#include <hip/hip_runtime.h>

namespace bm {

// The index of the token at position pos <= 2^30 of a sample with that many pads.  One that is
// more than 2^30 before its sample's beginning (a sample that never begins) stays there: no
// token of a call comes up to index 0 then, and sums with sizes hold in 32 bits.
__host__ __device__ __forceinline__ int index_of(int pos, int pad) {
  const int i = pos - pad;
  return i < -(1 << 30) ? -(1 << 30) : i;
}

// Row r of those that the store of a call's n_tok tokens looks at: its token, or -1 if the cache
// keeps none for it.  r0: the index of the call's first token; the call's last tokens, as
// many as the window takes, come behind `lead` possible sinks among the others.
__host__ __device__ __forceinline__ int kept_token(int r, int lead, int n_tok, int window, int sinks, int r0) {
  const int first = n_tok > window ? n_tok - window : 0;    // the first token kept for the window
  const int t = r < lead ? (r0 < 0 ? -r0 : 0) + r : first + r - lead;
  if (r0 + t < 0 || (r < lead && (r0 + t >= sinks || t >= first))) return -1;
  return t;
}

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

}  // namespace bm
