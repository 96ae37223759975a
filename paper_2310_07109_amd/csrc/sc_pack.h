// Numbering of the packed rows, shared by the products and the row kernels
// around them, and the waits on loads in flight.
#pragma once
#include "sc_device.h"

namespace sc {

// Packed rows.  The surviving rows of all sequences are numbered in sequence
// order (packed row p of sequence b is its row p - pre[b], pre = exclusive
// prefix sum of the lengths), so that the products run on ceil(R / BM) tiles
// of R = sum of the lengths rows instead of one partly empty tile per
// sequence and 128 rows.  Every workgroup derives the numbering from the
// lengths itself: the host never learns them.

// Wave 0 writes pre[0 .. B] (pre[B] = R); lengths clamped to [0, n], all n
// without lengths.
SC_DEV void pack_prefix(int* pre, const int* len, int B, int n) {
  if (threadIdx.x >= 64) return;
  const int lane = threadIdx.x;
  int carry = 0;
  for (int c = 0; c < B; c += 64) {
    const int b = c + lane;
    const int v = b < B ? (len ? clampi(len[b], 0, n) : n) : 0;
    const int incl = prefix_sum(v);
    if (b < B) pre[b] = carry + incl - v;
    carry += __builtin_amdgcn_readlane(incl, 63);
  }
  if (lane == 0) pre[B] = carry;
}

// The sequence holding packed row p < pre[B]: the largest b with pre[b] <= p
// (empty sequences share their start with the next one).
SC_DEV int pack_seq(const int* pre, int B, int p) {
  int lo = 0, hi = B - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (pre[mid] <= p) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// s_waitcnt vmcnt(n) alone (expcnt and lgkmcnt at their no-wait maxima)
template <int N>
SC_DEV void wait_vm() {
  static_assert(N >= 0 && N < 64, "vmcnt range");
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4) | (15 << 8));
}

// Waits until at most `later` (< kNBuf) stages of kPer loads and kExtra newer
// accesses are in flight.
template <int kNBuf, int kPer, int kExtra = 0, int kL = kNBuf - 1>
SC_DEV void wait_stages(int later) {
  if constexpr (kL == 0) {
    wait_vm<kExtra>();
  } else {
    if (later >= kL) wait_vm<kL * kPer + kExtra>();
    else wait_stages<kNBuf, kPer, kExtra, kL - 1>(later);
  }
}

}  // namespace sc
