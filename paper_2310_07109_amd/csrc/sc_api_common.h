// What the C entry points share: overlap checks, workspace carving and the debug
// build's device-side checks.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/sc.h"
#include "sc_internal.h"

namespace {

bool overlaps(const void* a, size_t na, const void* b, size_t nb) {
  if (!a || !b || na == 0 || nb == 0) return false;
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + nb && y < x + na;
}

size_t elem_size(int dtype) { return dtype == SC_BF16 ? 2 : 4; }

// Carves 256-byte aligned pieces out of the caller's workspace.
struct Carver {
  char* base;
  size_t off = 0;
  explicit Carver(void* p) : base(static_cast<char*>(p)) {}
  template <typename T>
  T* take(size_t count) {
    off = (off + 255) & ~size_t(255);
    T* p = base ? reinterpret_cast<T*>(base + off) : nullptr;
    off += count * sizeof(T);
    return p;
  }
};

#ifdef SC_DEBUG
}  // namespace
// The device word of the descriptor check.
static __device__ int32_t g_debug_err;
namespace {
// Debug build: before an entry point enqueues anything, its descriptor's
// device-resident arrays are checked and the stream drained; then the entry
// point's own work is waited for and a failed launch or execution reported.
sc_status debug_rows(const int32_t* valid_len, const int32_t* gpos, int B, int n, int G, void* stream) {
  int32_t* err = nullptr;
  if (hipGetSymbolAddress(reinterpret_cast<void**>(&err), HIP_SYMBOL(g_debug_err)) != hipSuccess || !err)
    return SC_EHIP;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (sc::launch_validate_desc(valid_len, gpos, B, n, G, err, s) != hipSuccess) return SC_EHIP;
  int32_t bits = 0;
  if (hipMemcpyAsync(&bits, err, sizeof(bits), hipMemcpyDeviceToHost, s) != hipSuccess ||
      hipStreamSynchronize(s) != hipSuccess)
    return SC_EHIP;
  return bits != 0 ? SC_EINVAL : SC_OK;
}

sc_status debug_post(sc_status st, void* stream) {
  if (st != SC_OK) return st;
  if (hipStreamSynchronize(static_cast<hipStream_t>(stream)) != hipSuccess || hipGetLastError() != hipSuccess)
    return SC_EHIP;
  return SC_OK;
}
#endif

}  // namespace

#ifdef SC_DEBUG
#define SC_DEBUG_RUN(pre, stream, call)    \
  do {                                     \
    const sc_status pre_ = (pre);          \
    if (pre_ != SC_OK) return pre_;        \
    return debug_post(call, stream);       \
  } while (0)
#endif
