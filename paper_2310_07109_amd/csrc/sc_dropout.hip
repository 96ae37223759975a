// Dropout with a residual sum; the mask comes from a counter and is never stored.
//
//   out = res_scale * residual + (r >= t ? x * s : 0),  s = 65536 / (65536 - t),
// r: 16 bits an element of Philox4x32-10 (Salmon, Moraes, Dror, Shaw, "Parallel random
// numbers: as easy as 1, 2, 3", 2011), one call of it for eight channels of a row.
//
// A read of x (and the residual) and a write of out bound it, with the generator's twenty
// 32 x 32 -> 64 bit products for eight elements beside them: at 16 bits an element both
// take about as long, at 32 the products alone would.  32768 x 1024 bf16 with a residual, 30 us
// for 201 MB, 38 among other work (part of the rows lie in the last-level cache); 1503 x 1111
// float32, ragged, 5.
#include <algorithm>

#include "sc_device.h"
#include "sc_internal.h"

namespace sc {
namespace {

typedef __attribute__((ext_vector_type(4))) unsigned u32x4;

// The four words of a counter under a key.
SC_DEV u32x4 philox(unsigned c0, unsigned c1, unsigned c2, unsigned c3, unsigned k0, unsigned k1) {
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const unsigned long long p = (unsigned long long)c0 * 0xD2511F53u, q = (unsigned long long)c2 * 0xCD9E8D57u;
    const unsigned n0 = (unsigned)(q >> 32) ^ c1 ^ k0, n2 = (unsigned)(p >> 32) ^ c3 ^ k1;
    c1 = (unsigned)q;
    c3 = (unsigned)p;
    c0 = n0;
    c2 = n2;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return u32x4{c0, c1, c2, c3};
}

typedef u32x4 __attribute__((aligned(2))) u32x4_any;

// Eight elements at any element's address (the hardware takes 16 bytes there).
template <typename T>
struct Eight {
  typedef u32x4_any Vec;
  static constexpr int kVecs = (int)sizeof(T) / 2;
  u32x4 u[kVecs];
  SC_DEV void load(const T* p, int count) {
    if (count >= 8) {
#pragma unroll
      for (int i = 0; i < kVecs; ++i) u[i] = reinterpret_cast<const Vec*>(p)[i];
    } else {
      T e[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) e[i] = i < count ? p[i] : (T)0.f;
      __builtin_memcpy(u, e, sizeof(e));
    }
  }
  SC_DEV void store(T* p, int count) const {
    if (count >= 8) {
#pragma unroll
      for (int i = 0; i < kVecs; ++i) reinterpret_cast<Vec*>(p)[i] = u[i];
    } else {
      T e[8];
      __builtin_memcpy(e, u, sizeof(e));
#pragma unroll
      for (int i = 0; i < 7; ++i)
        if (i < count) p[i] = e[i];
    }
  }
  SC_DEV float at(int i) const {
    const unsigned w = sizeof(T) == 4 ? u[i / 4 % kVecs][i % 4]
                       : i & 1        ? u[0][i / 2] & 0xffff0000u
                                      : u[0][i / 2] << 16;
    return __builtin_bit_cast(float, w);
  }
  SC_DEV void set(const float (&v)[8]) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < 8; ++i) u[i / 4][i % 4] = __builtin_bit_cast(unsigned, v[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) u[0][i] = pack_bf16(v[2 * i], v[2 * i + 1]);
    }
  }
};

// Groups of eight channels (`per` a row), numbered through the batch and dealt to the
// threads in turn; a thread steps from one to the next without a division.
template <typename T>
__global__ __launch_bounds__(256) void k_dropout(Dropout a, unsigned per, long long groups) {
  const long long step = (long long)gridDim.x * 256;
  long long i = (long long)blockIdx.x * 256 + threadIdx.x;
  if (i >= groups) return;
  const unsigned long long key = *reinterpret_cast<const unsigned long long*>(a.seed);
  const unsigned k0 = (unsigned)key, k1 = (unsigned)(key >> 32);
  unsigned row = (unsigned)(i / per), g = (unsigned)(i - (long long)row * per);
  const unsigned drow = (unsigned)(step / per), dg = (unsigned)(step - (long long)drow * per);
  const unsigned n = (unsigned)a.n;
  unsigned b = row / n, j = row - b * n;
  const unsigned db = drow / n, dj = drow - db * n;
  for (; i < groups; i += step) {
    const long long at = (long long)row * a.D + 8 * g;
    const int count = a.D - (int)(8 * g);
    Eight<T> x, o;
    const bool live = !a.len || (int)j < clampi(a.len[b], 0, a.n);
    float v[8];
    if (live) {
      x.load(static_cast<const T*>(a.x) + at, count);
      Eight<T> res;
      if (a.residual) res.load(static_cast<const T*>(a.residual) + at, count);
      const u32x4 w = philox(g, j, b, (unsigned)a.site, k0, k1);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const unsigned r = e & 1 ? w[e / 2] >> 16 : w[e / 2] & 0xffffu;
        const float s = r >= a.threshold ? x.at(e) * a.scale : 0.f;
        v[e] = a.residual ? fmaf(a.res_scale, res.at(e), s) : s;
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = 0.f;
    }
    o.set(v);
    o.store(static_cast<T*>(a.out) + at, count);
    g += dg;
    row += drow;
    j += dj;
    b += db;
    if (g >= per) {
      g -= per;
      ++row;
      ++j;
    }
    if (j >= n) {
      j -= n;
      ++b;
    }
  }
}

}  // namespace

hipError_t launch_dropout(const Dropout& a, hipStream_t s) {
  const unsigned per = (unsigned)(((long long)a.D + 7) / 8);
  const long long groups = (long long)a.B * a.n * per;
  const dim3 grid((unsigned)std::min<long long>((groups + 255) / 256, 8192)), block(256);
  if (a.f32)
    hipLaunchKernelGGL(k_dropout<float>, grid, block, 0, s, a, per, groups);
  else
    hipLaunchKernelGGL(k_dropout<__bf16>, grid, block, 0, s, a, per, groups);
  return hipGetLastError();
}

}  // namespace sc
