// The gated feed-forward block, forward: y = (act(x Wg) * (x Wu)) Wd.  The products are in
// sc_ffn.h; the matrix units bound them where there are rows, the weights' bytes where
// there are few.
#include <algorithm>

#include "sc_ffn.h"

namespace sc {
namespace {

// A wavefront a row: of the batch, then of the weights.
__global__ __launch_bounds__(256) void k_ffn_rows(FfnRows a) {
  __shared__ int pre[kPackMaxB + 1];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const long long T = (long long)a.B * a.n;
  int R = (int)T;
  if (a.len) {
    pack_prefix(pre, a.len, a.B, a.n);
    __syncthreads();
    R = __builtin_amdgcn_readfirstlane(pre[a.B]);
    if (blockIdx.x == 0 && threadIdx.x == 0) a.count[0] = R;
  }
  auto copy = [&](const FfnCopy& c, long long from, long long to) {
    const __bf16* s = reinterpret_cast<const __bf16*>(c.src) + from * c.cols;
    __bf16* d = reinterpret_cast<__bf16*>(c.dst) + to * c.pitch;
    for (int i = 8 * lane; i < c.pitch; i += 512) {
      u32x4 v = {0, 0, 0, 0};
      if (i + 8 <= c.cols) {
        v = *reinterpret_cast<const u32x4_any*>(s + i);
      } else {
#pragma unroll
        for (int q = 0; q < 8; ++q)
          if (i + q < c.cols)
            v[q / 2] |= (unsigned)__builtin_bit_cast(unsigned short, s[i + q]) << (16 * (q & 1));
      }
      *reinterpret_cast<u32x4*>(d + i) = v;
    }
  };
  const bool rows = a.always || R != T;
  const long long step = (long long)gridDim.x * 4;
  for (long long r = (long long)blockIdx.x * 4 + w; r < T; r += step) {
    const int b = (int)(r / a.n), j = (int)(r - (long long)b * a.n);
    long long to = r;
    if (a.len) {
      const int first = pre[b];
      if (j >= pre[b + 1] - first) {
        if (a.zero) {
          char* z = a.zero + r * a.zero_bytes;
          for (long long c = 16 * lane; c < a.zero_bytes; c += 1024) {
            if (c + 16 <= a.zero_bytes) *reinterpret_cast<u32x4_any*>(z + c) = u32x4_any{0, 0, 0, 0};
            else
              for (long long i = c; i < a.zero_bytes; i += 2) *reinterpret_cast<unsigned short*>(z + i) = 0;
          }
        }
        continue;
      }
      to = first + j;
      if (lane == 0) a.map[to] = (int)r;
    }
    if (!rows) continue;
    for (int i = 0; i < a.copies; ++i)
      if (a.copy[i].rows == 0) copy(a.copy[i], r, to);
  }
  for (int i = 0; i < a.copies; ++i)
    for (long long r = (long long)blockIdx.x * 4 + w; r < a.copy[i].rows; r += step) copy(a.copy[i], r, r);
}

struct ForwardWs {
  int *count, *map;
  char *x, *w[3], *h;
};
size_t carve(const Ffn& a, void* base, bool save, ForwardWs* out) {
  const size_t T = (size_t)a.B * a.n, Dp = up8(a.D), Fp = up8(a.F);
  FfnCarve c{static_cast<char*>(base)};
  ForwardWs s = {};
  if (a.len) {
    s.count = reinterpret_cast<int*>(c.take(4));
    s.map = reinterpret_cast<int*>(c.take(4 * T));
  }
  if (ffn_odd(a)) {
    s.x = c.take(T * Dp * 2);
    s.w[0] = c.take(a.D * Fp * 2);
    s.w[1] = c.take(a.D * Fp * 2);
    s.w[2] = c.take(a.F * Dp * 2);
  }
  if (!save) s.h = c.take(T * Fp * 2);
  if (out) *out = s;
  return c.off;
}

template <int kAct>
hipError_t gate(const FfnArgs& g, int tile, hipStream_t s) {
  return g.blocks ? run_ffn<kGateKeep, kAct>(g, tile, s) : run_ffn<kGate, kAct>(g, tile, s);
}

}  // namespace

hipError_t launch_ffn_rows(const void* rows, hipStream_t s) {
  const FfnRows& r = *static_cast<const FfnRows*>(rows);
  long long most = (long long)r.B * r.n;
  for (int i = 0; i < r.copies; ++i) most = std::max<long long>(most, r.copy[i].rows);
  hipLaunchKernelGGL(k_ffn_rows, dim3((unsigned)std::min<long long>((most + 3) / 4, 1024)), dim3(256), 0, s, r);
  return hipGetLastError();
}

size_t ffn_saved_bytes(const Ffn& a) { return ffn_saved(a, nullptr).bytes; }
size_t ffn_workspace_bytes(const Ffn& a, bool save) { return carve(a, nullptr, save, nullptr); }

hipError_t launch_ffn(const Ffn& a, hipStream_t s) {
  const long long T = (long long)a.B * a.n;
  const int Dp = up8(a.D), Fp = up8(a.F);
  const bool odd = ffn_odd(a);
  ForwardWs ws;
  carve(a, a.ws, a.saved != nullptr, &ws);
  const char *x = static_cast<const char*>(a.x), *wg = static_cast<const char*>(a.wg),
             *wu = static_cast<const char*>(a.wu), *wd = static_cast<const char*>(a.wd);
  if (a.len || odd) {
    FfnRows r = {};
    r.len = a.len;
    r.B = a.B;
    r.n = a.n;
    r.map = ws.map;
    r.count = ws.count;
    r.zero = static_cast<char*>(a.y);
    r.zero_bytes = 2LL * a.D;
    r.always = odd;
    if (odd) {
      r.copies = 4;
      r.copy[0] = {x, ws.x, 0, a.D, Dp};
      r.copy[1] = {wg, ws.w[0], a.D, a.F, Fp};
      r.copy[2] = {wu, ws.w[1], a.D, a.F, Fp};
      r.copy[3] = {wd, ws.w[2], a.F, a.D, Dp};
      x = ws.x;
      wg = ws.w[0];
      wu = ws.w[1];
      wd = ws.w[2];
    }
    const hipError_t e = launch_ffn_rows(&r, s);
    if (e != hipSuccess) return e;
  }
  char* h = ws.h;
  FfnArgs g = {};
  g.T = (int)T;
  g.count = ws.count;
  g.map = ws.map;
  g.map_a = ws.map != nullptr && !odd;
  if (a.saved) {
    const FfnSaved sv = ffn_saved(a, a.saved);
    h = sv.h;
    g.blocks = sv.blocks;
    g.across = (Fp + 31) / 32;
  }
  g.a = {{x, nullptr}, nullptr, 2u * Dp, g.map_a ? (int)T : 0};
  g.b = {{wg, wu}, nullptr, 2u * Fp, a.D};
  g.N = Fp;
  g.K = Dp;
  g.out[0] = h;
  g.ld = Fp;
  const int tile = ffn_plan(T, 2LL * Fp, (Dp + 63) / 64, 1).tile;
  const hipError_t e = a.act == kActGelu   ? gate<kActGelu>(g, tile, s)
                       : a.act == kActSilu ? gate<kActSilu>(g, tile, s)
                                           : gate<kActNone>(g, tile, s);
  if (e != hipSuccess) return e;
  FfnArgs d = {};
  d.T = (int)T;
  d.count = ws.count;
  d.map = ws.map;
  d.a = {{h, nullptr}, nullptr, 2u * Fp, 0};
  d.b = {{wd, nullptr}, nullptr, 2u * Dp, a.F};
  d.N = a.D;
  d.K = Fp;
  d.out[0] = a.y;
  d.ld = a.D;
  return run_ffn<kDown, kActNone>(d, ffn_plan(T, a.D, (Fp + 63) / 64, 1).tile, s);
}

}  // namespace sc
