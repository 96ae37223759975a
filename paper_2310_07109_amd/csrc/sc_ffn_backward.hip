// The gated feed-forward block, backward (the products are in sc_ffn.h).
#include <algorithm>

#include "sc_ffn.h"

namespace sc {
namespace {

struct BackwardWs {
  int *count, *map;
  char *x, *dy, *w[3], *dg, *du;
  float *part_d, *part_gu;
};

// The weight gradients' sums over rows, cut into slabs so that every workgroup has a tile.
constexpr int kMostSlabs = 16;
FfnPlan weight_plan(const Ffn& a, int mats) {
  const long long T = (long long)a.B * a.n;
  return ffn_plan(a.D, (long long)mats * a.F, (T + 63) / 64, kMostSlabs);
}

size_t carve(const Ffn& a, void* base, BackwardWs* out) {
  const size_t T = (size_t)a.B * a.n, Dp = up8(a.D), Fp = up8(a.F), DF = (size_t)a.D * a.F;
  FfnCarve c{static_cast<char*>(base)};
  BackwardWs s = {};
  if (a.len) {
    s.count = reinterpret_cast<int*>(c.take(4));
    s.map = reinterpret_cast<int*>(c.take(4 * T));
  }
  if (a.len || ffn_odd(a)) {
    s.x = c.take(T * Dp * 2);
    s.dy = c.take(T * Dp * 2);
  }
  if (ffn_odd(a)) {
    s.w[0] = c.take(a.D * Fp * 2);
    s.w[1] = c.take(a.D * Fp * 2);
    s.w[2] = c.take(a.F * Dp * 2);
  }
  s.dg = c.take(T * Fp * 2);
  s.du = c.take(T * Fp * 2);
  const int sd = weight_plan(a, 1).slabs, sg = weight_plan(a, 2).slabs;
  if (sd > 1) s.part_d = reinterpret_cast<float*>(c.take(4 * DF * sd));
  if (sg > 1) s.part_gu = reinterpret_cast<float*>(c.take(4 * DF * 2 * sg));
  if (out) *out = s;
  return c.off;
}

// The slabs' sums, in order, rounded once: up to three gradients of `count` elements.  HBM
// bounds it: five slabs each of dWd, dWg and dWu of 1024 x 2816, 173 MB, 31 us.
struct SlabSums {
  const float* part[3];
  __bf16* out[3];
  int slabs[3];
  long long count;
};
__global__ __launch_bounds__(256) void k_ffn_slabs(SlabSums a) {
  const int m = blockIdx.y;
  const float* p = a.part[m];
  __bf16* o = a.out[m];
  if (!o) return;
  const long long step = (long long)gridDim.x * 1024;
  for (long long i = ((long long)blockIdx.x * 256 + threadIdx.x) * 4; i < a.count; i += step) {
    if (i + 4 <= a.count) {
      f32x4 s = *reinterpret_cast<const f32x4_any*>(p + i);
      for (int k = 1; k < a.slabs[m]; ++k) s += *reinterpret_cast<const f32x4_any*>(p + k * a.count + i);
      *reinterpret_cast<u32x2_any*>(o + i) = u32x2_any{pack_bf16(s[0], s[1]), pack_bf16(s[2], s[3])};
    } else {
      for (long long q = i; q < a.count; ++q) {
        float s = p[q];
        for (int k = 1; k < a.slabs[m]; ++k) s += p[k * a.count + q];
        o[q] = (__bf16)s;
      }
    }
  }
}

}  // namespace

size_t ffn_backward_workspace_bytes(const Ffn& a) { return carve(a, nullptr, nullptr); }

hipError_t launch_ffn_backward(const Ffn& a, hipStream_t s) {
  const long long T = (long long)a.B * a.n, DF = (long long)a.D * a.F;
  const int Dp = up8(a.D), Fp = up8(a.F);
  const bool odd = ffn_odd(a);
  BackwardWs ws;
  carve(a, a.ws, &ws);
  const char *x = static_cast<const char*>(a.x), *dy = static_cast<const char*>(a.dy),
             *wg = static_cast<const char*>(a.wg), *wu = static_cast<const char*>(a.wu),
             *wd = static_cast<const char*>(a.wd);
  hipError_t e;
  if (a.len || odd) {
    FfnRows r = {};
    r.len = a.len;
    r.B = a.B;
    r.n = a.n;
    r.map = ws.map;
    r.count = ws.count;
    r.zero = static_cast<char*>(a.dx);
    r.zero_bytes = 2LL * a.D;
    r.always = odd;
    r.copies = 2;
    r.copy[0] = {x, ws.x, 0, a.D, Dp};
    r.copy[1] = {dy, ws.dy, 0, a.D, Dp};
    if (odd) {
      r.copies = 5;
      r.copy[2] = {wg, ws.w[0], a.D, a.F, Fp};
      r.copy[3] = {wu, ws.w[1], a.D, a.F, Fp};
      r.copy[4] = {wd, ws.w[2], a.F, a.D, Dp};
      x = ws.x;
      dy = ws.dy;
      wg = ws.w[0];
      wu = ws.w[1];
      wd = ws.w[2];
    }
    e = launch_ffn_rows(&r, s);
    if (e != hipSuccess) return e;
  }
  const FfnSaved sv = ffn_saved(a, const_cast<void*>(a.saved));
  const FfnOperand opx = {{x, nullptr}, ws.x, 2u * Dp, 0}, opdy = {{dy, nullptr}, ws.dy, 2u * Dp, 0};
  FfnArgs base = {};
  base.T = (int)T;
  base.count = ws.count;
  FfnArgs dh = base, dx = base, dwd = base, dwgu = base;
  SlabSums sums = {};
  sums.count = DF;
  const bool need_dh = a.dx || a.dwg || a.dwu;
  const FfnSize size_h = {T, Fp, (Dp + 63) / 64, true}, size_x = {T, a.D, 2 * ((Fp + 63) / 64), false},
                size_d = {a.D, a.F, (T + 63) / 64, false}, size_gu = {a.D, 2LL * a.F, (T + 63) / 64, false};
  const FfnPlan plan_h = ffn_plan(size_h.rows, size_h.cols, size_h.stages, 1, true),
                plan_x = ffn_plan(size_x.rows, size_x.cols, size_x.stages, 1), plan_d = weight_plan(a, 1),
                plan_gu = weight_plan(a, 2);
  const FfnTwoPlan two_h = ffn_plan_two(size_h, plan_h, size_d, plan_d),
                   two_x = ffn_plan_two(size_x, plan_x, size_gu, plan_gu);
  dh.a = opdy;
  dh.b = {{wd, nullptr}, nullptr, 2u * Dp, a.F};
  dh.N = Fp;
  dh.K = Dp;
  dh.out[0] = ws.dg;
  dh.out[1] = ws.du;
  dh.ld = Fp;
  dh.blocks = sv.blocks;
  dh.across = (Fp + 31) / 32;
  dx.map = ws.map;
  dx.a = {{ws.dg, ws.du}, nullptr, 2u * Fp, 0};
  dx.b = {{wg, wu}, nullptr, 2u * Fp, a.D};
  dx.N = a.D;
  dx.K = Fp;
  dx.out[0] = a.dx;
  dx.ld = a.D;
  dwd.a = {{sv.h, nullptr}, nullptr, 2u * Fp, 0};
  dwd.b = opdy;
  dwd.M = a.F;
  dwd.N = a.D;
  dwd.out[0] = a.dwd;
  dwd.ld = a.D;
  dwd.slabs = plan_d.slabs;
  dwd.part = ws.part_d;
  dwgu.a = opx;
  dwgu.b = {{ws.dg, ws.du}, nullptr, 2u * Fp, 0};
  dwgu.M = a.D;
  dwgu.N = a.F;
  dwgu.out[0] = a.dwg;
  dwgu.out[1] = a.dwu;
  dwgu.ld = a.F;
  dwgu.slabs = plan_gu.slabs;
  dwgu.part = ws.part_gu;
  if (a.dwd && dwd.slabs > 1) {
    sums.part[0] = ws.part_d;
    sums.out[0] = static_cast<__bf16*>(a.dwd);
    sums.slabs[0] = dwd.slabs;
  }
  if (dwgu.slabs > 1)
    for (int i = 0; i < 2; ++i) {
      sums.part[1 + i] = ws.part_gu + i * dwgu.slabs * DF;
      sums.out[1 + i] = static_cast<__bf16*>(i ? a.dwu : a.dwg);
      sums.slabs[1 + i] = dwgu.slabs;
    }
  if (need_dh && a.dwd && two_h.tile >= 0) {
    e = run_ffn_two<kDh, kDwd>(dh, dwd, two_h.tile, two_h.ratio, s);
    if (e != hipSuccess) return e;
  } else {
    if (need_dh) {
      e = run_ffn<kDh, kActNone>(dh, plan_h.tile, s);
      if (e != hipSuccess) return e;
    }
    if (a.dwd) {
      e = run_ffn<kDwd, kActNone>(dwd, plan_d.tile, s);
      if (e != hipSuccess) return e;
    }
  }
  if (a.dx && a.dwg && a.dwu && two_x.tile >= 0) {
    e = run_ffn_two<kDx, kDwgu>(dx, dwgu, two_x.tile, two_x.ratio, s);
    if (e != hipSuccess) return e;
  } else {
    if (a.dx) {
      e = run_ffn<kDx, kActNone>(dx, plan_x.tile, s);
      if (e != hipSuccess) return e;
    }
    if (a.dwg || a.dwu) {
      e = run_ffn<kDwgu, kActNone>(dwgu, plan_gu.tile, s);
      if (e != hipSuccess) return e;
    }
  }
  if (sums.out[0] || sums.out[1] || sums.out[2]) {
    hipLaunchKernelGGL(k_ffn_slabs, dim3((unsigned)std::min<long long>((DF + 1023) / 1024, 1024), 3), dim3(256), 0, s,
                       sums);
    return hipGetLastError();
  }
  return hipSuccess;
}

}  // namespace sc
