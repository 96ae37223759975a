// Rotary positions of queries and keys, with their norms per head.
//
//   u = norm(x) * w;  (a, b) -> A (a cos phi - b sin phi, a sin phi + b cos phi),
//   phi = p f_i; backward: the rotation by -phi, then the norm's gradient
//   dx = inv (g - hat mean(g hat) - mean(g)),  g = w du,  hat = (x - mean) inv
//   (mean only for LayerNorm), dw = sum du hat.
//
// One read and one write of every head bound it.  A lane holds eight pairs of a head,
// both halves of each, so the rotation is within a lane and d / 16 lanes (rounded up
// to a power of two) hold a head; its sums go over them by DPP.
//
// The angles of a token serve all its heads: a workgroup makes the cosines and sines
// of its tokens once, in LDS.  An angle is a turn in 64-bit fixed point: position times
// frequency modulo 2^64 is exact in integers whatever the position, and what is left is
// at most an eighth of a turn for a polynomial.
#include <algorithm>

#include "sc_device.h"
#include "sc_internal.h"

namespace sc {
namespace {

typedef __attribute__((ext_vector_type(4))) unsigned u32x4;

constexpr int kThreads = 256;
constexpr int kMaxTokens = 16;  // of a workgroup at a time

struct RotaryArgs {
  const char *x[3], *g[3];  // q, k, v and, backward, the gradients of the outputs
  char *o[3];               // outputs
  long long xs[3], gs[3], os[3];  // bytes between tokens
  const float* w[2];
  const int* len;
  const int* pos;
  float* part;  // backward: [workgroups, 2, d] sums of the weights' gradients, or null
  int B, n, heads, h1, h2;  // heads: of a token in all; h1, h2: the first key and value head
  int d, R, lanes;          // lanes of a head
  int tokens, interleaved, norm, rms;
  float eps, amplitude;
  RotaryTurns turns;
};

// cos and sin of `turn` / 2^32 of a turn: the quadrant by integers, the rest (at most an
// eighth of a turn) by the Taylor series, cut below 2^-27.
SC_DEV void cos_sin(unsigned turn, float& c, float& s) {
  const unsigned q = (turn + 0x20000000u) >> 30;
  const float x = (float)(int)(turn - (q << 30)) * 1.4629180792671596e-09f;  // 2 pi / 2^32
  const float x2 = x * x;
  float a = fmaf(x2, 2.7557319223985893e-06f, -0.0001984126984126984f);
  a = fmaf(a, x2, 0.008333333333333333f);
  a = fmaf(a, x2, -0.16666666666666666f);
  a = fmaf(a * x2, x, x);
  float b = fmaf(x2, -2.7557319223985888e-07f, 2.48015873015873e-05f);
  b = fmaf(b, x2, -0.001388888888888889f);
  b = fmaf(b, x2, 0.041666666666666664f);
  b = fmaf(b, x2, -0.5f);
  b = fmaf(b, x2, 1.f);
  const bool odd = q & 1;
  c = odd ? a : b;
  s = odd ? b : a;
  if (q == 1 || q == 2) c = -c;
  if (q >= 2) s = -s;
}

// Sum over the `lanes` (a power of two up to 16) neighbours that hold a head.
SC_DEV float head_sum(float v, int lanes) {
  if (lanes > 1) v += dpp<kDppXor1>(v);
  if (lanes > 2) v += dpp<kDppXor2>(v);
  if (lanes > 4) v += dpp<kDppHalfMirror>(v);
  if (lanes > 8) v += dpp<kDppMirror>(v);
  return v;
}

// Eight pairs of a head, pair i at elements e0 + i, e1 + i (half) or e0 + 2 i,
// e0 + 2 i + 1 (interleaved).
template <typename T, bool kVec>
struct Pairs {
  float a[8], b[8];
  SC_DEV static float one(const T* p) { return (float)*p; }
  SC_DEV static void vec(const T* p, float* v) {  // eight elements at 16 bytes
    if constexpr (sizeof(T) == 4) {
      const f32x4 lo = *reinterpret_cast<const f32x4*>(p), hi = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = lo[i], v[4 + i] = hi[i];
    } else {
      const u32x4 u = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[2 * i] = __builtin_bit_cast(float, u[i] << 16);
        v[2 * i + 1] = __builtin_bit_cast(float, u[i] & 0xffff0000u);
      }
    }
  }
  SC_DEV static void put(T* p, const float* v) {
    if constexpr (sizeof(T) == 4) {
      *reinterpret_cast<f32x4*>(p) = f32x4{v[0], v[1], v[2], v[3]};
      *reinterpret_cast<f32x4*>(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
    } else {
      *reinterpret_cast<u32x4*>(p) =
          u32x4{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
    }
  }
};

// Where a lane's pairs are: pair i (of the lane) is live below `live`, rotated below
// `rot`; elements first(i) and second(i).
struct Place {
  int p0, live, rot, R2, d2, R, interleaved;
  SC_DEV Place(int d, int R_, int inter, int sub)
      : p0(8 * sub), live(d / 2 - 8 * sub), rot(R_ / 2 - 8 * sub), R2(R_ / 2), d2(d / 2), R(R_), interleaved(inter) {}
  SC_DEV int first(int i) const {
    const int p = p0 + i;
    return interleaved ? 2 * p : i < rot ? p : p + R2;  // passed pair q = p - R2: element R + q
  }
  SC_DEV int second(int i) const {
    const int p = p0 + i;
    return interleaved ? 2 * p + 1 : i < rot ? p + R2 : p + d2;  // R + (d - R) / 2 + q
  }
};

template <typename T, bool kVec>
SC_DEV void load_pairs(Pairs<T, kVec>& v, const T* x, const Place& pl) {
  if constexpr (kVec) {
    if (pl.live > 0) {
      if (pl.interleaved) {
        float t[16];
        Pairs<T, kVec>::vec(x + pl.first(0), t);
        Pairs<T, kVec>::vec(x + pl.first(0) + 8, t + 8);
#pragma unroll
        for (int i = 0; i < 8; ++i) v.a[i] = t[2 * i], v.b[i] = t[2 * i + 1];
      } else {
        Pairs<T, kVec>::vec(x + pl.first(0), v.a);
        Pairs<T, kVec>::vec(x + pl.second(0), v.b);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v.a[i] = v.b[i] = 0.f;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v.a[i] = i < pl.live ? (float)x[pl.first(i)] : 0.f;
      v.b[i] = i < pl.live ? (float)x[pl.second(i)] : 0.f;
    }
  }
}

template <typename T, bool kVec>
SC_DEV void store_pairs(const Pairs<T, kVec>& v, T* x, const Place& pl) {
  if constexpr (kVec) {
    if (pl.live <= 0) return;
    if (pl.interleaved) {
      float t[16];
#pragma unroll
      for (int i = 0; i < 8; ++i) t[2 * i] = v.a[i], t[2 * i + 1] = v.b[i];
      Pairs<T, kVec>::put(x + pl.first(0), t);
      Pairs<T, kVec>::put(x + pl.first(0) + 8, t + 8);
    } else {
      Pairs<T, kVec>::put(x + pl.first(0), v.a);
      Pairs<T, kVec>::put(x + pl.second(0), v.b);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < pl.live) {
        x[pl.first(i)] = (T)v.a[i];
        x[pl.second(i)] = (T)v.b[i];
      }
  }
}

// kWeight of a lane's pairs (1 beyond the head's end or without weights).
SC_DEV void load_weight(const float* w, const Place& pl, float (&a)[8], float (&b)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const bool on = w && i < pl.live;
    a[i] = on ? w[pl.first(i)] : 1.f;
    b[i] = on ? w[pl.second(i)] : 1.f;
  }
}

// The normalised head in place of x (elements beyond the head's end stay 0); returns
// 1 / deviation.
template <typename P>
SC_DEV float normalise(P& v, const RotaryArgs& a, const Place& pl) {
  const float scale = 1.f / (float)a.d;
  if (!a.rms) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s += v.a[i] + v.b[i];
    const float mean = head_sum(s, a.lanes) * scale;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < pl.live) {
        v.a[i] -= mean;
        v.b[i] -= mean;
      }
  }
  float q = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) q = fmaf(v.a[i], v.a[i], fmaf(v.b[i], v.b[i], q));
  const float inv = 1.f / sqrtf(fmaf(head_sum(q, a.lanes), scale, a.eps));
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    v.a[i] *= inv;
    v.b[i] *= inv;
  }
  return inv;
}

template <typename T, bool kVec, bool kBack>
__global__ __launch_bounds__(kThreads) void k_rotary(RotaryArgs a) {
  __shared__ float2 cs[kMaxTokens * 128];
  __shared__ float red[kBack ? 4 : 1][2][256];
  const int tid = threadIdx.x, lane = tid & 63, lanes = a.lanes;
  const int sub = tid & (lanes - 1), R2 = a.R / 2;
  const long long rows = (long long)a.B * a.n;
  const Place pl(a.d, a.R, a.interleaved, sub);
  float dwa[2][8], dwb[2][8];
  if constexpr (kBack) {
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int i = 0; i < 8; ++i) dwa[p][i] = dwb[p][i] = 0.f;
  }
  for (long long t0 = (long long)blockIdx.x * a.tokens; t0 < rows; t0 += (long long)gridDim.x * a.tokens) {
    const int nt = (int)min((long long)a.tokens, rows - t0);
    if (R2 > 0) {
      __syncthreads();  // the last tokens' angles are read
      for (int i = tid; i < nt * R2; i += kThreads) {
        const int t = i / R2, f = i - t * R2;
        const long long row = t0 + t;
        const long long p = a.pos ? a.pos[row] : (int)((unsigned)row % (unsigned)a.n);
        const unsigned turn = (unsigned)(((unsigned long long)p * a.turns.t[f]) >> 32);
        float c, s;
        cos_sin(turn, c, s);
        cs[t * R2 + f] = make_float2(c * a.amplitude, (kBack ? -s : s) * a.amplitude);
      }
      __syncthreads();
    }
    const int items = nt * a.heads, step = kThreads / lanes;
    const int rounds = (items + step - 1) / step;  // whole rounds: sums over lanes stay in one wave's lanes
    int item = tid / lanes;
    for (int r = 0; r < rounds; ++r, item += step) {
      const bool on = item < items;
      const int t = on ? item / a.heads : 0, head = on ? item - t * a.heads : a.h2;
      const long long row = t0 + t;
      const int part = head >= a.h2 ? 2 : head >= a.h1 ? 1 : 0;
      const long long at = (long long)(head - (part == 2 ? a.h2 : part == 1 ? a.h1 : 0)) * a.d;
      T* o = reinterpret_cast<T*>((part == 2 ? a.o[2] : part == 1 ? a.o[1] : a.o[0]) +
                                  row * (part == 2 ? a.os[2] : part == 1 ? a.os[1] : a.os[0])) + at;
      bool live = on;
      if (a.len && on) {
        const unsigned b = (unsigned)row / (unsigned)a.n;
        live = (int)((unsigned)row - b * a.n) < clampi(a.len[b], 0, a.n);
      }
      Pairs<T, kVec> v, g;
#pragma unroll
      for (int i = 0; i < 8; ++i) v.a[i] = v.b[i] = 0.f;
      if (live && (!kBack || (a.norm && part < 2))) {
        const T* x = reinterpret_cast<const T*>((part == 2 ? a.x[2] : part == 1 ? a.x[1] : a.x[0]) +
                                                row * (part == 2 ? a.xs[2] : part == 1 ? a.xs[1] : a.xs[0])) + at;
        load_pairs(v, x, pl);
      }
      float wa[8], wb[8];
      const bool turned = part < 2;
      if (a.norm && turned) load_weight(part == 1 ? a.w[1] : a.w[0], pl, wa, wb);
      if constexpr (!kBack) {
        if (a.norm && turned) {
          // in every lane of the head alike
          normalise(v, a, pl);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            v.a[i] *= wa[i];
            v.b[i] *= wb[i];
          }
        }
        if (turned && live) {
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (i < pl.rot) {
              const float2 z = cs[t * R2 + pl.p0 + i];
              const float p = v.a[i], q = v.b[i];
              v.a[i] = p * z.x - q * z.y;
              v.b[i] = p * z.y + q * z.x;
            }
        }
        if (on) store_pairs(v, o, pl);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) g.a[i] = g.b[i] = 0.f;
        if (live) {
          const T* p = reinterpret_cast<const T*>((part == 2 ? a.g[2] : part == 1 ? a.g[1] : a.g[0]) +
                                                  row * (part == 2 ? a.gs[2] : part == 1 ? a.gs[1] : a.gs[0])) + at;
          load_pairs(g, p, pl);
          if (turned) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
              if (i < pl.rot) {
                const float2 z = cs[t * R2 + pl.p0 + i];
                const float p = g.a[i], q = g.b[i];
                g.a[i] = p * z.x - q * z.y;
                g.b[i] = p * z.y + q * z.x;
              }
          }
        }
        if (a.norm && turned) {
          const float inv = normalise(v, a, pl);
          float gh = 0.f, gs = 0.f;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float ha = g.a[i] * v.a[i], hb = g.b[i] * v.b[i];
            dwa[0][i] += part == 0 ? ha : 0.f;
            dwb[0][i] += part == 0 ? hb : 0.f;
            dwa[1][i] += part == 1 ? ha : 0.f;
            dwb[1][i] += part == 1 ? hb : 0.f;
            g.a[i] *= wa[i];
            g.b[i] *= wb[i];
            gh = fmaf(g.a[i], v.a[i], fmaf(g.b[i], v.b[i], gh));
            gs += g.a[i] + g.b[i];
          }
          const float scale = 1.f / (float)a.d;
          gh = head_sum(gh, lanes) * scale;
          gs = a.rms ? 0.f : head_sum(gs, lanes) * scale;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            g.a[i] = live ? inv * (g.a[i] - fmaf(v.a[i], gh, gs)) : 0.f;
            g.b[i] = live ? inv * (g.b[i] - fmaf(v.b[i], gh, gs)) : 0.f;
          }
        }
        if (on) store_pairs(g, o, pl);
      }
    }
  }
  if constexpr (kBack) {
    if (!a.part) return;
    // over the lanes of a wave that hold the same pairs, then over the waves
    const int w = tid >> 6;
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float x = dwa[p][i], y = dwb[p][i];
        for (int m = lanes; m < 64; m *= 2) {
          x += __shfl_xor(x, m);
          y += __shfl_xor(y, m);
        }
        if (lane < lanes && i < pl.live) {
          red[w][p][pl.first(i)] = x;
          red[w][p][pl.second(i)] = y;
        }
      }
    __syncthreads();
    for (int c = tid; c < 2 * a.d; c += kThreads) {
      const int p = c >= a.d, e = p ? c - a.d : c;
      a.part[((long long)blockIdx.x * 2 + p) * a.d + e] =
          (red[0][p][e] + red[1][p][e]) + (red[2][p][e] + red[3][p][e]);
    }
  }
}

// The workgroups' sums of 16 columns (of 2 d), 16 lanes a column, then a tree.
__global__ __launch_bounds__(256) void k_rotary_weights(const float* __restrict__ part, float* __restrict__ dq_w,
                                                        float* __restrict__ dk_w, int wgs, int d) {
  __shared__ float red[16][17];
  const int col = threadIdx.x & 15, row = threadIdx.x >> 4, c = blockIdx.x * 16 + col;
  float s = 0.f;
  if (c < 2 * d)
    for (int i = row; i < wgs; i += 16) s += part[(long long)i * 2 * d + c];
  red[row][col] = s;
  __syncthreads();
  for (int h = 8; h > 0; h >>= 1) {
    if (row < h) red[row][col] += red[row + h][col];
    __syncthreads();
  }
  if (row == 0 && c < 2 * d) {
    float* o = c < d ? dq_w : dk_w;
    if (o) o[c < d ? c : c - d] = red[0][col];
  }
}

constexpr int kWeightWgs = 1024;  // workgroups that leave sums

int tokens_of(long long rows) { return (int)std::max<long long>(1, std::min<long long>(kMaxTokens, rows / 2048)); }

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

template <bool kBack>
hipError_t run(const Rotary& r, hipStream_t s) {
  RotaryArgs a;
  const long long e = r.f32 ? 4 : 2;
  const void* xs[3] = {r.q, r.k, r.v};
  const void* gs[3] = {r.gq, r.gk, r.gv};
  void* os[3] = {r.oq, r.ok, r.ov};
  const int heads[3] = {os[0] ? r.Hq : 0, os[1] ? r.Hk : 0, os[2] ? r.Hk : 0};
  const long long ld[3] = {r.q_stride, r.k_stride, r.v_stride};
  bool vec = true;
  for (int i = 0; i < 3; ++i) {
    const long long dense = (long long)(i == 0 ? r.Hq : r.Hk) * r.d;
    a.x[i] = static_cast<const char*>(xs[i]);
    a.g[i] = static_cast<const char*>(gs[i]);
    a.o[i] = static_cast<char*>(os[i]);
    a.xs[i] = ld[i] * e;
    a.gs[i] = dense * e;
    a.os[i] = (kBack ? ld[i] : dense) * e;
    if (!os[i]) continue;
    vec = vec && aligned16(xs[i]) && aligned16(gs[i]) && aligned16(os[i]) && ld[i] * e % 16 == 0 && dense * e % 16 == 0;
  }
  // sixteen elements of a lane as vectors: of the rotated part or of the rest, not both
  vec = vec && r.d % 16 == 0 && (r.interleaved || r.R % 16 == 0);
  a.w[0] = r.q_w;
  a.w[1] = r.k_w;
  a.len = r.len;
  a.pos = r.pos;
  a.part = kBack && (r.dq_w || r.dk_w) ? r.ws : nullptr;
  a.B = r.B;
  a.n = r.n;
  a.h1 = heads[0];
  a.h2 = heads[0] + heads[1];
  a.heads = a.h2 + heads[2];
  a.d = r.d;
  a.R = r.R;
  a.lanes = 1;
  while (a.lanes * 16 < r.d) a.lanes *= 2;
  const long long rows = (long long)r.B * r.n;
  a.tokens = tokens_of(rows);
  a.interleaved = r.interleaved;
  a.norm = r.norm;
  a.rms = r.rms;
  a.eps = r.eps;
  a.amplitude = r.amplitude;
  a.turns = r.turns;
  const long long tiles = (rows + a.tokens - 1) / a.tokens;
  const int wgs = (int)std::min<long long>(tiles, a.part ? kWeightWgs : 1 << 16);
  const dim3 grid(wgs), block(kThreads);
  if (r.f32) {
    if (vec)
      hipLaunchKernelGGL((k_rotary<float, true, kBack>), grid, block, 0, s, a);
    else
      hipLaunchKernelGGL((k_rotary<float, false, kBack>), grid, block, 0, s, a);
  } else if (vec) {
    hipLaunchKernelGGL((k_rotary<__bf16, true, kBack>), grid, block, 0, s, a);
  } else {
    hipLaunchKernelGGL((k_rotary<__bf16, false, kBack>), grid, block, 0, s, a);
  }
  if (a.part)
    hipLaunchKernelGGL(k_rotary_weights, dim3((2 * r.d + 15) / 16), dim3(256), 0, s, a.part, r.dq_w, r.dk_w, wgs, r.d);
  return hipGetLastError();
}

}  // namespace

size_t rotary_backward_floats(long long rows, int d) {
  const int t = tokens_of(rows);
  return (size_t)std::min<long long>((rows + t - 1) / t, kWeightWgs) * 2 * d;
}
hipError_t launch_rotary(const Rotary& r, hipStream_t s) { return run<false>(r, s); }
hipError_t launch_rotary_backward(const Rotary& r, hipStream_t s) { return run<true>(r, s); }

}  // namespace sc
