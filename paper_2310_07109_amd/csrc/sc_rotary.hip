// Rotary positions of queries and keys, with their norms per head.
//
//   u = norm(x) * w;  (a, b) -> A (a cos phi - b sin phi, a sin phi + b cos phi),
//   phi = p f_i; backward: the rotation by -phi, then the norm's gradient
//   dx = inv (g - hat mean(g hat) - mean(g)),  g = w du,  hat = (x - mean) inv
//   (mean only for LayerNorm), dw = sum du hat.
//
// One read and one write of every head bound it: 65536 rows of 12 + 12 + 12 heads of 64,
// bf16, a third of them valid, 97 us for 413 MB (4.2 TB/s, where a copy reaches 5.1); backward
// with RMS norms, 32768 rows of 16 + 4 + 4 heads of 64, bf16, 63 us for 285 MB (4.5).  A lane
// holds eight pairs of a head, both halves of each, so the rotation is within a lane and
// d / 16 lanes (rounded up to a power of two) hold a head; its sums go over them by DPP.
//
// The angles of a token serve all its heads: a workgroup makes the cosines and sines
// of its tokens once, in LDS.  An angle is a turn in 64-bit fixed point: position times
// frequency modulo 2^64 is exact in integers whatever the position, and what is left is
// at most an eighth of a turn for a polynomial.  Queries, keys and values have workgroups
// of their own, so that a lane's weights, and the sums of their gradients, stay in
// registers over all the heads that it sees.
#include <algorithm>

#include "sc_device.h"
#include "sc_internal.h"

namespace sc {
namespace {

typedef __attribute__((ext_vector_type(4))) unsigned u32x4;

constexpr int kThreads = 256;
constexpr int kMaxTokens = 16;  // of a workgroup at a time

struct RotaryPart {
  const char *x, *g;      // input and, backward, the gradient of the output
  char* o;                // output
  long long xs, gs, os;   // bytes between tokens
  const float* w;         // or null
  float* part;            // backward: [workgroups, d] sums of the weight's gradient, or null
  int heads, wgs;
};
struct RotaryArgs {
  RotaryPart part[3];  // q, k, v
  const int* len;
  const int* pos;
  int B, n, d, R, lanes;  // lanes of a head
  int tokens, norm, rms;
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
  SC_DEV static void vec(const T* p, float (&v)[8]) {  // eight elements at 16 bytes
    if constexpr (sizeof(T) == 4) {
      const f32x4 lo = *reinterpret_cast<const f32x4*>(p), hi = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = i < 4 ? lo[i & 3] : hi[i & 3];
    } else {
      const u32x4 u = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[2 * i] = __builtin_bit_cast(float, u[i] << 16);
        v[2 * i + 1] = __builtin_bit_cast(float, u[i] & 0xffff0000u);
      }
    }
  }
  SC_DEV static void put(T* p, const float (&v)[8]) {
    if constexpr (sizeof(T) == 4) {
      *reinterpret_cast<f32x4*>(p) = f32x4{v[0], v[1], v[2], v[3]};
      *reinterpret_cast<f32x4*>(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
    } else {
      *reinterpret_cast<u32x4*>(p) =
          u32x4{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
    }
  }
  SC_DEV void take(const T* p) {  // eight interleaved pairs
    if constexpr (sizeof(T) == 4) {
      f32x4 x[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = reinterpret_cast<const f32x4*>(p)[j];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        a[i] = x[i / 2][2 * (i & 1)];
        b[i] = x[i / 2][2 * (i & 1) + 1];
      }
    } else {
      u32x4 x[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) x[j] = reinterpret_cast<const u32x4*>(p)[j];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const unsigned u = x[i / 4][i & 3];
        a[i] = __builtin_bit_cast(float, u << 16);
        b[i] = __builtin_bit_cast(float, u & 0xffff0000u);
      }
    }
  }
  SC_DEV void give(T* p) const {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        reinterpret_cast<f32x4*>(p)[j] = f32x4{a[2 * j], b[2 * j], a[2 * j + 1], b[2 * j + 1]};
    } else {
#pragma unroll
      for (int j = 0; j < 2; ++j)
        reinterpret_cast<u32x4*>(p)[j] = u32x4{pack_bf16(a[4 * j], b[4 * j]), pack_bf16(a[4 * j + 1], b[4 * j + 1]),
                                               pack_bf16(a[4 * j + 2], b[4 * j + 2]), pack_bf16(a[4 * j + 3], b[4 * j + 3])};
    }
  }
};

// Where a lane's pairs are: pair i (of the lane) is live below `live`, rotated below
// `rot`; elements first(i) and second(i).
template <bool kInter>
struct Place {
  int p0, live, rot, R2, d2;
  SC_DEV Place(int d, int R, int sub)
      : p0(8 * sub), live(d / 2 - 8 * sub), rot(R / 2 - 8 * sub), R2(R / 2), d2(d / 2) {}
  SC_DEV int first(int i) const {
    const int p = p0 + i;
    return kInter ? 2 * p : i < rot ? p : p + R2;  // passed pair q = p - R2: element R + q
  }
  SC_DEV int second(int i) const {
    const int p = p0 + i;
    return kInter ? 2 * p + 1 : i < rot ? p + R2 : p + d2;  // R + (d - R) / 2 + q
  }
};

template <typename T, bool kVec, bool kInter>
SC_DEV void load_pairs(Pairs<T, kVec>& v, const T* x, const Place<kInter>& pl) {
  if constexpr (kVec) {
    // lanes beyond the head's end read its start, and keep nothing of it
    const bool live = pl.live > 0;
    if constexpr (kInter) {
      v.take(x + (live ? pl.first(0) : 0));
    } else {
      Pairs<T, kVec>::vec(x + (live ? pl.first(0) : 0), v.a);
      Pairs<T, kVec>::vec(x + (live ? pl.second(0) : 0), v.b);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v.a[i] = live ? v.a[i] : 0.f;
      v.b[i] = live ? v.b[i] : 0.f;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v.a[i] = i < pl.live ? (float)x[pl.first(i)] : 0.f;
      v.b[i] = i < pl.live ? (float)x[pl.second(i)] : 0.f;
    }
  }
}

template <typename T, bool kVec, bool kInter>
SC_DEV void store_pairs(const Pairs<T, kVec>& v, T* x, const Place<kInter>& pl) {
  if constexpr (kVec) {
    if (pl.live <= 0) return;
    if constexpr (kInter) {
      v.give(x + pl.first(0));
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

// Weights of a lane's pairs (1 beyond the head's end or without weights).
template <bool kInter>
SC_DEV void load_weight(const float* w, const Place<kInter>& pl, float (&a)[8], float (&b)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const bool on = w && i < pl.live;
    a[i] = on ? w[pl.first(i)] : 1.f;
    b[i] = on ? w[pl.second(i)] : 1.f;
  }
}

// The normalised head in place of x (elements beyond the head's end stay 0); returns
// 1 / deviation.
template <typename P, bool kInter>
SC_DEV float normalise(P& v, const RotaryArgs& a, const Place<kInter>& pl) {
  const float scale = 1.f / (float)a.d;
  if (!a.rms) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s += v.a[i] + v.b[i];
    const float mean = head_sum(s, a.lanes) * scale;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v.a[i] -= i < pl.live ? mean : 0.f;
      v.b[i] -= i < pl.live ? mean : 0.f;
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

// The rotation of a lane's pairs by the cosines and sines of a token, kept apart in LDS.
template <typename P, bool kInter>
SC_DEV void rotate(P& v, const float* cs, const float* sn, const Place<kInter>& pl, bool whole) {
  if (whole) {  // all eight pairs or none
    if (pl.rot <= 0) return;
    float c[8], s[8];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const f32x4 x = *reinterpret_cast<const f32x4*>(cs + pl.p0 + 4 * h);
      const f32x4 y = *reinterpret_cast<const f32x4*>(sn + pl.p0 + 4 * h);
#pragma unroll
      for (int e = 0; e < 4; ++e) c[4 * h + e] = x[e], s[4 * h + e] = y[e];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float p = v.a[i], q = v.b[i];
      v.a[i] = p * c[i] - q * s[i];
      v.b[i] = p * s[i] + q * c[i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float c = cs[pl.p0 + i], s = sn[pl.p0 + i], p = v.a[i], q = v.b[i];
      v.a[i] = i < pl.rot ? p * c - q * s : p;
      v.b[i] = i < pl.rot ? p * s + q * c : q;
    }
  }
}

template <typename T, bool kVec, bool kInter, bool kBack>
__global__ __launch_bounds__(kThreads) void k_rotary(RotaryArgs a) {
  __shared__ __attribute__((aligned(16))) float cs[kMaxTokens][kRotaryMaxD / 2], sn[kMaxTokens][kRotaryMaxD / 2];
  __shared__ int live_of[kMaxTokens];
  __shared__ float red[kBack ? 4 : 1][256];
  const int tid = threadIdx.x, lane = tid & 63, lanes = a.lanes;
  const int q0 = a.part[0].wgs, k0 = q0 + a.part[1].wgs;
  const int which = (int)blockIdx.x < q0 ? 0 : (int)blockIdx.x < k0 ? 1 : 2;
  const RotaryPart pt = which == 0 ? a.part[0] : which == 1 ? a.part[1] : a.part[2];
  const int wg = (int)blockIdx.x - (which == 0 ? 0 : which == 1 ? q0 : k0);
  const bool turned = which < 2, norm = a.norm && turned;
  const int sub = tid & (lanes - 1), R2 = turned ? a.R / 2 : 0, heads = pt.heads;
  const bool whole = kVec && a.R % 16 == 0;
  const long long rows = (long long)a.B * a.n;
  const Place<kInter> pl(a.d, a.R, sub);
  float wa[8], wb[8], dwa[8], dwb[8];
  if (norm) load_weight(pt.w, pl, wa, wb);
  if constexpr (kBack) {
#pragma unroll
    for (int i = 0; i < 8; ++i) dwa[i] = dwb[i] = 0.f;
  }
  for (long long t0 = (long long)wg * a.tokens; t0 < rows; t0 += (long long)pt.wgs * a.tokens) {
    const int nt = (int)min((long long)a.tokens, rows - t0);
    __syncthreads();  // the last tokens' angles are read
    if (tid < nt) {
      const unsigned row = (unsigned)(t0 + tid), b = row / (unsigned)a.n;
      live_of[tid] = !a.len || (int)(row - b * a.n) < clampi(a.len[b], 0, a.n);
    }
    for (int i = tid; i < nt * R2; i += kThreads) {
      const int t = i / R2, f = i - t * R2;
      const long long row = t0 + t;
      const long long p = a.pos ? a.pos[row] : (int)((unsigned)row % (unsigned)a.n);
      const unsigned turn = (unsigned)(((unsigned long long)p * a.turns.t[f]) >> 32);
      float c, s;
      cos_sin(turn, c, s);
      cs[t][f] = c * a.amplitude;
      sn[t][f] = (kBack ? -s : s) * a.amplitude;
    }
    __syncthreads();
    const int items = nt * heads, step = kThreads / lanes;
    const int rounds = (items + step - 1) / step;  // whole rounds: sums over lanes stay in one wave's lanes
    int item = tid / lanes, t = item / heads, head = item - t * heads;
    const int dt = step / heads, dh = step - dt * heads;
    for (int r = 0; r < rounds; ++r) {
      const bool on = item < items;
      const int tok = on ? t : 0;
      const long long row = t0 + tok, at = (long long)head * a.d * (int)sizeof(T);
      const bool live = on && live_of[tok];
      Pairs<T, kVec> v, g;
#pragma unroll
      for (int i = 0; i < 8; ++i) v.a[i] = v.b[i] = 0.f;
      if (live && (!kBack || norm)) load_pairs(v, reinterpret_cast<const T*>(pt.x + row * pt.xs + at), pl);
      T* o = reinterpret_cast<T*>(pt.o + row * pt.os + at);
      if constexpr (!kBack) {
        if (norm) {
          normalise(v, a, pl);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            v.a[i] *= wa[i];
            v.b[i] *= wb[i];
          }
        }
        if (turned && live) rotate(v, cs[tok], sn[tok], pl, whole);
        if (on) store_pairs(v, o, pl);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) g.a[i] = g.b[i] = 0.f;
        if (live) {
          load_pairs(g, reinterpret_cast<const T*>(pt.g + row * pt.gs + at), pl);
          if (turned) rotate(g, cs[tok], sn[tok], pl, whole);
        }
        if (norm) {
          const float inv = normalise(v, a, pl);
          float gh = 0.f, gs = 0.f;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            dwa[i] = fmaf(g.a[i], v.a[i], dwa[i]);
            dwb[i] = fmaf(g.b[i], v.b[i], dwb[i]);
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
      item += step;
      t += dt;
      head += dh;
      if (head >= heads) {
        head -= heads;
        ++t;
      }
    }
  }
  if constexpr (kBack) {
    if (!pt.part) return;
    // over the lanes of a wave that hold the same pairs, then over the waves
    const int w = tid >> 6;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float x = dwa[i], y = dwb[i];
      for (int m = lanes; m < 64; m *= 2) {
        x += __shfl_xor(x, m);
        y += __shfl_xor(y, m);
      }
      if (lane < lanes && i < pl.live) {
        red[w][pl.first(i)] = x;
        red[w][pl.second(i)] = y;
      }
    }
    __syncthreads();
    for (int e = tid; e < a.d; e += kThreads)
      pt.part[(long long)wg * a.d + e] = (red[0][e] + red[1][e]) + (red[2][e] + red[3][e]);
  }
}

// The workgroups' sums of 16 columns, 16 lanes a column, then a tree: a chain of loads
// bounds it, 4 us for 512 records of 64 channels of q and of k.
struct WeightSums {
  const float* part[2];
  float* out[2];
  int wgs[2];
};
__global__ __launch_bounds__(256) void k_rotary_weights(WeightSums a, int d) {
  __shared__ float red[16][17];
  const int m = blockIdx.y, col = threadIdx.x & 15, row = threadIdx.x >> 4, c = blockIdx.x * 16 + col;
  if (!a.out[m]) return;
  const float* p = a.part[m];
  float s = 0.f;
  if (c < d) {
#pragma unroll 8
    for (int i = row; i < a.wgs[m]; i += 16) s += p[(long long)i * d + c];
  }
  red[row][col] = s;
  __syncthreads();
  for (int h = 8; h > 0; h >>= 1) {
    if (row < h) red[row][col] += red[row + h][col];
    __syncthreads();
  }
  if (row == 0 && c < d) a.out[m][c] = red[0][col];
}

constexpr int kWeightWgs = 512;  // workgroups of a part that leave sums

int lanes_of(int d) {
  int lanes = 1;
  while (lanes * 16 < d) lanes *= 2;
  return lanes;
}
// Tokens of a workgroup at a time: enough for a head to every group of lanes, more where
// there are many, since their angles are made together.
int tokens_of(long long rows, int d, int heads) {
  const long long fill = kThreads / lanes_of(d) / std::max(1, heads);
  return (int)std::max<long long>(1, std::min<long long>(kMaxTokens, std::max(fill, rows / 1024)));
}

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

template <typename T, bool kVec, bool kBack>
void start(const RotaryArgs& a, int grid, int interleaved, hipStream_t s) {
  if (interleaved)
    hipLaunchKernelGGL((k_rotary<T, kVec, true, kBack>), dim3(grid), dim3(kThreads), 0, s, a);
  else
    hipLaunchKernelGGL((k_rotary<T, kVec, false, kBack>), dim3(grid), dim3(kThreads), 0, s, a);
}

template <bool kBack>
hipError_t run(const Rotary& r, hipStream_t s) {
  RotaryArgs a;
  const long long e = r.f32 ? 4 : 2, rows = (long long)r.B * r.n;
  const void* xs[3] = {r.q, r.k, r.v};
  const void* gs[3] = {r.gq, r.gk, r.gv};
  void* os[3] = {r.oq, r.ok, r.ov};
  const long long ld[3] = {r.q_stride, r.k_stride, r.v_stride};
  const float* ws[3] = {r.q_w, r.k_w, nullptr};
  float* dw[3] = {r.dq_w, r.dk_w, nullptr};
  a.tokens = tokens_of(rows, r.d, std::max(r.Hq, r.Hk));
  const long long tiles = (rows + a.tokens - 1) / a.tokens;
  bool vec = true;
  float* part = r.ws;
  WeightSums sums = {};
  int grid = 0;
  for (int i = 0; i < 3; ++i) {
    RotaryPart& p = a.part[i];
    p.heads = os[i] ? (i == 0 ? r.Hq : r.Hk) : 0;
    const long long dense = (long long)p.heads * r.d;
    p.x = static_cast<const char*>(xs[i]);
    p.g = static_cast<const char*>(gs[i]);
    p.o = static_cast<char*>(os[i]);
    p.xs = ld[i] * e;
    p.gs = dense * e;
    p.os = (kBack ? ld[i] : dense) * e;
    p.w = ws[i];
    p.part = nullptr;
    p.wgs = os[i] ? (int)std::min<long long>(tiles, kBack && dw[i] ? kWeightWgs : 1 << 16) : 0;
    grid += p.wgs;
    if (kBack && dw[i]) {
      p.part = part;
      sums.part[i] = part;
      sums.out[i] = dw[i];
      sums.wgs[i] = p.wgs;
      part += (long long)p.wgs * r.d;
    }
    if (os[i])
      vec = vec && aligned16(xs[i]) && aligned16(gs[i]) && aligned16(os[i]) && ld[i] * e % 16 == 0 && dense * e % 16 == 0;
  }
  // sixteen elements of a lane as vectors: of the rotated part or of the rest, not both
  vec = vec && r.d % 16 == 0 && (r.interleaved || r.R % 16 == 0);
  a.len = r.len;
  a.pos = r.pos;
  a.B = r.B;
  a.n = r.n;
  a.d = r.d;
  a.R = r.R;
  a.lanes = lanes_of(r.d);
  a.norm = r.norm;
  a.rms = r.rms;
  a.eps = r.eps;
  a.amplitude = r.amplitude;
  a.turns = r.turns;
  if (r.f32) {
    if (vec)
      start<float, true, kBack>(a, grid, r.interleaved, s);
    else
      start<float, false, kBack>(a, grid, r.interleaved, s);
  } else if (vec) {
    start<__bf16, true, kBack>(a, grid, r.interleaved, s);
  } else {
    start<__bf16, false, kBack>(a, grid, r.interleaved, s);
  }
  if (sums.out[0] || sums.out[1])
    hipLaunchKernelGGL(k_rotary_weights, dim3((r.d + 15) / 16, 2), dim3(256), 0, s, sums, r.d);
  return hipGetLastError();
}

}  // namespace

size_t rotary_backward_floats(long long rows, int d, int heads) {
  const int t = tokens_of(rows, d, heads);
  return (size_t)std::min<long long>((rows + t - 1) / t, kWeightWgs) * 2 * d;
}
hipError_t launch_rotary(const Rotary& r, hipStream_t s) { return run<false>(r, s); }
hipError_t launch_rotary_backward(const Rotary& r, hipStream_t s) { return run<true>(r, s); }

}  // namespace sc
