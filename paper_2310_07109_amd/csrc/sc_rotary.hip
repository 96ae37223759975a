// Rotary positions of queries and keys, with their norms per head.
//
//   u = norm(x) * w;  (a, b) -> A (a cos phi - b sin phi, a sin phi + b cos phi),
//   phi = p f_i; backward: the rotation by -phi, then the norm's gradient
//   dx = inv (g - hat mean(g hat) - mean(g)),  g = w du,  hat = (x - mean) inv
//   (mean only for LayerNorm), dw = sum du hat.
//
// One read and one write of every head bound it: 65536 rows of 12 + 12 + 12 heads of 64, bf16,
// a third of them valid, 80 us for 413 MB (5.2 TB/s, as a copy; 91 in the median of calls back
// to back); backward with RMS norms, 32768 rows of 16 + 4 + 4 heads, 62 us for 285 MB (4.6).
// A lane holds eight pairs of a head, both halves of each, so the rotation is within a lane
// and d / 16 lanes (rounded up to a power of two) hold a head; its sums go over them by DPP.
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
  int heads, wgs, move;
};
struct RotaryArgs {
  RotaryPart part[3];  // q, k, v
  const int* len;
  const int* pos;
  int B, n, d, R, lanes;  // lanes of a head
  int tokens, tiles, norm, rms, in_turn;
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

// kN (4 or 8) successive elements at a vector's address.
template <int kN, typename T>
SC_DEV void take(const T* p, float* v) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int h = 0; h < kN / 4; ++h) {
      const f32x4 x = reinterpret_cast<const f32x4*>(p)[h];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[4 * h + i] = x[i];
    }
  } else {
    typedef __attribute__((ext_vector_type(kN / 2))) unsigned Vec;
    const Vec u = *reinterpret_cast<const Vec*>(p);
#pragma unroll
    for (int i = 0; i < kN / 2; ++i) {
      v[2 * i] = __builtin_bit_cast(float, u[i] << 16);
      v[2 * i + 1] = __builtin_bit_cast(float, u[i] & 0xffff0000u);
    }
  }
}
template <int kN, typename T>
SC_DEV void put(T* p, const float* v) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int h = 0; h < kN / 4; ++h)
      reinterpret_cast<f32x4*>(p)[h] = f32x4{v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]};
  } else {
    typedef __attribute__((ext_vector_type(kN / 2))) unsigned Vec;
    Vec u;
#pragma unroll
    for (int i = 0; i < kN / 2; ++i) u[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
    *reinterpret_cast<Vec*>(p) = u;
  }
}

// Eight pairs of a head, pair i at elements e0 + i, e1 + i (half) or e0 + 2 i,
// e0 + 2 i + 1 (interleaved).
struct Pairs {
  float a[8], b[8];
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

// kVec: pairs of a vector, 8 or 4, which are all rotated, all passed or all beyond the head's
// end; 0: an element an access.
template <int kVec, typename T, bool kInter>
SC_DEV void load_pairs(Pairs& v, const T* x, const Place<kInter>& pl) {
  if constexpr (kVec) {
#pragma unroll
    for (int h = 0; h < 8; h += kVec) {
      const bool live = h < pl.live;  // beyond the head's end its start is read, and nothing of it kept
      if constexpr (kInter) {
        float e[2 * kVec];
        const T* p = x + (live ? pl.first(h) : 0);
        take<kVec>(p, e);
        take<kVec>(p + kVec, e + kVec);
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
          v.a[h + i] = live ? e[2 * i] : 0.f;
          v.b[h + i] = live ? e[2 * i + 1] : 0.f;
        }
      } else {
        take<kVec>(x + (live ? pl.first(h) : 0), v.a + h);
        take<kVec>(x + (live ? pl.second(h) : 0), v.b + h);
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
          v.a[h + i] = live ? v.a[h + i] : 0.f;
          v.b[h + i] = live ? v.b[h + i] : 0.f;
        }
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v.a[i] = i < pl.live ? (float)x[pl.first(i)] : 0.f;
      v.b[i] = i < pl.live ? (float)x[pl.second(i)] : 0.f;
    }
  }
}

template <int kVec, typename T, bool kInter>
SC_DEV void store_pairs(const Pairs& v, T* x, const Place<kInter>& pl) {
  if constexpr (kVec) {
#pragma unroll
    for (int h = 0; h < 8; h += kVec) {
      if (h >= pl.live) return;
      if constexpr (kInter) {
        float e[2 * kVec];
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
          e[2 * i] = v.a[h + i];
          e[2 * i + 1] = v.b[h + i];
        }
        put<kVec>(x + pl.first(h), e);
        put<kVec>(x + pl.first(h) + kVec, e + kVec);
      } else {
        put<kVec>(x + pl.first(h), v.a + h);
        put<kVec>(x + pl.second(h), v.b + h);
      }
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
template <bool kInter>
SC_DEV float normalise(Pairs& v, const RotaryArgs& a, const Place<kInter>& pl) {
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
template <bool kInter>
SC_DEV void rotate(Pairs& v, const float* cs, const float* sn, const Place<kInter>& pl) {
  if (pl.rot <= 0) return;
#pragma unroll
  for (int h = 0; h < 8; h += 4) {
    const f32x4 c = *reinterpret_cast<const f32x4*>(cs + pl.p0 + h), s = *reinterpret_cast<const f32x4*>(sn + pl.p0 + h);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int i = h + e;
      const float p = v.a[i], q = v.b[i];
      v.a[i] = i < pl.rot ? p * c[e] - q * s[e] : p;
      v.b[i] = i < pl.rot ? p * s[e] + q * c[e] : q;
    }
  }
}

template <typename T, int kVec, bool kInter, bool kBack>
__global__ __launch_bounds__(kThreads) void k_rotary(RotaryArgs a) {
  __shared__ __attribute__((aligned(16))) float cs[kMaxTokens][kRotaryMaxD / 2], sn[kMaxTokens][kRotaryMaxD / 2];
  __shared__ int live_of[kMaxTokens];
  __shared__ float red[kBack ? 4 : 1][256];
  const int tid = threadIdx.x, lane = tid & 63, lanes = a.lanes;
  const int q0 = a.part[0].wgs, k0 = q0 + a.part[1].wgs, bid = blockIdx.x;
  const int which = a.in_turn ? bid % 3 : bid < q0 ? 0 : bid < k0 ? 1 : 2;
  const RotaryPart pt = which == 0 ? a.part[0] : which == 1 ? a.part[1] : a.part[2];
  const int wg = a.in_turn ? bid / 3 : bid - (which == 0 ? 0 : which == 1 ? q0 : k0);
  const bool turned = which < 2, norm = a.norm && turned;
  const int sub = tid & (lanes - 1), R2 = turned ? a.R / 2 : 0, heads = pt.heads;
  const long long rows = (long long)a.B * a.n;
  const Place<kInter> pl(a.d, a.R, sub);
  float wa[8], wb[8], dwa[8], dwb[8];
  if (norm) load_weight(pt.w, pl, wa, wb);
  if constexpr (kBack) {
#pragma unroll
    for (int i = 0; i < 8; ++i) dwa[i] = dwb[i] = 0.f;
  }
  // A workgroup's place in a whole round of tiles moves on from one to the next, so that it
  // comes to another part of a sequence, and not to the padding of every one or of none.
  int place = wg;
  for (int tile = wg; tile < a.tiles; tile += pt.wgs) {
    const int round = tile - wg;
    const long long t0 = (long long)(round + (round + pt.wgs <= a.tiles ? place : wg)) * a.tokens;
    place += pt.move;
    if (place >= pt.wgs) place -= pt.wgs;
    const int nt = (int)min((long long)a.tokens, rows - t0);
    __syncthreads();  // the last tokens' angles are read
    if (tid < nt) {
      const unsigned row = (unsigned)(t0 + tid), b = row / (unsigned)a.n;
      live_of[tid] = !a.len || (int)(row - b * a.n) < clampi(a.len[b], 0, a.n);
    }
    __syncthreads();
    for (int i = tid; i < nt * R2; i += kThreads) {
      const int t = i / R2, f = i - t * R2;
      if (!live_of[t]) continue;
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
      Pairs v, g;
#pragma unroll
      for (int i = 0; i < 8; ++i) v.a[i] = v.b[i] = 0.f;
      if (live && (!kBack || norm)) load_pairs<kVec>(v, reinterpret_cast<const T*>(pt.x + row * pt.xs + at), pl);
      T* o = reinterpret_cast<T*>(pt.o + row * pt.os + at);
      if constexpr (!kBack) {
        if (live && turned) {  // a head's lanes are live together
          if (norm) {
            normalise(v, a, pl);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              v.a[i] *= wa[i];
              v.b[i] *= wb[i];
            }
          }
          rotate(v, cs[tok], sn[tok], pl);
        }
        if (on) store_pairs<kVec>(v, o, pl);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) g.a[i] = g.b[i] = 0.f;
        if (live) {
          load_pairs<kVec>(g, reinterpret_cast<const T*>(pt.g + row * pt.gs + at), pl);
          if (turned) rotate(g, cs[tok], sn[tok], pl);
        }
        if (norm && live) {
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
            g.a[i] = inv * (g.a[i] - fmaf(v.a[i], gh, gs));
            g.b[i] = inv * (g.b[i] - fmaf(v.b[i], gh, gs));
          }
        }
        if (on) store_pairs<kVec>(g, o, pl);
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

template <typename T, int kVec, bool kBack>
void start(const RotaryArgs& a, int grid, int interleaved, hipStream_t s) {
  if (interleaved)
    hipLaunchKernelGGL((k_rotary<T, kVec, true, kBack>), dim3(grid), dim3(kThreads), 0, s, a);
  else
    hipLaunchKernelGGL((k_rotary<T, kVec, false, kBack>), dim3(grid), dim3(kThreads), 0, s, a);
}

template <typename T, bool kBack>
void start(const RotaryArgs& a, int width, int grid, int interleaved, hipStream_t s) {
  if (width == 8)
    start<T, 8, kBack>(a, grid, interleaved, s);
  else if (width == 4)
    start<T, 4, kBack>(a, grid, interleaved, s);
  else
    start<T, 0, kBack>(a, grid, interleaved, s);
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
  const long long tiles = (rows + a.tokens - 1) / a.tokens;  // below 2^28: 16 tokens each where there are many
  a.tiles = (int)tiles;
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
    // 5 / 13 of a sequence further from round to round (64 x 1024 rows, a third of them valid,
    // 16 + 4 + 4 heads of 64, backward with RMS norms: 107 us, with rounds of whole sequences 134)
    const int per = std::max(1, r.n / a.tokens);
    p.move = p.wgs ? ((5 * per / 13 - p.wgs) % per + per) % per % p.wgs : 0;
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
  // The pairs of a vector are all of the rotated part, or all of the rest (heads of 80 with 40
  // rotated, halves, bf16, 16384 rows of 48: 68 us by 4 pairs, 178 by elements).
  auto fits = [&](int pairs) { return r.d % (2 * pairs) == 0 && (r.interleaved || r.R % (2 * pairs) == 0); };
  const int width = !vec ? 0 : fits(8) ? 8 : fits(4) ? 4 : 0;
  // Workgroups of the same tokens follow one another where the parts are alike (a call of
  // 65536 rows, a third of them valid, 12 + 12 + 12 heads of 64: 97 us, part after part 115);
  // otherwise the longest part goes first (32768 rows of 16 + 4 + 4 heads of 128: 97, in turn 103).
  a.in_turn = a.part[0].wgs == a.part[1].wgs && a.part[0].wgs == a.part[2].wgs && r.Hq == r.Hk;
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
  if (r.f32)
    start<float, kBack>(a, width, grid, r.interleaved, s);
  else
    start<__bf16, kBack>(a, width, grid, r.interleaved, s);
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
