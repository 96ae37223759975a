// Norms before and after a block, fused with the block's gate and the residual's
// scale, and their gradients.  Per row of D channels
//
//   u = post ? norm(t) post_w + post_b : t
//   r = scale x + gate u
//   y = norm(r) pre_w + pre_b
//
// A row stays in the registers of the threads that own it (a wavefront, or a
// workgroup for long rows) from its loads to its stores: every tensor is read
// or written once, and the statistics are two-pass float32 sums over registers.
// The backward pass reads the forward's inputs again and recomputes both norms
// instead of loading statistics.
#include <algorithm>
#include <type_traits>

#include "sc_device.h"
#include "sc_internal.h"
#include "sc_quant.h"

namespace sc {
namespace {

constexpr int kGateChannel = 1, kGateSequence = 2, kGateToken = 3;

// Threads of a workgroup that gives kTpr threads to a row.
template <int kTpr>
constexpr int kThreads = kTpr < 256 ? 256 : kTpr;

// Sum or maximum over the threads of a row: a wavefront, or those of a workgroup
// through LDS (two sets of slots in turn: a set is written again only after the
// barrier of the other).
template <int kTpr>
struct RowReduce {
  static constexpr int kWaves = kTpr / 64;
  float* slots;  // LDS, 2 x kWaves
  int flip = 0;
  SC_DEV const float* share(float v) {
    float* s = slots + kWaves * flip;
    flip ^= 1;
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
    __syncthreads();
    return s;
  }
  SC_DEV float sum(float v) {
    v = butterfly_sum(v);
    if constexpr (kWaves > 1) {
      const float* s = share(v);
      v = s[0];
#pragma unroll
      for (int i = 1; i < kWaves; ++i) v += s[i];
    }
    return v;
  }
  SC_DEV float max(float v) {
    v = butterfly_max(v);
    if constexpr (kWaves > 1) {
      const float* s = share(v);
      v = s[0];
#pragma unroll
      for (int i = 1; i < kWaves; ++i) v = vmax(v, s[i]);
    }
    return v;
  }
};

// kVec consecutive elements as one access.
template <int kVec>
SC_DEV void load_vec(const float* p, float* v) {
  if constexpr (kVec == 4) {
    const f32x4 x = *reinterpret_cast<const f32x4*>(p);
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] = x[q];
  } else {
    v[0] = *p;
  }
}
template <int kVec>
SC_DEV void load_vec(const __bf16* p, float* v) {
  if constexpr (kVec == 4) {
    const bf16x4 x = *reinterpret_cast<const bf16x4*>(p);
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] = (float)x[q];
  } else {
    v[0] = (float)*p;
  }
}
template <int kVec>
SC_DEV void store_vec(float* p, const float* v) {
  if constexpr (kVec == 4)
    *reinterpret_cast<f32x4*>(p) = f32x4{v[0], v[1], v[2], v[3]};
  else
    *p = v[0];
}
template <int kVec>
SC_DEV void store_vec(__bf16* p, const float* v) {
  if constexpr (kVec == 4)
    *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
  else
    *p = (__bf16)v[0];
}

// The channels of a thread: kPer groups of kVec, group u at (u kTpr + thread) kVec.
template <int kVec, int kPer, int kTpr>
struct Cols {
  int D, t;  // t: thread of the row
  SC_DEV int at(int u) const { return (u * kTpr + t) * kVec; }
  SC_DEV bool in(int u) const { return at(u) < D; }
  template <typename T>
  SC_DEV void load(const T* row, float* v) const {
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
      if (in(u)) {
        load_vec<kVec>(row + at(u), v + u * kVec);
      } else {
#pragma unroll
        for (int q = 0; q < kVec; ++q) v[u * kVec + q] = 0.f;
      }
    }
  }
  template <typename T>
  SC_DEV void store(T* row, const float* v) const {
#pragma unroll
    for (int u = 0; u < kPer; ++u)
      if (in(u)) store_vec<kVec>(row + at(u), v + u * kVec);
  }
  template <typename T>
  SC_DEV void zero(T* row) const {
    const float z[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < kPer; ++u)
      if (in(u)) store_vec<kVec>(row + at(u), z);
  }
};

// v -> (v - mean) / sqrt(var + eps), or v / sqrt(mean(v^2) + eps); channels beyond
// D stay 0.  Returns the factor.
template <int kVec, int kPer, int kTpr>
SC_DEV float normalise(float* v, const Cols<kVec, kPer, kTpr>& c, RowReduce<kTpr>& red, bool rms, float eps,
                       float fd) {
  constexpr int E = kVec * kPer;
  if (!rms) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < E; ++i) s += v[i];
    const float mean = red.sum(s) / fd;  // divided: a constant row has no deviation
#pragma unroll
    for (int u = 0; u < kPer; ++u)
      if (c.in(u)) {
#pragma unroll
        for (int q = 0; q < kVec; ++q) v[u * kVec + q] -= mean;
      }
  }
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < E; ++i) s = fmaf(v[i], v[i], s);
  const float inv = 1.f / sqrtf(red.sum(s) / fd + eps);
#pragma unroll
  for (int i = 0; i < E; ++i) v[i] *= inv;
  return inv;
}

// v = v w + b (w, b: or null)
template <int kVec, int kPer, int kTpr>
SC_DEV void affine(float* v, const float* w, const float* b, const Cols<kVec, kPer, kTpr>& c) {
  constexpr int E = kVec * kPer;
  float p[E];
  if (w) {
    c.load(w, p);
#pragma unroll
    for (int i = 0; i < E; ++i) v[i] *= p[i];
  }
  if (b) {
    c.load(b, p);
#pragma unroll
    for (int i = 0; i < E; ++i) v[i] += p[i];
  }
}

template <typename T, int kVec, int kPer, int kTpr>
SC_DEV void load_gate(float* g, const Norm& a, long long row, int b, const Cols<kVec, kPer, kTpr>& c) {
  if (a.gate_mode == kGateChannel)
    c.load(static_cast<const float*>(a.gate), g);
  else
    c.load(static_cast<const T*>(a.gate) + (a.gate_mode == kGateSequence ? b : row) * (long long)a.D, g);
}

// Rows dealt round-robin over the launch's row slots.
template <typename T, int kVec, int kPer, int kTpr>
__global__ __launch_bounds__(kThreads<kTpr>) void k_norm(Norm a) {
  constexpr int E = kVec * kPer, kRows = kThreads<kTpr> / kTpr;
  __shared__ float slots[2 * kTpr / 64];
  RowReduce<kTpr> red{slots};
  const Cols<kVec, kPer, kTpr> c{a.D, (int)threadIdx.x % kTpr};
  const float fd = (float)a.D;
  const int Dp = (a.D + kI8Pitch - 1) / kI8Pitch * kI8Pitch;
  const long long rows = (long long)a.B * a.n;
  const int slot = kTpr == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0;
  for (long long row = (long long)blockIdx.x * kRows + slot; row < rows; row += (long long)gridDim.x * kRows) {
    const int b = (int)(row / a.n), j = (int)(row - (long long)b * a.n);
    T* r = static_cast<T*>(a.r) + row * a.D;
    T* y = static_cast<T*>(a.y) + row * a.D;
    int8_t* yq = a.yq + row * Dp;
    if (a.len && j >= clampi(a.len[b], 0, a.n)) {
      if (a.skip_pad) continue;
      if (a.r) c.zero(r);
      if (a.y) c.zero(y);
      if (a.yq) {
        for (int k = 4 * c.t; k < Dp; k += 4 * kTpr) *reinterpret_cast<unsigned*>(yq + k) = 0u;
        if (c.t == 0) a.yscale[row] = 0.f;
      }
      continue;
    }
    const long long from = a.xidx ? row - j + clampi(a.xidx[row], 0, a.n - 1) : row;
    float x[E], v[E];
    c.load(static_cast<const T*>(a.x) + from * a.D, x);
#pragma unroll
    for (int i = 0; i < E; ++i) x[i] *= a.scale;
    if (a.t) {
      c.load(static_cast<const T*>(a.t) + row * a.D, v);
      float g[E];
      if (a.gate_mode) load_gate<T>(g, a, row, b, c);
      if (a.post) {
        normalise(v, c, red, a.rms, a.eps, fd);
        affine(v, a.post_w, a.post_b, c);
      }
      if (a.gate_mode) {
#pragma unroll
        for (int i = 0; i < E; ++i) x[i] = fmaf(g[i], v[i], x[i]);
      } else {
#pragma unroll
        for (int i = 0; i < E; ++i) x[i] += v[i];
      }
    }
    if (a.r) c.store(r, x);
    if (!a.pre) continue;
    normalise(x, c, red, a.rms, a.eps, fd);
    affine(x, a.pre_w, a.pre_b, c);
    if (a.y) c.store(y, x);
    if (a.yq) {  // the stored values, in the row's type
      float m = 0.f;
#pragma unroll
      for (int i = 0; i < E; ++i) {
        x[i] = (float)(T)x[i];
        m = vmax(m, fabsf(x[i]));
      }
      const RowQuant q = row_quant(red.max(m));
#pragma unroll
      for (int u = 0; u < kPer; ++u) {
        if constexpr (kVec == 4) {
          const unsigned p = pack_i8(quant_one<T>(q, x[4 * u]), quant_one<T>(q, x[4 * u + 1]),
                                     quant_one<T>(q, x[4 * u + 2]), quant_one<T>(q, x[4 * u + 3]));
          if (c.at(u) < Dp) *reinterpret_cast<unsigned*>(yq + c.at(u)) = p & q.live;
        } else {
          if (c.at(u) < Dp) yq[c.at(u)] = (int8_t)(quant_one<T>(q, x[u]) & q.live);
        }
      }
      if (c.t == 0) a.yscale[row] = q.scale;
    }
  }
}

// Backward.  With rhat, that the normalised rows and 1/s their factors:
//   d  = dr + (1/s) (g - [mean g] - rhat mean(g rhat)),  g = dy pre_w
//   dx = scale d;  du = gate d;  dgate = d u
//   dt = (1/s) (h - [mean h] - that mean(h that)),       h = du post_w
// ([ ]: LayerNorm only) and the sums over rows dpre_w = dy rhat, dpre_b = dy,
// dpost_w = du that, dpost_b = du.  A block takes items (sequence b, part ch):
// rows ch kRows + slot, step nch kRows, of the sequence (one sequence of all
// rows unless the gate goes by sequence), keeps the sums of its channels in
// registers, adds its row slots in order through LDS and leaves one partial
// record; k_norm_sums adds the records in order.
template <int kVec, int kPer, int kTpr>
SC_DEV void norm_input_grad(float* g, const float* hat, float inv, const Cols<kVec, kPer, kTpr>& c,
                            RowReduce<kTpr>& red, bool rms, float fd) {
  constexpr int E = kVec * kPer;
  float s = 0.f, m = 0.f;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    s = fmaf(g[i], hat[i], s);
    m += g[i];
  }
  s = red.sum(s) / fd;
  m = rms ? 0.f : red.sum(m) / fd;
#pragma unroll
  for (int i = 0; i < E; ++i) g[i] = inv * (g[i] - m - hat[i] * s);
}

constexpr int kNormBlocks = 512;  // blocks of the backward launch at most
enum { kSumPreW, kSumPreB, kSumPostW, kSumPostB, kSumGate, kSums };

struct NormPlan {
  int Bs, ns;       // sequences and rows of each, as the items see them
  int nch, blocks;  // parts of a sequence, blocks of the launch
};
SC_DEV __host__ bool norm_seq(const Norm& a) { return a.gate_mode == kGateSequence && a.dgate; }
NormPlan norm_plan(const Norm& a, int rows_per_block, bool seq) {
  NormPlan p;
  p.Bs = seq ? a.B : 1;
  p.ns = seq ? a.n : a.B * a.n;
  const int most = (int)(((long long)p.ns + rows_per_block - 1) / rows_per_block);
  p.nch = std::max(1, std::min(most, kNormBlocks / p.Bs));
  p.blocks = (int)std::min<long long>((long long)p.Bs * p.nch, kNormBlocks);
  return p;
}

// Adds the kRows row slots of v in order and stores the sum of the block's
// channels at out.  buf: LDS, kRows x D floats for kRows > 1.
template <int kVec, int kPer, int kTpr>
SC_DEV void block_sum(const float* v, float* out, float* buf, const Cols<kVec, kPer, kTpr>& c) {
  constexpr int kRows = kThreads<kTpr> / kTpr;
  if constexpr (kRows == 1) {
    c.store(out, v);
  } else {
    __syncthreads();
    c.store(buf + (threadIdx.x / kTpr) * c.D, v);
    __syncthreads();
    for (int k = threadIdx.x; k < c.D; k += 256) {
      float s = buf[k];
#pragma unroll
      for (int i = 1; i < kRows; ++i) s += buf[i * c.D + k];
      out[k] = s;
    }
  }
}

template <typename T, int kVec, int kPer, int kTpr>
__global__ __launch_bounds__(kThreads<kTpr>) void k_norm_bwd(Norm a, NormPlan pl) {
  constexpr int E = kVec * kPer, kRows = kThreads<kTpr> / kTpr;
  extern __shared__ __attribute__((aligned(16))) float buf[];
  __shared__ float slots[2 * kTpr / 64];
  RowReduce<kTpr> red{slots};
  const Cols<kVec, kPer, kTpr> c{a.D, (int)threadIdx.x % kTpr};
  const float fd = (float)a.D;
  const int slot = kTpr == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0;
  const bool seq = norm_seq(a);
  float sum[kSums][E];
#pragma unroll
  for (int k = 0; k < kSums; ++k)
#pragma unroll
    for (int i = 0; i < E; ++i) sum[k][i] = 0.f;
  const long long items = (long long)pl.Bs * pl.nch;
  float* gpart = a.ws + (long long)pl.blocks * kSums * a.D;
  for (long long it = blockIdx.x; it < items; it += gridDim.x) {
    const int bs = (int)(it / pl.nch), ch = (int)(it - (long long)bs * pl.nch);
    for (long long k = ch * kRows + slot; k < pl.ns; k += pl.nch * kRows) {
      const long long row = (long long)bs * pl.ns + k;
      const int b = (int)(row / a.n), j = (int)(row - (long long)b * a.n);
      if (a.len && j >= clampi(a.len[b], 0, a.n)) {
        if (a.dx) c.zero(static_cast<T*>(a.dx) + row * a.D);
        if (a.dt) c.zero(static_cast<T*>(a.dt) + row * a.D);
        if (a.dgate && a.gate_mode == kGateToken) c.zero(static_cast<T*>(a.dgate) + row * a.D);
        continue;
      }
      float x[E], that[E], g[E], dr[E], dy[E], tinv = 0.f;
      c.load(static_cast<const T*>(a.x) + row * a.D, x);
      if (a.t) c.load(static_cast<const T*>(a.t) + row * a.D, that);
      if (a.gate_mode) load_gate<T>(g, a, row, b, c);
      if (a.dr) {
        c.load(static_cast<const T*>(a.dr) + row * a.D, dr);
      } else {
#pragma unroll
        for (int i = 0; i < E; ++i) dr[i] = 0.f;
      }
      if (a.dy) c.load(static_cast<const T*>(a.dy) + row * a.D, dy);
      if (a.post) tinv = normalise(that, c, red, a.rms, a.eps, fd);
      // u, in its place of use: r below and dgate
      float u[E];
      if (a.t) {
#pragma unroll
        for (int i = 0; i < E; ++i) u[i] = that[i];
        if (a.post) affine(u, a.post_w, a.post_b, c);
      } else {
#pragma unroll
        for (int i = 0; i < E; ++i) u[i] = 0.f;
      }
      if (a.dy) {
#pragma unroll
        for (int i = 0; i < E; ++i) x[i] = fmaf(a.gate_mode ? g[i] : 1.f, u[i], a.scale * x[i]);
        const float rinv = normalise(x, c, red, a.rms, a.eps, fd);
#pragma unroll
        for (int i = 0; i < E; ++i) {
          sum[kSumPreW][i] = fmaf(dy[i], x[i], sum[kSumPreW][i]);
          sum[kSumPreB][i] += dy[i];
        }
        affine(dy, a.pre_w, nullptr, c);
        norm_input_grad(dy, x, rinv, c, red, a.rms, fd);
#pragma unroll
        for (int i = 0; i < E; ++i) dr[i] += dy[i];
      }
      if (a.dx) {
#pragma unroll
        for (int i = 0; i < E; ++i) x[i] = a.scale * dr[i];
        c.store(static_cast<T*>(a.dx) + row * a.D, x);
      }
      if (!a.t) continue;
      if (a.gate_mode) {
#pragma unroll
        for (int i = 0; i < E; ++i) u[i] *= dr[i];
        if (a.dgate && a.gate_mode == kGateToken) {
          c.store(static_cast<T*>(a.dgate) + row * a.D, u);
        } else {
#pragma unroll
          for (int i = 0; i < E; ++i) sum[kSumGate][i] += u[i];
        }
#pragma unroll
        for (int i = 0; i < E; ++i) dr[i] *= g[i];
      }
      if (a.post) {
#pragma unroll
        for (int i = 0; i < E; ++i) {
          sum[kSumPostW][i] = fmaf(dr[i], that[i], sum[kSumPostW][i]);
          sum[kSumPostB][i] += dr[i];
        }
        affine(dr, a.post_w, nullptr, c);
        norm_input_grad(dr, that, tinv, c, red, a.rms, fd);
      }
      if (a.dt) c.store(static_cast<T*>(a.dt) + row * a.D, dr);
    }
    if (seq) {
      block_sum(sum[kSumGate], gpart + it * a.D, buf, c);
#pragma unroll
      for (int i = 0; i < E; ++i) sum[kSumGate][i] = 0.f;
    }
  }
  float* part = a.ws + (long long)blockIdx.x * kSums * a.D;
  if (a.dpre_w) block_sum(sum[kSumPreW], part + kSumPreW * a.D, buf, c);
  if (a.dpre_b) block_sum(sum[kSumPreB], part + kSumPreB * a.D, buf, c);
  if (a.dpost_w) block_sum(sum[kSumPostW], part + kSumPostW * a.D, buf, c);
  if (a.dpost_b) block_sum(sum[kSumPostB], part + kSumPostB * a.D, buf, c);
  if (a.dgate && a.gate_mode == kGateChannel) block_sum(sum[kSumGate], part + kSumGate * a.D, buf, c);
}

// 64 channels of one output a workgroup: 16 waves add every 16th record in
// order, then the waves in order.  Outputs o < kSums: the sums over blocks;
// beyond: the gate's gradient of sequence o - kSums, over its parts.
template <typename T>
__global__ __launch_bounds__(1024) void k_norm_sums(Norm a, NormPlan pl) {
  __shared__ float buf[16][64];
  const int lane = threadIdx.x & 63, k = blockIdx.x * 64 + lane, w = threadIdx.x >> 6;
  const int count = kSums + (norm_seq(a) ? a.B : 0);
  for (int o = blockIdx.y; o < count; o += gridDim.y) {
    float* out = o == kSumPreW    ? a.dpre_w
                 : o == kSumPreB  ? a.dpre_b
                 : o == kSumPostW ? a.dpost_w
                 : o == kSumPostB ? a.dpost_b
                 : o == kSumGate && a.gate_mode == kGateChannel ? static_cast<float*>(a.dgate) : nullptr;
    if (o < kSums && !out) continue;
    const long long step = o < kSums ? (long long)kSums * a.D : a.D;
    const float* src = a.ws + (o < kSums ? (long long)o * a.D
                                         : ((long long)pl.blocks * kSums + (long long)(o - kSums) * pl.nch) * a.D);
    const int records = o < kSums ? pl.blocks : pl.nch;
    float s = 0.f;
    if (k < a.D) {
#pragma unroll 8
      for (int i = w; i < records; i += 16) s += src[i * step + k];
    }
    buf[w][lane] = s;
    __syncthreads();
    if (w == 0 && k < a.D) {
#pragma unroll
      for (int i = 1; i < 16; ++i) s += buf[i][lane];
      if (o < kSums)
        out[k] = s;
      else
        static_cast<T*>(a.dgate)[(long long)(o - kSums) * a.D + k] = (T)s;
    }
    __syncthreads();
  }
}

template <int kV, int kP, int kT>
struct NormShape {
  static constexpr int kVec = kV, kPer = kP, kTpr = kT;
};

// Calls f with the shape for D: a wavefront per row up to 1024 channels (256 where
// rows are not aligned), a workgroup beyond.
template <typename F>
hipError_t norm_shape(int D, bool vec, F&& f) {
  if (vec) {
    if (D <= 256) return f(NormShape<4, 1, 64>{});
    if (D <= 512) return f(NormShape<4, 2, 64>{});
    if (D <= 768) return f(NormShape<4, 3, 64>{});
    if (D <= 1024) return f(NormShape<4, 4, 64>{});
    if (D <= 2048) return f(NormShape<4, 2, 256>{});
    return f(NormShape<4, 2, 512>{});
  }
  if (D <= 256) return f(NormShape<1, 4, 64>{});
  if (D <= 1024) return f(NormShape<1, 4, 256>{});
  if (D <= 2048) return f(NormShape<1, 8, 256>{});
  return f(NormShape<1, 8, 512>{});
}

// Every row of every tensor starts at a multiple of an access of four.
bool norm_vec(const Norm& a) {
  const uintptr_t e = a.f32 ? 16 : 8;
  uintptr_t all = 0;
  for (const void* p : {a.x, a.t, (const void*)a.r, (const void*)a.y, a.dr, a.dy, (const void*)a.dx, (const void*)a.dt})
    all |= reinterpret_cast<uintptr_t>(p) & (e - 1);
  for (const float* p : {a.post_w, a.post_b, a.pre_w, a.pre_b}) all |= reinterpret_cast<uintptr_t>(p) & 15;
  for (const void* p : {a.gate, (const void*)a.dgate})
    all |= reinterpret_cast<uintptr_t>(p) & (a.gate_mode == kGateChannel ? 15 : e - 1);
  all |= reinterpret_cast<uintptr_t>(a.yq) & 3;
  return a.D % 4 == 0 && all == 0;
}

template <typename T>
hipError_t run_norm(const Norm& a, hipStream_t s) {
  return norm_shape(a.D, norm_vec(a), [&](auto shape) {
    using S = decltype(shape);
    constexpr int kT = kThreads<S::kTpr>;
    const long long rows = (long long)a.B * a.n, per = kT / S::kTpr;
    const unsigned blocks = (unsigned)std::min<long long>((rows + per - 1) / per, 8192);
    hipLaunchKernelGGL((k_norm<T, S::kVec, S::kPer, S::kTpr>), dim3(blocks), dim3(kT), 0, s, a);
    return hipGetLastError();
  });
}

template <typename T>
hipError_t run_norm_backward(const Norm& a, hipStream_t s) {
  return norm_shape(a.D, norm_vec(a), [&](auto shape) {
    using S = decltype(shape);
    constexpr int kT = kThreads<S::kTpr>, kRows = kT / S::kTpr;
    const bool seq = norm_seq(a);
    const NormPlan pl = norm_plan(a, kRows, seq);
    hipLaunchKernelGGL((k_norm_bwd<T, S::kVec, S::kPer, S::kTpr>), dim3(pl.blocks), dim3(kT),
                       kRows > 1 ? kRows * a.D * sizeof(float) : 0, s, a, pl);
    if (a.dpre_w || a.dpre_b || a.dpost_w || a.dpost_b || (a.gate_mode == kGateChannel && a.dgate) || seq)
      hipLaunchKernelGGL(k_norm_sums<T>, dim3((a.D + 63) / 64, std::min(kSums + (seq ? a.B : 0), 32768)), dim3(1024), 0,
                         s, a, pl);
    return hipGetLastError();
  });
}

}  // namespace

hipError_t launch_block_norm(const Norm& a, hipStream_t s) {
  return a.f32 ? run_norm<float>(a, s) : run_norm<__bf16>(a, s);
}

// The records of every block and, for a gate by sequence, of every item: the
// most over what the tensors' alignment and a missing dgate may choose.
size_t block_norm_backward_floats(const Norm& a) {
  size_t most = 0;
  for (int rows : {1, 4})
    for (int seq = 0; seq <= (a.gate_mode == kGateSequence ? 1 : 0); ++seq) {
      const NormPlan pl = norm_plan(a, rows, seq);
      most = std::max(most, ((size_t)pl.blocks * kSums + (seq ? (size_t)pl.Bs * pl.nch : 0)) * a.D);
    }
  return most;
}

hipError_t launch_block_norm_backward(const Norm& a, hipStream_t s) {
  return a.f32 ? run_norm_backward<float>(a, s) : run_norm_backward<__bf16>(a, s);
}

}  // namespace sc
