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
//
// Both are bound by memory: 32768 x 1024 bf16 with both norms and a gate by
// channel or sequence, forward 268 MB in 45-54 us (5.0-6.0 TB/s; a large copy 5.1),
// backward 403 MB in 86-95 us and its sums in 4-5; as float32 backward 805 MB in 154-158.
// Rows of more than 1024 channels wait for their workgroup's reductions: 3 x 501 x 1111
// float32 backward 20 us and its sums 4, where the bytes take 7.
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

// Sums (one, or two at once) or maximum over the threads of a row: a wavefront, or those
// of a workgroup through LDS (two sets of slots in turn: a set is written again only
// after the barrier of the other).
template <int kTpr>
struct RowReduce {
  static constexpr int kWaves = kTpr / 64;
  float* slots;  // LDS, 2 x 2 x kWaves
  int flip = 0;
  SC_DEV const float* share(float v, float v2 = 0.f) {
    float* s = slots + 2 * kWaves * flip;
    flip ^= 1;
    if ((threadIdx.x & 63) == 0) {
      s[threadIdx.x >> 6] = v;
      s[kWaves + (threadIdx.x >> 6)] = v2;
    }
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
  SC_DEV void sum(float& v, float& v2) {
    v = butterfly_sum(v);
    v2 = butterfly_sum(v2);
    if constexpr (kWaves > 1) {
      const float* s = share(v, v2);
      v = s[0];
      v2 = s[kWaves];
#pragma unroll
      for (int i = 1; i < kWaves; ++i) {
        v += s[i];
        v2 += s[kWaves + i];
      }
    }
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

// One access of a thread: kVec elements of T, as the bits that buffer loads and
// stores move.
template <typename T, int kVec>
struct Bits;
template <>
struct Bits<float, 4> {
  using Raw = __attribute__((ext_vector_type(4))) unsigned;
  SC_DEV static Raw load(__amdgpu_buffer_rsrc_t r, int off) { return __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, 0); }
  SC_DEV static void store(__amdgpu_buffer_rsrc_t r, int off, Raw v) {
    __builtin_amdgcn_raw_buffer_store_b128(v, r, off, 0, 0);
  }
  SC_DEV static void unpack(Raw v, float* f) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const unsigned e = v[q];  // the bit cast of a vector's element reads its first one
      f[q] = __builtin_bit_cast(float, e);
    }
  }
  SC_DEV static Raw pack(const float* f) {
    return Raw{__builtin_bit_cast(unsigned, f[0]), __builtin_bit_cast(unsigned, f[1]),
               __builtin_bit_cast(unsigned, f[2]), __builtin_bit_cast(unsigned, f[3])};
  }
};
template <>
struct Bits<__bf16, 4> {
  using Raw = __attribute__((ext_vector_type(2))) unsigned;
  SC_DEV static Raw load(__amdgpu_buffer_rsrc_t r, int off) { return __builtin_amdgcn_raw_buffer_load_b64(r, off, 0, 0); }
  SC_DEV static void store(__amdgpu_buffer_rsrc_t r, int off, Raw v) {
    __builtin_amdgcn_raw_buffer_store_b64(v, r, off, 0, 0);
  }
  SC_DEV static void unpack(Raw v, float* f) {
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      f[2 * q] = __builtin_bit_cast(float, v[q] << 16);
      f[2 * q + 1] = __builtin_bit_cast(float, v[q] & 0xffff0000u);
    }
  }
  SC_DEV static Raw pack(const float* f) { return Raw{pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3])}; }
};
template <>
struct Bits<float, 1> {  // weights, beside bf16 rows an element an access
  using Raw = unsigned;
  SC_DEV static Raw load(__amdgpu_buffer_rsrc_t r, int off) { return __builtin_amdgcn_raw_buffer_load_b32(r, off, 0, 0); }
  SC_DEV static void unpack(Raw v, float* f) { *f = __builtin_bit_cast(float, v); }
};
template <>
struct Bits<__bf16, 1> {
  using Raw = unsigned short;
  SC_DEV static Raw load(__amdgpu_buffer_rsrc_t r, int off) { return __builtin_amdgcn_raw_buffer_load_b16(r, off, 0, 0); }
  SC_DEV static void store(__amdgpu_buffer_rsrc_t r, int off, Raw v) {
    __builtin_amdgcn_raw_buffer_store_b16(v, r, off, 0, 0);
  }
  SC_DEV static void unpack(Raw v, float* f) { *f = __builtin_bit_cast(float, (unsigned)v << 16); }
  SC_DEV static Raw pack(const float* f) { return __builtin_bit_cast(unsigned short, (__bf16)*f); }
};

// One row of a tensor as a buffer of its D elements: accesses beyond it load zeros
// and store nothing, so the channels past D need no branch, nor does an absent
// tensor (a buffer of no elements).  The hardware checks every dword of an access, and
// needs no more than dword alignment, so rows that end inside an access are fine.
// With a branch around each access the compiler waited for every load on its own
// (backward of 32768 x 1024: 229 us).
template <typename T>
SC_DEV __amdgpu_buffer_rsrc_t row_buffer(const T* base, long long row, int D, bool present) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(base) + row * D, 0, present ? D * (int)sizeof(T) : 0,
                                           0x00027000);
}

// The channels of a thread: kPer accesses of kVec, access u at (u kTpr + thread)
// kVec; kWidth of them in all, D used.
template <typename T, int kVec, int kPer, int kTpr>
struct Cols {
  using B = Bits<T, kVec>;
  using Raw = typename B::Raw;
  static constexpr int kWidth = kVec * kPer * kTpr, kPerThread = kPer;
  int D, t;  // t: thread of the row
  SC_DEV int at(int u) const { return (u * kTpr + t) * kVec; }
  SC_DEV bool in(int u, int q) const { return at(u) + q < D; }
  SC_DEV void load(__amdgpu_buffer_rsrc_t r, Raw (&v)[kPer]) const {
#pragma unroll
    for (int u = 0; u < kPer; ++u) v[u] = B::load(r, at(u) * (int)sizeof(T));
  }
  SC_DEV void unpack(const Raw (&r)[kPer], float* v) const {
#pragma unroll
    for (int u = 0; u < kPer; ++u) B::unpack(r[u], v + u * kVec);
  }
  SC_DEV void store(__amdgpu_buffer_rsrc_t r, const float* v) const {
#pragma unroll
    for (int u = 0; u < kPer; ++u) B::store(r, at(u) * (int)sizeof(T), B::pack(v + u * kVec));
  }
  SC_DEV void zero(__amdgpu_buffer_rsrc_t r) const {
    const float z[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < kPer; ++u) B::store(r, at(u) * (int)sizeof(T), B::pack(z));
  }
  // access u of one of the weight rows in LDS, or all of it
  SC_DEV void weight(const float* lds, int u, float* v) const {
    if constexpr (kVec == 4) {
      const f32x4 x = *reinterpret_cast<const f32x4*>(lds + at(u));
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] = x[q];
    } else {
      *v = lds[at(u)];
    }
  }
  SC_DEV void weights(const float* lds, float* v) const {
#pragma unroll
    for (int u = 0; u < kPer; ++u) weight(lds, u, v + u * kVec);
  }
};

// Both norms' weights and a gate by channel in LDS, a row of kWidth each: absent
// ones are 1 and 0, the channels past D are 0 (so that sums over them stay 0).  The
// row slots share the rows, and a slot's loads are all in flight together (one at a
// time they took 40 round trips at 1111 channels: 25 us of a backward launch).
enum { kPostW, kPostB, kPreW, kPreB, kGateRow, kWeights };
template <int kVec, int kPer, int kTpr>
SC_DEV void stage_weights(float* lds, const Norm& a, int count) {
  using C = Cols<float, kVec, kPer, kTpr>;
  constexpr int kRows = kThreads<kTpr> / kTpr, kMine = (kWeights + kRows - 1) / kRows;
  const C c{a.D, (int)threadIdx.x % kTpr};
  const int slot = kRows > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / kTpr) : 0;
  const float* src[kWeights] = {a.post_w, a.post_b, a.pre_w, a.pre_b,
                                a.gate_mode == kGateChannel ? static_cast<const float*>(a.gate) : nullptr};
  typename C::Raw raw[kMine][kPer];
#pragma unroll
  for (int m = 0; m < kMine; ++m) {
    const float* p = nullptr;
#pragma unroll
    for (int k = 0; k < kWeights; ++k)
      if (k == slot + m * kRows && k < count) p = src[k];
    c.load(row_buffer(p, 0, a.D, p != nullptr), raw[m]);
  }
#pragma unroll
  for (int m = 0; m < kMine; ++m) {
    const int k = slot + m * kRows;
    if (k >= count) continue;
    bool have = false;
#pragma unroll
    for (int i = 0; i < kWeights; ++i)
      if (i == k) have = src[i] != nullptr;
    const float absent = k == kPostB || k == kPreB ? 0.f : 1.f;
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
      float v[kVec];
      C::B::unpack(raw[m][u], v);
#pragma unroll
      for (int q = 0; q < kVec; ++q)
        lds[k * C::kWidth + c.at(u) + q] = have || !c.in(u, q) ? v[q] : absent;
    }
  }
  __syncthreads();
}

// v -> (v - mean) / sqrt(var + eps), or v / sqrt(mean(v^2) + eps); channels beyond
// D stay 0.  Returns the factor.
template <typename C, typename R, int E>
SC_DEV float normalise(float (&v)[E], const C& c, R& red, bool rms, float eps, float fd) {
  constexpr int kPer = C::kPerThread, kVec = E / kPer;
  if (!rms) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < E; ++i) s += v[i];
    const float mean = red.sum(s) / fd;  // divided: a constant row of an exact sum has no deviation
#pragma unroll
    for (int u = 0; u < kPer; ++u)
#pragma unroll
      for (int q = 0; q < kVec; ++q) v[u * kVec + q] -= c.in(u, q) ? mean : 0.f;
  }
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < E; ++i) s = fmaf(v[i], v[i], s);
  const float inv = 1.f / sqrtf(red.sum(s) / fd + eps);
#pragma unroll
  for (int i = 0; i < E; ++i) v[i] *= inv;
  return inv;
}

// v = v w + b from the weight rows
template <typename C, int E>
SC_DEV void affine(float (&v)[E], const float* lds, int w, int b, const C& c) {
  float p[E], q[E];
  c.weights(lds + w * C::kWidth, p);
  c.weights(lds + b * C::kWidth, q);
#pragma unroll
  for (int i = 0; i < E; ++i) v[i] = fmaf(v[i], p[i], q[i]);
}
template <typename C, int E>
SC_DEV void times(float (&v)[E], const float* lds, int w, const C& c) {
  float p[E];
  c.weights(lds + w * C::kWidth, p);
#pragma unroll
  for (int i = 0; i < E; ++i) v[i] *= p[i];
}

// A row's sequence and whether it is padding; all of it wave-uniform.
struct RowAt {
  unsigned row;
  int b;
  bool live;
};
SC_DEV RowAt row_at(const Norm& a, unsigned row, bool exists) {
  RowAt r;
  r.row = row;
  r.b = exists ? (int)(row / (unsigned)a.n) : 0;
  r.live = exists && (!a.len || (int)(row - (unsigned)r.b * a.n) < clampi(scalar_load(a.len, r.b), 0, a.n));
  return r;
}
// The gate's row of a gate by sequence or token.
SC_DEV long long gate_row(const Norm& a, const RowAt& r) {
  return a.gate_mode == kGateSequence ? (long long)r.b : (long long)r.row;
}
SC_DEV bool gate_rows(const Norm& a) { return a.gate_mode >= kGateSequence; }

// Rows dealt round-robin over the launch's row slots.  The next row's loads are in
// flight while a row is computed, the first row's while the weights are staged.
template <typename T, int kVec, int kPer, int kTpr>
__global__ __launch_bounds__(kThreads<kTpr>) void k_norm(Norm a) {
  constexpr int E = kVec * kPer, kRows = kThreads<kTpr> / kTpr;
  using C = Cols<T, kVec, kPer, kTpr>;
  __shared__ float slots[4 * kTpr / 64];
  __shared__ __attribute__((aligned(16))) float lw[kWeights * C::kWidth];
  RowReduce<kTpr> red{slots};
  const C c{a.D, (int)threadIdx.x % kTpr};
  const float fd = (float)a.D;
  const int Dp = (a.D + kI8Pitch - 1) / kI8Pitch * kI8Pitch;
  const unsigned rows = (unsigned)a.B * (unsigned)a.n, step = gridDim.x * kRows;
  // Slot i's row of round k is k step + (i + k turn) mod step: without the turn a slot
  // whose place in the sequences is padding in one round would be so in every round.
  const unsigned turn = (unsigned)(0.382f * (float)step) / kRows * kRows;
  const unsigned slot = kTpr == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0;
  typename C::Raw rx[kPer], rt[kPer], rg[kPer];
  auto fetch = [&](const RowAt& r) {
    long long from = r.row;
    if (a.xidx && r.live) from = (long long)r.b * a.n + clampi(scalar_load(a.xidx, r.row), 0, a.n - 1);
    c.load(row_buffer(static_cast<const T*>(a.x), from, a.D, r.live), rx);
    c.load(row_buffer(static_cast<const T*>(a.t), r.row, a.D, r.live && a.t), rt);
    if (gate_rows(a)) c.load(row_buffer(static_cast<const T*>(a.gate), gate_row(a, r), a.D, r.live), rg);
  };
  unsigned place = blockIdx.x * kRows + slot, round = 0;  // round: its first row
  RowAt cur = row_at(a, place, place < rows);
  fetch(cur);
  stage_weights<kVec, kPer, kTpr>(lw, a, kWeights);
  while (round < rows) {
    round += step;  // below 2^31 + 2^24
    place = place + turn < step ? place + turn : place + turn - step;
    const RowAt next = row_at(a, round + place, round + place < rows);
    if (cur.row >= rows) {  // the last round is not whole
      cur = next;
      continue;
    }
    const long long row = cur.row;
    const auto r = row_buffer(static_cast<const T*>(a.r), row, a.D, a.r);
    const auto y = row_buffer(static_cast<const T*>(a.y), row, a.D, a.y);
    int8_t* yq = a.yq + row * Dp;
    if (!cur.live) {
      fetch(next);
      if (!a.skip_pad) {
        if (a.r) c.zero(r);
        if (a.y) c.zero(y);
        if (a.yq) {
          for (int k = 4 * c.t; k < Dp; k += 4 * kTpr) *reinterpret_cast<unsigned*>(yq + k) = 0u;
          if (c.t == 0) a.yscale[row] = 0.f;
        }
      }
      cur = next;
      continue;
    }
    float x[E], v[E], g[E];
    c.unpack(rx, x);
    c.unpack(rt, v);
    if (gate_rows(a))
      c.unpack(rg, g);
    else
      c.weights(lw + kGateRow * C::kWidth, g);
    fetch(next);
    if (a.post) {
      normalise(v, c, red, a.rms, a.eps, fd);
      affine(v, lw, kPostW, kPostB, c);
    }
#pragma unroll
    for (int i = 0; i < E; ++i) x[i] = fmaf(g[i], v[i], a.scale * x[i]);
    if (a.r) c.store(r, x);
    if (a.pre) {
      normalise(x, c, red, a.rms, a.eps, fd);
      affine(x, lw, kPreW, kPreB, c);
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
          if (c.at(u) >= Dp) continue;
          if constexpr (kVec == 4) {
            const unsigned p = pack_i8(quant_one<T>(q, x[4 * u]), quant_one<T>(q, x[4 * u + 1]),
                                       quant_one<T>(q, x[4 * u + 2]), quant_one<T>(q, x[4 * u + 3]));
            *reinterpret_cast<unsigned*>(yq + c.at(u)) = p & q.live;
          } else {
            yq[c.at(u)] = (int8_t)(quant_one<T>(q, x[u]) & q.live);
          }
        }
        if (c.t == 0) a.yscale[row] = q.scale;
      }
    }
    cur = next;
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
template <typename R, int E>
SC_DEV void norm_input_grad(float (&g)[E], const float (&hat)[E], float inv, R& red, bool rms, float fd) {
  float s = 0.f, m = 0.f;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    s = fmaf(g[i], hat[i], s);
    m += g[i];
  }
  red.sum(s, m);
  s /= fd;
  m = rms ? 0.f : m / fd;
#pragma unroll
  for (int i = 0; i < E; ++i) g[i] = inv * (g[i] - fmaf(hat[i], s, m));
}

constexpr int kNormFwdBlocks = 2048;  // blocks of the forward launch at most
constexpr int kNormBlocks = 512;      // and of the backward launch
enum { kSumPreW, kSumPreB, kSumPostW, kSumPostB, kSumGate, kSums };

struct NormPlan {
  int Bs, ns;       // sequences and rows of each, as the items see them
  int nch, blocks;  // parts of a sequence, blocks of the launch
};
NormPlan norm_plan(const Norm& a, int rows_per_block) {
  const bool seq = a.gate_mode == kGateSequence;
  NormPlan p;
  p.Bs = seq ? a.B : 1;
  p.ns = seq ? a.n : a.B * a.n;
  const int most = (int)(((long long)p.ns + rows_per_block - 1) / rows_per_block);
  p.nch = std::max(1, std::min(most, kNormBlocks / p.Bs));
  p.blocks = (int)std::min<long long>((long long)p.Bs * p.nch, kNormBlocks);
  return p;
}

// Adds the row slots of v in order and stores the sum of the block's channels at
// out.  buf: LDS, kRows x kWidth floats.
template <typename C, int kRows, int E>
SC_DEV void block_sum(const float (&v)[E], float* out, float* buf, const C& c) {
  constexpr int kPer = C::kPerThread, kVec = E / kPer;
  const int slot = threadIdx.x / (blockDim.x / kRows);
  __syncthreads();
#pragma unroll
  for (int u = 0; u < kPer; ++u)
#pragma unroll
    for (int q = 0; q < kVec; ++q) buf[slot * C::kWidth + c.at(u) + q] = v[u * kVec + q];
  __syncthreads();
  for (int k = threadIdx.x; k < c.D; k += blockDim.x) {
    float s = buf[k];
#pragma unroll
    for (int i = 1; i < kRows; ++i) s += buf[i * C::kWidth + k];
    out[k] = s;
  }
}

// kToken: a gate by token, read with the rows; else the gate's row (of ones, the
// channels' or the sequence's) is in LDS.  Weights and gate are read from LDS
// where they are used, u is made twice: at 16 channels a thread the sums, the rows
// in flight and the row at hand leave no registers for them.
template <typename T, int kVec, int kPer, int kTpr, bool kToken>
__global__ __launch_bounds__(kThreads<kTpr>) __attribute__((amdgpu_waves_per_eu(2))) void k_norm_bwd(Norm a,
                                                                                                     NormPlan pl) {
  constexpr int E = kVec * kPer, kRows = kThreads<kTpr> / kTpr;
  using C = Cols<T, kVec, kPer, kTpr>;
  __shared__ float slots[4 * kTpr / 64];
  __shared__ __attribute__((aligned(16))) float lw[kWeights * C::kWidth], buf[kRows * C::kWidth];
  RowReduce<kTpr> red{slots};
  const C c{a.D, (int)threadIdx.x % kTpr};
  const float fd = (float)a.D;
  const unsigned slot = kTpr == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0;
  const bool seq = a.gate_mode == kGateSequence;
  float sum[kSums][E];
#pragma unroll
  for (int k = 0; k < kSums; ++k)
#pragma unroll
    for (int i = 0; i < E; ++i) sum[k][i] = 0.f;
  typename C::Raw rx[kPer], rt[kPer], rg[kPer], rr[kPer], ry[kPer];
  auto fetch = [&](const RowAt& r) {
    c.load(row_buffer(static_cast<const T*>(a.t), r.row, a.D, r.live && a.t), rt);
    c.load(row_buffer(static_cast<const T*>(a.x), r.row, a.D, r.live), rx);
    if constexpr (kToken) c.load(row_buffer(static_cast<const T*>(a.gate), r.row, a.D, r.live), rg);
    c.load(row_buffer(static_cast<const T*>(a.dy), r.row, a.D, r.live && a.dy), ry);
    c.load(row_buffer(static_cast<const T*>(a.dr), r.row, a.D, r.live && a.dr), rr);
  };
  const unsigned items = (unsigned)pl.Bs * (unsigned)pl.nch, step = (unsigned)pl.nch * kRows;
  float* gpart = a.ws + (long long)pl.blocks * kSums * a.D;
  bool staged = false;
  for (unsigned it = blockIdx.x; it < items; it += gridDim.x) {
    const unsigned bs = it / (unsigned)pl.nch, first = bs * (unsigned)pl.ns;
    const unsigned end = first + (unsigned)pl.ns;  // this item's rows: below 2^31
    const unsigned row = first + (it - bs * (unsigned)pl.nch) * kRows + slot;
    RowAt cur = row_at(a, row, row < end);
    fetch(cur);
    if (seq) {
      __syncthreads();  // the last item's rows are done
      if (threadIdx.x < kTpr) {
        typename C::Raw rg[kPer];
        c.load(row_buffer(static_cast<const T*>(a.gate), bs, a.D, true), rg);
#pragma unroll
        for (int u = 0; u < kPer; ++u) C::B::unpack(rg[u], lw + kGateRow * C::kWidth + c.at(u));
      }
      if (staged) __syncthreads();
    }
    if (!staged) stage_weights<kVec, kPer, kTpr>(lw, a, seq ? kGateRow : kWeights);
    staged = true;
    for (; cur.row < end;) {
      const RowAt next = row_at(a, cur.row + step, cur.row + step < end);
      const auto dx = row_buffer(static_cast<const T*>(a.dx), cur.row, a.D, a.dx);
      const auto dt = row_buffer(static_cast<const T*>(a.dt), cur.row, a.D, a.dt);
      const auto dg = row_buffer(static_cast<const T*>(a.dgate), cur.row, a.D, kToken && a.dgate);
      if (!cur.live) {
        fetch(next);
        c.zero(dx);
        c.zero(dt);
        if (kToken) c.zero(dg);
        cur = next;
        continue;
      }
      float x[E], that[E], g[E], dr[E], dy[E], tinv = 0.f;
      c.unpack(rt, that);
      c.unpack(rx, x);
      if constexpr (kToken) c.unpack(rg, g);
      c.unpack(ry, dy);
      c.unpack(rr, dr);
      fetch(next);
      if (a.post) tinv = normalise(that, c, red, a.rms, a.eps, fd);
      // u of access k, and the gate unless it came with the row
      auto block = [&](int k, float (&u)[kVec]) {
        float w[kVec], b[kVec];
#pragma unroll
        for (int q = 0; q < kVec; ++q) u[q] = that[k * kVec + q];
        if (a.post) {
          c.weight(lw + kPostW * C::kWidth, k, w);
          c.weight(lw + kPostB * C::kWidth, k, b);
#pragma unroll
          for (int q = 0; q < kVec; ++q) u[q] = fmaf(u[q], w[q], b[q]);
        }
      };
      auto gate = [&](int k, float (&v)[kVec]) {
        if constexpr (kToken) {
#pragma unroll
          for (int q = 0; q < kVec; ++q) v[q] = g[k * kVec + q];
        } else {
          c.weight(lw + kGateRow * C::kWidth, k, v);
        }
      };
      if (a.dy) {
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
          float u[kVec], v[kVec];
          block(k, u);
          gate(k, v);
#pragma unroll
          for (int q = 0; q < kVec; ++q) x[k * kVec + q] = fmaf(v[q], u[q], a.scale * x[k * kVec + q]);
        }
        const float rinv = normalise(x, c, red, a.rms, a.eps, fd);
#pragma unroll
        for (int i = 0; i < E; ++i) {
          sum[kSumPreW][i] = fmaf(dy[i], x[i], sum[kSumPreW][i]);
          sum[kSumPreB][i] += dy[i];
        }
        times(dy, lw, kPreW, c);
        norm_input_grad(dy, x, rinv, red, a.rms, fd);
#pragma unroll
        for (int i = 0; i < E; ++i) dr[i] += dy[i];
      }
#pragma unroll
      for (int i = 0; i < E; ++i) x[i] = a.scale * dr[i];
      c.store(dx, x);
      if (a.gate_mode) {
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
          float u[kVec], v[kVec];
          block(k, u);
          gate(k, v);
#pragma unroll
          for (int q = 0; q < kVec; ++q) {
            const int i = k * kVec + q;
            if constexpr (kToken)
              x[i] = u[q] * dr[i];
            else
              sum[kSumGate][i] = fmaf(u[q], dr[i], sum[kSumGate][i]);
            dr[i] *= v[q];
          }
        }
        if constexpr (kToken) c.store(dg, x);
      }
      if (a.post) {
#pragma unroll
        for (int i = 0; i < E; ++i) {
          sum[kSumPostW][i] = fmaf(dr[i], that[i], sum[kSumPostW][i]);
          sum[kSumPostB][i] += dr[i];
        }
        times(dr, lw, kPostW, c);
        norm_input_grad(dr, that, tinv, red, a.rms, fd);
      }
      c.store(dt, dr);
      cur = next;
    }
    if (seq && a.dgate) {
      block_sum<C, kRows>(sum[kSumGate], gpart + (long long)it * a.D, buf, c);
#pragma unroll
      for (int i = 0; i < E; ++i) sum[kSumGate][i] = 0.f;
    }
  }
  float* part = a.ws + (long long)blockIdx.x * kSums * a.D;
  if (a.dpre_w) block_sum<C, kRows>(sum[kSumPreW], part + kSumPreW * a.D, buf, c);
  if (a.dpre_b) block_sum<C, kRows>(sum[kSumPreB], part + kSumPreB * a.D, buf, c);
  if (a.dpost_w) block_sum<C, kRows>(sum[kSumPostW], part + kSumPostW * a.D, buf, c);
  if (a.dpost_b) block_sum<C, kRows>(sum[kSumPostB], part + kSumPostB * a.D, buf, c);
  if (a.dgate && a.gate_mode == kGateChannel) block_sum<C, kRows>(sum[kSumGate], part + kSumGate * a.D, buf, c);
}

// 64 channels of one output a workgroup: 16 waves add every 16th record in
// order, then the waves in order.  Outputs o < kSums: the sums over blocks;
// beyond: the gate's gradient of sequence o - kSums, over its parts.
template <typename T>
__global__ __launch_bounds__(1024) void k_norm_sums(Norm a, NormPlan pl) {
  __shared__ float buf[16][64];
  const int lane = threadIdx.x & 63, k = blockIdx.x * 64 + lane, w = threadIdx.x >> 6;
  const int count = kSums + (a.gate_mode == kGateSequence && a.dgate ? a.B : 0);
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

// Calls f with the shape for D: a wavefront per row up to 1024 channels (256 for bf16
// rows of odd length or address, an element an access), a workgroup beyond.
template <typename T, typename F>
hipError_t norm_shape(int D, bool vec, F&& f) {
  if (sizeof(T) == 4 || vec) {
    if (D <= 256) return f(NormShape<4, 1, 64>{});
    if (D <= 512) return f(NormShape<4, 2, 64>{});
    if (D <= 768) return f(NormShape<4, 3, 64>{});
    if (D <= 1024) return f(NormShape<4, 4, 64>{});
    if (D <= 2048) return f(NormShape<4, 2, 256>{});
    return f(NormShape<4, 2, 512>{});
  }
  if constexpr (sizeof(T) == 2) {
    if (D <= 256) return f(NormShape<1, 4, 64>{});
    if (D <= 1024) return f(NormShape<1, 4, 256>{});
    if (D <= 2048) return f(NormShape<1, 8, 256>{});
    return f(NormShape<1, 8, 512>{});
  }
  return hipErrorInvalidValue;  // not reached
}

// Rows of four elements an access: every row of every tensor starts at a dword.
// (yq is 16-byte aligned.)
bool norm_vec(const Norm& a) {
  if (a.f32) return true;
  uintptr_t all = 0;
  for (const void* p : {a.x, a.t, (const void*)a.r, (const void*)a.y, a.dr, a.dy, (const void*)a.dx, (const void*)a.dt})
    all |= reinterpret_cast<uintptr_t>(p) & 3;
  if (a.gate_mode != kGateChannel) all |= (reinterpret_cast<uintptr_t>(a.gate) | reinterpret_cast<uintptr_t>(a.dgate)) & 3;
  return a.D % 2 == 0 && all == 0;
}

template <typename T>
hipError_t run_norm(const Norm& a, hipStream_t s) {
  return norm_shape<T>(a.D, norm_vec(a), [&](auto shape) {
    using S = decltype(shape);
    constexpr int kT = kThreads<S::kTpr>;
    const long long rows = (long long)a.B * a.n, per = kT / S::kTpr;
    const unsigned blocks = (unsigned)std::min<long long>((rows + per - 1) / per, kNormFwdBlocks);
    hipLaunchKernelGGL((k_norm<T, S::kVec, S::kPer, S::kTpr>), dim3(blocks), dim3(kT), 0, s, a);
    return hipGetLastError();
  });
}

template <typename T>
hipError_t run_norm_backward(const Norm& a, hipStream_t s) {
  return norm_shape<T>(a.D, norm_vec(a), [&](auto shape) {
    using S = decltype(shape);
    constexpr int kT = kThreads<S::kTpr>, kRows = kT / S::kTpr;
    const bool seq = a.gate_mode == kGateSequence && a.dgate;
    const NormPlan pl = norm_plan(a, kRows);
    if (a.gate_mode == kGateToken)
      hipLaunchKernelGGL((k_norm_bwd<T, S::kVec, S::kPer, S::kTpr, true>), dim3(pl.blocks), dim3(kT), 0, s, a, pl);
    else
      hipLaunchKernelGGL((k_norm_bwd<T, S::kVec, S::kPer, S::kTpr, false>), dim3(pl.blocks), dim3(kT), 0, s, a, pl);
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
// most over the rows per block that the tensors' alignment may choose.
size_t block_norm_backward_floats(const Norm& a) {
  size_t most = 0;
  for (int rows : {1, 4}) {
    const NormPlan pl = norm_plan(a, rows);
    most = std::max(most,
                    ((size_t)pl.blocks * kSums + (a.gate_mode == kGateSequence ? (size_t)pl.Bs * pl.nch : 0)) * a.D);
  }
  return most;
}

hipError_t launch_block_norm_backward(const Norm& a, hipStream_t s) {
  return a.f32 ? run_norm_backward<float>(a, s) : run_norm_backward<__bf16>(a, s);
}

}  // namespace sc
