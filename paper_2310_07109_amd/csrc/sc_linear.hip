// Matrix products in 8-bit integers with a scale for each token and channel.
//
//   out[t, n] = act(s_t w_n sum_k q[t, k] wq[n, k] + bias[n])
//
// k_quant_rows    the tokens' 8-bit rows (sc_quant.h), one wavefront a row.
// k_quant_weight  the weights', once per model.
// k_linear        the product on v_mfma_i32_32x32x32_i8: sums of up to 131072
//                 products of 127 x 127 fit an int32, so they are exact in any
//                 order, and a row's result does not depend on the tile that
//                 computed it.
// k_linear_few    the same for a few rows: quantisation and product in one launch.
#include <algorithm>

#include "sc_device.h"
#include "sc_internal.h"
#include "sc_pack.h"
#include "sc_quant.h"

namespace sc {
namespace {

typedef __attribute__((ext_vector_type(4))) int i32x4;
typedef __attribute__((ext_vector_type(16))) int i32x16;

// -------------------------------------------------------- activations ----
// gelu(v) = max(v, 0) - |v| Phi(-|v|), with Phi(-a) = exp2(P(a)): log2 Phi(-a)
// is close to a parabola, so a short polynomial (fitted here, minimax in the
// relative error of Phi) replaces the rational form and its reciprocal, and a
// negative leading coefficient lets it run on to 0 beyond the fitted range.
// Stored as bf16: degree 5 on [0, 5], relative error 1.6e-4 there, a twelfth of
// half a bf16 step.  Stored as float32: degree 12 on [0, 9], absolute error
// 2.4e-7.  NaN stays NaN; |v| beyond 16 is cut for the product with Phi = 0.
template <bool kF32>
SC_DEV float gelu_exp2(float v) {
  const float a = __builtin_elementwise_minimum(fabsf(v), 16.f);  // without the quieting that fminf needs
  float p;
  if constexpr (kF32) {
    p = -4.266044115186496e-11f;
    p = fmaf(p, a, 2.5370372469524227e-09f);
    p = fmaf(p, a, -6.685024089847502e-08f);
    p = fmaf(p, a, 1.0232761269435287e-06f);
    p = fmaf(p, a, -9.952474101737607e-06f);
    p = fmaf(p, a, 6.172758003231138e-05f);
    p = fmaf(p, a, -0.00020646034681703895f);
    p = fmaf(p, a, -0.00019499764312058687f);
    p = fmaf(p, a, 0.007243024185299873f);
    p = fmaf(p, a, -0.05268990248441696f);
    p = fmaf(p, a, -0.45911744236946106f);
    p = fmaf(p, a, -1.1511205434799194f);
    p = fmaf(p, a, -0.9999995827674866f);
  } else {
    p = -0.0002699175092857331f;
    p = fmaf(p, a, 0.005297347437590361f);
    p = fmaf(p, a, -0.046319346874952316f);
    p = fmaf(p, a, -0.46690741181373596f);
    p = fmaf(p, a, -1.1477890014648438f);
    p = fmaf(p, a, -1.0002282857894897f);
  }
  return fmaf(-a, fast_exp2(p), vmax(v, 0.f));
}

template <bool kF32, bool kGelu>
SC_DEV float finish(int acc, float sx, float sw, float bias) {
  const float v = fmaf((float)acc * sx, sw, bias);
  return kGelu ? gelu_exp2<kF32>(v) : v;
}

SC_DEV void store_out(float* p, float v) { *p = v; }
SC_DEV void store_out(__bf16* p, float v) { *p = (__bf16)v; }

// ------------------------------------------------------- quantisation ----
// A row as a buffer of its K elements: loads beyond it give zeros, without a
// branch; a row that is not live has no elements.
template <typename T>
SC_DEV __amdgpu_buffer_rsrc_t row_buffer(const T* row, int K, bool live) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(row), 0, live ? K * (int)sizeof(T) : 0, 0x00027000);
}

typedef __attribute__((ext_vector_type(4))) unsigned u32x4;

// Eight elements from column c on; zeros at and beyond K.  kVec: K is a multiple of
// 8 and the row 16-byte aligned.
template <typename T, bool kVec>
struct Unit8 {
  static constexpr int kWords = (int)sizeof(T) * 2;
  unsigned w[kVec || sizeof(T) == 4 ? kWords : 8];
  SC_DEV void load(__amdgpu_buffer_rsrc_t row, int c) {
    if constexpr (kVec) {
#pragma unroll
      for (int i = 0; i < kWords / 4; ++i) {
        const u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(row, c * (int)sizeof(T) + 16 * i, 0, 0);
#pragma unroll
        for (int q = 0; q < 4; ++q) w[4 * i + q] = v[q];
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if constexpr (sizeof(T) == 4)
          w[i] = __builtin_amdgcn_raw_buffer_load_b32(row, (c + i) * 4, 0, 0);
        else
          w[i] = __builtin_amdgcn_raw_buffer_load_b16(row, (c + i) * 2, 0, 0);
      }
    }
  }
  SC_DEV float at(int i) const {
    unsigned u;
    if constexpr (sizeof(T) == 4)
      u = w[i];
    else if constexpr (kVec)
      u = i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16;
    else
      u = w[i] << 16;
    return __builtin_bit_cast(float, u);
  }
  SC_DEV float amax() const {
    float a = fabsf(at(0));
#pragma unroll
    for (int i = 1; i < 8; ++i) a = vmax(a, fabsf(at(i)));
    return a;
  }
  SC_DEV uint2 quant(const RowQuant& r) const {
    unsigned q[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = quant_one<T>(r, at(i));
    return make_uint2(pack_i8(q[0], q[1], q[2], q[3]) & r.live, pack_i8(q[4], q[5], q[6], q[7]) & r.live);
  }
};

// One row of K elements held by a wavefront: kUnits units of eight a lane (K <= 512
// kUnits), quantised into Kp bytes by dst(column, bytes).
template <typename T, bool kVec, int kUnits>
struct RowHeld {
  Unit8<T, kVec> u[kUnits];
  SC_DEV void load(__amdgpu_buffer_rsrc_t row, int lane) {
#pragma unroll
    for (int i = 0; i < kUnits; ++i) u[i].load(row, 8 * (lane + 64 * i));
  }
  template <typename Dst>
  SC_DEV float quant(int Kp, Dst dst, int lane) const {
    float a = 0.f;
#pragma unroll
    for (int i = 0; i < kUnits; ++i) a = vmax(a, u[i].amax());
    const RowQuant r = row_quant(butterfly_max(a));
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
      const int c = 8 * (lane + 64 * i);
      if (c < Kp) dst(c, u[i].quant(r));
    }
    return r.scale;
  }
};
// The same for longer rows, read twice.
template <typename T, bool kVec, typename Dst>
SC_DEV float quant_long(__amdgpu_buffer_rsrc_t row, int Kp, Dst dst, int lane) {
  float a = 0.f;
#pragma unroll 2
  for (int c = 8 * lane; c < Kp; c += 512) {
    Unit8<T, kVec> u;
    u.load(row, c);
    a = vmax(a, u.amax());
  }
  const RowQuant r = row_quant(butterfly_max(a));
#pragma unroll 2
  for (int c = 8 * lane; c < Kp; c += 512) {
    Unit8<T, kVec> u;
    u.load(row, c);
    dst(c, u.quant(r));
  }
  return r.scale;
}

// Rows dealt round-robin over the launch's waves.  packed: row p of the output
// is the p-th surviving row (pack_seq), read through xidx; else rows keep their
// places and padding rows become zeros.  The next row's loads are in flight while
// a row is quantised.
template <typename T, bool kVec, int kUnits>
__global__ __launch_bounds__(256) void k_quant_rows(const T* __restrict__ x, int8_t* __restrict__ xq,
                                                    float* __restrict__ scale, int B, int n, int K, int Kp,
                                                    const int* __restrict__ len, const int* __restrict__ xidx,
                                                    int packed) {
  extern __shared__ int pre[];
  const int lane = threadIdx.x & 63;
  unsigned rows = (unsigned)B * (unsigned)n;
  if (packed && len) {
    pack_prefix(pre, len, B, n);
    __syncthreads();
    rows = __builtin_amdgcn_readfirstlane(pre[B]);
  }
  const unsigned step = gridDim.x * 4;
  auto buffer = [&](unsigned p) {
    long long from = p;
    bool live = p < rows;
    if (live && packed) {
      if (len) {
        const int b = __builtin_amdgcn_readfirstlane(pack_seq(pre, B, (int)p));
        from = (long long)b * n + ((int)p - __builtin_amdgcn_readfirstlane(pre[b]));
      }
      if (xidx) from = from / n * n + clampi(scalar_load(xidx, from), 0, n - 1);
    } else if (live && len) {
      const unsigned b = p / (unsigned)n;
      live = (int)(p - b * n) < clampi(scalar_load(len, b), 0, n);
    }
    return row_buffer(x + from * K, K, live);
  };
  unsigned p = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (p >= rows) return;
  if constexpr (kUnits > 0) {
    RowHeld<T, kVec, kUnits> next;
    next.load(buffer(p), lane);
    for (; p < rows; p += step) {
      const RowHeld<T, kVec, kUnits> row = next;
      next.load(buffer(p + step), lane);
      int8_t* d = xq + (long long)p * Kp;
      const float s = row.quant(Kp, [&](int c, uint2 v) { *reinterpret_cast<uint2*>(d + c) = v; }, lane);
      if (lane == 0) scale[p] = s;
    }
  } else {
    for (; p < rows; p += step) {
      int8_t* d = xq + (long long)p * Kp;
      const float s = quant_long<T, kVec>(buffer(p), Kp, [&](int c, uint2 v) { *reinterpret_cast<uint2*>(d + c) = v; },
                                          lane);
      if (lane == 0) scale[p] = s;
    }
  }
}

// 64 output channels a workgroup: the channels' maxima over K (four waves, a
// quarter of the rows each), then 64 x 64 tiles quantised and transposed in LDS.
template <typename T>
__global__ __launch_bounds__(256) void k_quant_weight(const T* __restrict__ w, int8_t* __restrict__ wq,
                                                      float* __restrict__ scale, int K, int N, int Kp) {
  __shared__ float smax[4][64];
  __shared__ __attribute__((aligned(16))) unsigned char tile[64][80];
  const int col = threadIdx.x & 63, wv = threadIdx.x >> 6, n = blockIdx.x * 64 + col;
  float a = 0.f;
  if (n < N)
    for (int k = wv; k < K; k += 4) a = vmax(a, fabsf((float)w[(long long)k * N + n]));
  smax[wv][col] = a;
  __syncthreads();
  const RowQuant r = row_quant(vmax(vmax(smax[0][col], smax[1][col]), vmax(smax[2][col], smax[3][col])));
  if (wv == 0 && n < N) scale[n] = r.scale;
  for (int k0 = 0; k0 < Kp; k0 += 64) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int k = k0 + 16 * wv + i;
      const float v = n < N && k < K ? (float)w[(long long)k * N + n] : 0.f;
      tile[col][16 * wv + i] = (unsigned char)(quant_one<T>(r, v) & r.live);
    }
    __syncthreads();
    const int row = threadIdx.x >> 2, un = threadIdx.x & 3;
    if (blockIdx.x * 64 + row < N)
      *reinterpret_cast<uint4*>(wq + (long long)(blockIdx.x * 64 + row) * Kp + k0 + 16 * un) =
          *reinterpret_cast<const uint4*>(&tile[row][16 * un]);
    __syncthreads();
  }
}

// ------------------------------------------------------------ product ----
struct LinearArgs {
  const int8_t* xq;
  const float* xs;
  const int8_t* wq;
  const float* ws;
  const float* bias;
  void* out;
  int B, n, N, Kp;
  const int* len;
  int packed;    // xq and xs hold the surviving rows alone, in order
  int skip_pad;  // padding rows of out are left as they are
  int vec;       // rows of out are whole 16-byte units
};

constexpr int kBK = 128;        // bytes of a row per K stage: whole lines (64-byte pieces halve the loads' rate)
constexpr int kLinWgs = 256;    // one workgroup per CU, each taking tiles in turn
constexpr int kLinLds = 147456; // stage buffers: 2 x 64, 3 x 48, 4 x 32 or 9 x 16 KB
constexpr int kLinModes = 4;
constexpr int kGroupM = 8;
// k_linear_few: at most kFewRows rows of kFewK bytes, kFewWgs workgroups and
// kFewWork bytes of rows over all of them.  us in a graph, bf16 rows, this kernel and
// the two launches of the others: K 512 N 1536 1 row 3.9 and 6.5, 128 rows 6.0 and
// 7.4, 256 rows 8.6 and 7.5; K 768 N 2304 64 rows 6.6 and 8.3, 128 rows 8.7 and 8.2;
// K 1024 N 4096 64 rows 7.9 and 9.0, 128 rows 12.6 and 9.1; K 4096 N 1024 1 row 9.3
// and 17.1, 128 rows 13.8 and 18.8, 256 rows 23.8 and 19.3.  8-bit rows alike.
constexpr int kFewRows = 512, kFewK = 4096, kFewWgs = 1024, kFewWork = 5 << 19;

// Tile shapes: kKS waves share a part of the tile, each with its part of every stage.
template <int kM>
struct LinTile;
template <>
struct LinTile<0> { static constexpr int kBM = 256, kBN = 256, kWgM = 2, kWgN = 4, kKS = 1; };
template <>
struct LinTile<1> { static constexpr int kBM = 256, kBN = 128, kWgM = 4, kWgN = 2, kKS = 1; };
template <>
struct LinTile<2> { static constexpr int kBM = 128, kBN = 128, kWgM = 4, kWgN = 2, kKS = 1; };
template <>
struct LinTile<3> { static constexpr int kBM = 64, kBN = 64, kWgM = 2, kWgN = 2, kKS = 2; };

struct LinPlan {
  int mode, T, Nt;
};
// The mode with the least rounds of workgroups times the cost of a tile: of a stage
// and of what stands beside the stages, in cycles.
SC_DEV LinPlan lin_plan(int R, int N, int ns) {
  LinPlan p = {0, 0, 0};
  long long best = 1LL << 62;
#pragma unroll
  for (int m = 0; m < kLinModes; ++m) {
    const int bm = m <= 1 ? 256 : m == 2 ? 128 : 64, bn = m == 0 ? 256 : m == 3 ? 64 : 128;
    const int stage = m == 0 ? 2400 : m == 1 ? 1400 : m == 2 ? 800 : 450;
    const int fixed = m == 0 ? 12000 : m == 1 ? 7000 : m == 2 ? 4500 : 3000;
    const int T = (R + bm - 1) / bm, Nt = (N + bn - 1) / bn;
    const long long rounds = ((long long)T * Nt + kLinWgs - 1) / kLinWgs;
    const long long t = rounds * (ns * stage + fixed);
    if (t < best) {
      best = t;
      p.mode = m;
      p.T = T;
      p.Nt = Nt;
    }
  }
  return p;
}

// 128-byte rows in LDS, 16-byte units swizzled by bits 1-3 of the row: the fragment
// reads of 32x32x32 products (lane l: row l % 32, unit l / 32 of a chunk's two) run at
// 225 bytes per clock and CU (swizzled by bits 0-2: 126).
SC_DEV int q_off(int row, int unit) { return row * kBK + 16 * (unit ^ ((row >> 1) & 7)); }

SC_DEV i32x4 lds_read_q(unsigned addr) {
  return *(const __attribute__((address_space(3))) i32x4*)(size_t)addr;
}

// Orders a wavefront's LDS accesses across its lanes: without it the compiler may take
// what a lane read before for what it reads after other lanes' writes.
SC_DEV void wave_exchange() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// The row numbering (sc_pack.h) with a table of fixed size: the prefix sums of every
// `per`-th sequence, the rest by a scan of at most per - 1 lengths.
constexpr int kCoarse = 1024;
struct Packed {
  const int* pre;  // LDS
  const int* len;
  int B, n, per, count;
  SC_DEV int length(int b) const { return clampi(len[b], 0, n); }
  // Wave 0 fills the table; returns nothing, R is pre[count].
  SC_DEV static void fill(int* pre, const int* len, int B, int n, int per, int count) {
    if (threadIdx.x >= 64) return;
    const int lane = threadIdx.x;
    int carry = 0;
    for (int c = 0; c < count; c += 64) {
      int v = 0;
      for (int i = 0; i < per; ++i) {
        const int b = (c + lane) * per + i;
        if (c + lane < count && b < B) v += clampi(len[b], 0, n);
      }
      const int incl = prefix_sum(v);
      if (c + lane < count) pre[c + lane] = carry + incl - v;
      carry += __builtin_amdgcn_readlane(incl, 63);
    }
    if (lane == 0) pre[count] = carry;
  }
  // The row of the batch that holds packed row p.
  SC_DEV int row(int p) const {
    const int c = pack_seq(pre, count, p);
    int b = c * per, first = pre[c];
    for (int i = 1; i < per; ++i) {
      const int l = length(b);
      if (p < first + l) break;
      first += l;
      ++b;
    }
    return b * n + (p - first);
  }
  // The row of the batch that holds padding row q (numbered like the packed ones).
  SC_DEV long long pad_row(long long q) const {
    int lo = 0, hi = count - 1;  // the largest c whose padding rows before it are at most q
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if ((long long)mid * per * n - pre[mid] <= q) lo = mid;
      else hi = mid - 1;
    }
    int b = lo * per;
    long long first = (long long)b * n - pre[lo];
    int l = length(b);
    for (int i = 1; i < per; ++i) {
      if (q < first + (n - l)) break;
      first += n - l;
      l = length(++b);
    }
    return (long long)b * n + l + (q - first);
  }
};

// A tile's rows and columns: in LDS, twice, the next tile's beside this one's.
struct LinTables {
  int grow[256], xrow[256];  // row of out (-1: none) and of xq
  float xs[256], sw[256], sb[256];
};

template <int kM, typename O, bool kGelu>
SC_DEV void linear_run(const LinearArgs& a, char* stage, LinTables* tab, const Packed& pk, int R, const LinPlan& pl) {
  using S = LinTile<kM>;
  constexpr int BM = S::kBM, BN = S::kBN, KS = S::kKS;
  constexpr int WM = BM / S::kWgM, WN = BN / S::kWgN, FI = WM / 32, FJ = WN / 32;
  constexpr int XL = BM / 64, WL = BN / 64, kDma = XL + WL;  // loads of a wave and stage, 8 rows each
  constexpr int kStage = (BM + BN) * kBK, kNBuf = kLinLds / kStage < 8 ? kLinLds / kStage : 8;
  constexpr int CH = 4 / KS;  // a wave's 32-byte chunks of a stage, one product each (even)
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), hi = lane >> 5,
            lr = lane & 31;
  const int wt = w / KS, ks = w % KS;
  const int wm = (wt / S::kWgN) * WM, wn = (wt % S::kWgN) * WN;
  const int ns = a.Kp / kBK;
  const long long items = (long long)pl.T * pl.Nt;
  // The tiles go to the XCDs in contiguous ranges (workgroup i runs on XCD i % 8), in
  // groups of kGroupM row tiles by all column tiles: what an XCD runs at a time shares
  // rows and weights in its L2.
  const int xcd = blockIdx.x & 7;
  const long long last = items * (xcd + 1) / 8;
  long long item = items * xcd / 8 + (blockIdx.x >> 3);
  if (item >= last) return;
  auto place = [&](long long it, int& m0, int& n0) {
    const int per = kGroupM * pl.Nt, gi = (int)(it / per), rem = (int)(it - (long long)gi * per);
    const int gs = min(kGroupM, pl.T - gi * kGroupM);
    m0 = __builtin_amdgcn_readfirstlane((gi * kGroupM + rem % gs) * BM);
    n0 = __builtin_amdgcn_readfirstlane(rem / gs * BN);
  };
  // What thread tid brings into a tile's tables: row m0 + tid, column n0 + tid.
  int b_gr = -1, b_xr = 0;
  float b_xs = 0.f, b_sw = 0.f, b_sb = 0.f;
  auto bring = [&](int m0, int n0) {
    if (tid < BM) {
      const int p = min(m0 + tid, R - 1);  // rows past the last one read it again
      const int gr = a.len ? pk.row(p) : p;
      b_gr = m0 + tid < R ? gr : -1;
      b_xr = a.packed ? p : gr;
      b_xs = a.xs[b_xr];
    }
    if (tid < BN) {
      const int c = min(n0 + tid, a.N - 1);
      b_sw = a.ws[c];
      b_sb = a.bias ? a.bias[c] : 0.f;
    }
  };
  auto put = [&](LinTables& d) {
    if (tid < BM) {
      d.grow[tid] = b_gr;
      d.xrow[tid] = b_xr;
      d.xs[tid] = b_xs;
    }
    if (tid < BN) {
      d.sw[tid] = b_sw;
      d.sb[tid] = b_sb;
    }
  };
  unsigned xoff[XL], woff[WL];
  auto offsets = [&](const LinTables& d, int n0) {
#pragma unroll
    for (int t = 0; t < XL; ++t) {
      const int R0 = (BM / 8) * w + 8 * t, swz = ((lane >> 4) & 3) | ((R0 >> 1) & 4);
      xoff[t] = (unsigned)d.xrow[R0 + (lane >> 3)] * (unsigned)a.Kp + 16u * ((lane & 7) ^ swz);
    }
#pragma unroll
    for (int t = 0; t < WL; ++t) {
      const int R0 = (BN / 8) * w + 8 * t, swz = ((lane >> 4) & 3) | ((R0 >> 1) & 4);
      woff[t] = (unsigned)min(n0 + R0 + (lane >> 3), a.N - 1) * (unsigned)a.Kp + 16u * ((lane & 7) ^ swz);
    }
  };
  const unsigned lds0 = lds_addr(stage);
  auto issue = [&](int s, int bf) {
    const int8_t *xb = a.xq + (size_t)s * kBK, *wb = a.wq + (size_t)s * kBK;
    const unsigned lx = lds0 + (unsigned)bf * kStage, lw = lx + BM * kBK;
#pragma unroll
    for (int t = 0; t < XL; ++t) lds_dma16(xb, xoff[t], lx + ((BM / 8) * w + 8 * t) * kBK);
#pragma unroll
    for (int t = 0; t < WL; ++t) lds_dma16(wb, woff[t], lw + ((BN / 8) * w + 8 * t) * kBK);
  };
  const unsigned xa = lds0 + q_off(wm + lr, hi), wa = lds0 + BM * kBK + q_off(wn + lr, hi);
  i32x16 acc[FI][FJ];
  i32x4 xf[2][FI], wf[2][FJ];  // two chunks' fragments
  auto frags = [&](int p, int bf, int c) {
    const unsigned o = (unsigned)bf * kStage, x = 32u * (c + ks * CH);
#pragma unroll
    for (int j = 0; j < FJ; ++j) wf[p][j] = lds_read_q((wa ^ x) + o + j * (32 * kBK));
#pragma unroll
    for (int i = 0; i < FI; ++i) xf[p][i] = lds_read_q((xa ^ x) + o + i * (32 * kBK));
  };
  auto mul = [&](int p) {
#pragma unroll
    for (int i = 0; i < FI; ++i)
#pragma unroll
      for (int j = 0; j < FJ; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(wf[p][j], xf[p][i], acc[i][j], 0, 0, 0);
  };
  auto next_buf = [&](int bf) { return bf == kNBuf - 1 ? 0 : bf + 1; };
  constexpr int kAhead = kNBuf - 1;  // stages of the next tile loaded beside the results, which leave through the last buffer
  int m0, n0, cur = 0;
  place(item, m0, n0);
  bring(m0, n0);
  put(tab[0]);
  __syncthreads();
  offsets(tab[0], n0);
#pragma unroll
  for (int p = 0; p < kAhead; ++p)
    if (p < ns) issue(p, p);
  while (true) {
#pragma unroll
    for (int i = 0; i < FI; ++i)
#pragma unroll
      for (int j = 0; j < FJ; ++j) acc[i][j] = i32x16{};
    if (kAhead < ns) issue(kAhead, kAhead);
    const long long nitem = item + (gridDim.x >> 3);
    const bool more = nitem < last;
    int nm0 = 0, nn0 = 0;
    if (more) place(nitem, nm0, nn0);
    wait_stages<kNBuf, kDma>(min(ns, kNBuf) - 1);
    __syncthreads();
    int bf = 0;
    frags(0, 0, 0);
    // One barrier per stage, before its last product: a chunk's fragments are in flight
    // during the products of the one before, across stages too, and a stage's buffer is
    // refilled once every wave holds its last fragments.
    for (int s = 0; s + 1 < ns; ++s) {
      const int bn = next_buf(bf);
#pragma unroll
      for (int c = 0; c + 1 < CH; ++c) {
        frags((c + 1) & 1, bf, c + 1);
        mul(c & 1);
      }
      wait_stages<kNBuf - 1, kDma>(min(ns - 2 - s, kNBuf - 2));
      __syncthreads();
      if (s + kNBuf < ns) issue(s + kNBuf, bf);
      frags(0, bn, 0);
      mul(1);
      bf = bn;
    }
#pragma unroll
    for (int c = 0; c + 1 < CH; ++c) {
      frags((c + 1) & 1, bf, c + 1);
      if (c == 0 && more) bring(nm0, nn0);
      mul(c & 1);
    }
    mul(1);
    __syncthreads();  // every wave has read the last stage
    const int on0 = n0;
    const LinTables& d = tab[cur];
    if (more) {
      put(tab[cur ^ 1]);
      __syncthreads();
      n0 = nn0;
      offsets(tab[cur ^ 1], n0);
#pragma unroll
      for (int p = 0; p < kAhead; ++p)
        if (p < ns) issue(p, p);
    }
    // Element e of a lane's acc[i][j] is row wm + 32 i + lr, column wn + 32 j + 8 (e / 4)
    // + 4 hi + e % 4.  A wave's part goes through the last stage buffer, kSr rows at a
    // time (16-byte units swizzled by the row), and leaves as whole 16-byte units.
    constexpr int es = sizeof(O), kUr = WN * es / 16, kRb = WN * es, kEpu = 16 / es;
    constexpr int kParts = 8 / KS, kSr = kParts * 32 * kRb <= kStage ? 32 : 16;
    static_assert(kParts * kSr * kRb <= kStage && (KS == 1 || kParts * 4096 * FI * FJ <= kStage), "staging rows");
    char* st = stage + kAhead * kStage + wt * (kSr * kRb);
    if constexpr (KS == 2) {  // the second half's sums through the same buffer
      int* red = reinterpret_cast<int*>(stage + kAhead * kStage) + wt * 1024 * FI * FJ;
      if (ks == 1) {
#pragma unroll
        for (int i = 0; i < FI; ++i)
#pragma unroll
          for (int j = 0; j < FJ; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) red[((i * FJ + j) * 16 + e) * 64 + lane] = acc[i][j][e];
      }
      __syncthreads();
      if (ks == 0) {
#pragma unroll
        for (int i = 0; i < FI; ++i)
#pragma unroll
          for (int j = 0; j < FJ; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] += red[((i * FJ + j) * 16 + e) * 64 + lane];
      }
      __syncthreads();
    }
    if (ks == 0) {
#pragma unroll
      for (int i = 0; i < FI; ++i) {
        const float xs = d.xs[wm + 32 * i + lr];
#pragma unroll
        for (int r0 = 0; r0 < 32; r0 += kSr) {
          if (kSr == 32 || (lr >= r0 && lr < r0 + kSr)) {
#pragma unroll
            for (int j = 0; j < FJ; ++j)
#pragma unroll
              for (int q = 0; q < 4; ++q) {
                const int c = 32 * j + 8 * q + 4 * hi;
                const f32x4 ws = *reinterpret_cast<const f32x4*>(d.sw + wn + c);
                const f32x4 bs = *reinterpret_cast<const f32x4*>(d.sb + wn + c);
                f32x4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = finish<es == 4, kGelu>(acc[i][j][4 * q + e], xs, ws[e], bs[e]);
                const int r = lr - r0, un = c * es / 16;
                char* o = st + r * kRb + 16 * (un ^ (r & (kUr - 1)));
                if constexpr (es == 4)
                  *reinterpret_cast<uint4*>(o) = __builtin_bit_cast(uint4, v);
                else
                  *reinterpret_cast<uint2*>(o + 8 * hi) = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
              }
          }
          wave_exchange();
#pragma unroll
          for (int x = 0; x < kSr * kUr / 64; ++x) {
            const int r = x * (64 / kUr) + lane / kUr, un = lane % kUr, gr = d.grow[wm + 32 * i + r0 + r];
            const int col = on0 + wn + un * kEpu;
            const uint4 v = *reinterpret_cast<const uint4*>(st + r * kRb + 16 * (un ^ (r & (kUr - 1))));
            if (gr < 0 || col >= a.N) continue;
            O* o = static_cast<O*>(a.out) + (long long)gr * a.N + col;
            if (a.vec) {
              *reinterpret_cast<uint4*>(o) = v;
            } else {
              const O* e = reinterpret_cast<const O*>(&v);
#pragma unroll
              for (int q = 0; q < kEpu; ++q)
                if (col + q < a.N) o[q] = e[q];
            }
          }
          wave_exchange();
        }
      }
    }
    if (!more) break;
    item = nitem;
    cur ^= 1;
    __syncthreads();  // the results have left the last stage buffer
  }
}

template <typename O, bool kGelu>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2))) void k_linear(LinearArgs a) {
  __shared__ __attribute__((aligned(1024))) char stage[kLinLds];
  __shared__ __attribute__((aligned(16))) LinTables tab[2];
  __shared__ int pre[kCoarse + 1];
  const int per = (a.B + kCoarse - 1) / kCoarse, count = (a.B + per - 1) / per;
  const Packed pk{pre, a.len, a.B, a.n, per, count};
  int R = a.B * a.n;
  if (a.len) {
    Packed::fill(pre, a.len, a.B, a.n, per, count);
    __syncthreads();
    R = __builtin_amdgcn_readfirstlane(pre[count]);
  }
  if (R > 0) {
    const LinPlan pl = lin_plan(R, a.N, a.Kp / kBK);
    if (pl.mode == 0)
      linear_run<0, O, kGelu>(a, stage, tab, pk, R, pl);
    else if (pl.mode == 1)
      linear_run<1, O, kGelu>(a, stage, tab, pk, R, pl);
    else if (pl.mode == 2)
      linear_run<2, O, kGelu>(a, stage, tab, pk, R, pl);
    else
      linear_run<3, O, kGelu>(a, stage, tab, pk, R, pl);
  }
  if (!a.len || a.skip_pad) return;
  // zeros into the padding rows, an even share a workgroup
  const long long P = (long long)a.B * a.n - R;
  const long long lo = P * blockIdx.x / gridDim.x, end = P * (blockIdx.x + 1) / gridDim.x;
  const int lane = threadIdx.x & 63;
  for (long long q = lo + (threadIdx.x >> 6); q < end; q += 8) {
    O* o = static_cast<O*>(a.out) + pk.pad_row(q) * a.N;
    if (a.vec) {
      for (int c = lane; c < a.N / (16 / (int)sizeof(O)); c += 64)
        reinterpret_cast<uint4*>(o)[c] = make_uint4(0, 0, 0, 0);
    } else {
      for (int c = lane; c < a.N; c += 64) o[c] = (O)0.f;
    }
  }
}

template <typename O, bool kGelu>
hipError_t run_linear(const LinearArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((k_linear<O, kGelu>), dim3(kLinWgs), dim3(512), 0, s, a);
  return hipGetLastError();
}

template <typename T, bool kVec>
hipError_t run_quant(const void* x, int8_t* xq, float* scale, int B, int n, int K, int Kp, const int* len,
                     const int* xidx, int packed, hipStream_t s) {
  const long long rows = (long long)B * n;
  const dim3 grid((unsigned)std::min<long long>((rows + 3) / 4, 4096));
  const size_t lds = packed && len ? sizeof(int) * (B + 1) : 0;
  const T* xt = static_cast<const T*>(x);
  if (Kp <= 1024)
    hipLaunchKernelGGL((k_quant_rows<T, kVec, 2>), grid, dim3(256), lds, s, xt, xq, scale, B, n, K, Kp, len, xidx,
                       packed);
  else if (Kp <= 4096)
    hipLaunchKernelGGL((k_quant_rows<T, kVec, 8>), grid, dim3(256), lds, s, xt, xq, scale, B, n, K, Kp, len, xidx,
                       packed);
  else
    hipLaunchKernelGGL((k_quant_rows<T, kVec, 0>), grid, dim3(256), lds, s, xt, xq, scale, B, n, K, Kp, len, xidx,
                       packed);
  return hipGetLastError();
}

// ----------------------------------------------------------- few rows ----
// A call of few rows is a chain of latencies: here it is one launch.  A workgroup
// takes 16 rows and 16 output channels, its four waves a quarter of K each: a wave
// starts its weights' loads (straight into the fragments' registers: each weight
// byte is used once), quantises four of the rows into LDS while they arrive, and
// multiplies; the quarters are added in LDS.  Every workgroup quantises its rows
// for itself: 16 x K elements from the L2 against a launch of its own.
template <typename T, bool kVec, int kUnits, typename O, bool kGelu>
__global__ __launch_bounds__(256) void k_linear_few(LinearArgs a, const T* __restrict__ x, int K) {
  constexpr int kMaxK = 512 * kUnits, kChunks = kMaxK / 256;  // 64-byte chunks of a wave
  constexpr bool kI8 = sizeof(T) == 1;
  __shared__ __attribute__((aligned(16))) int8_t sx[16 * (kMaxK + 16)];
  __shared__ int red[4][256];
  __shared__ float ss[16];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4,
            lr = lane & 15;
  const int n0 = blockIdx.x * 16, rows = a.B * a.n, Kp = a.Kp, pitch = Kp + 16, nc = Kp / 64;
  const long long m0 = (long long)blockIdx.y * 16;
  auto live = [&](long long m) {
    if (m >= rows) return false;
    if (!a.len) return true;
    const unsigned b = (unsigned)m / (unsigned)a.n;
    return (int)((unsigned)m - b * a.n) < clampi(scalar_load(a.len, b), 0, a.n);
  };
  const int8_t* wp = a.wq + (size_t)min(n0 + lr, a.N - 1) * Kp + 16 * g;
  i32x4 wf[kChunks];
#pragma unroll
  for (int i = 0; i < kChunks; ++i) {
    const int c = min(w + 4 * i, nc - 1);  // past the last: read again, not used
    wf[i] = *reinterpret_cast<const i32x4*>(wp + c * 64);
  }
  if constexpr (kI8) {
    for (int r = 4 * w; r < 4 * w + 4; ++r) {
      const bool on = live(m0 + r);
      const auto buf = row_buffer(x + (m0 + r) * Kp, Kp, on);
#pragma unroll
      for (int i = 0; i < (kMaxK + 1023) / 1024; ++i) {
        const int c = 16 * (lane + 64 * i);
        if (c < Kp)
          *reinterpret_cast<u32x4*>(sx + r * pitch + c) = __builtin_amdgcn_raw_buffer_load_b128(buf, c, 0, 0);
      }
      if (lane == 0) ss[r] = on ? a.xs[m0 + r] : 0.f;
    }
  } else {
    constexpr int kAtOnce = kUnits == 2 || (kVec && sizeof(T) == 2) ? 4 : 2;  // rows held at once, as registers allow
#pragma unroll
    for (int r0 = 0; r0 < 4; r0 += kAtOnce) {
      RowHeld<T, kVec, kUnits> h[kAtOnce];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const long long m = m0 + 4 * w + r0 + i;
        h[i].load(row_buffer(x + m * K, K, live(m)), lane);
      }
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        int8_t* d = sx + (4 * w + r0 + i) * pitch;
        const float s = h[i].quant(Kp, [&](int c, uint2 v) { *reinterpret_cast<uint2*>(d + c) = v; }, lane);
        if (lane == 0) ss[4 * w + r0 + i] = s;
      }
    }
  }
  __syncthreads();
  i32x4 acc = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < kChunks; ++i) {
    const int c = w + 4 * i;
    if (c < nc)
      acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(*reinterpret_cast<const i32x4*>(sx + lr * pitch + c * 64 + 16 * g), wf[i],
                                                  acc, 0, 0, 0);
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) red[w][(4 * g + e) * 16 + lr] = acc[e];
  __syncthreads();
  const int r = tid >> 4, col = n0 + (tid & 15);
  const long long m = m0 + r;
  if (m >= rows || col >= a.N) return;
  const int sum = red[0][tid] + red[1][tid] + red[2][tid] + red[3][tid];
  const bool on = live(m);
  if (!on && a.skip_pad) return;
  const float v = on ? finish<sizeof(O) == 4, kGelu>(sum, ss[r], a.ws[col], a.bias ? a.bias[col] : 0.f) : 0.f;
  store_out(static_cast<O*>(a.out) + m * a.N + col, v);
}

}  // namespace

hipError_t launch_quant_rows(const void* x, int f32, int8_t* xq, float* scale, int B, int n, int K, const int* len,
                             const int* xidx, int packed, hipStream_t s) {
  const int Kp = i8_pitch(K);
  const bool vec = K % 8 == 0 && reinterpret_cast<uintptr_t>(x) % 16 == 0;
  if (f32)
    return vec ? run_quant<float, true>(x, xq, scale, B, n, K, Kp, len, xidx, packed, s)
               : run_quant<float, false>(x, xq, scale, B, n, K, Kp, len, xidx, packed, s);
  return vec ? run_quant<__bf16, true>(x, xq, scale, B, n, K, Kp, len, xidx, packed, s)
             : run_quant<__bf16, false>(x, xq, scale, B, n, K, Kp, len, xidx, packed, s);
}

hipError_t launch_quant_weight(const void* w, int f32, int8_t* wq, float* scale, int K, int N, hipStream_t s) {
  const dim3 grid((N + 63) / 64);
  if (f32)
    hipLaunchKernelGGL(k_quant_weight<float>, grid, dim3(256), 0, s, static_cast<const float*>(w), wq, scale, K, N,
                       i8_pitch(K));
  else
    hipLaunchKernelGGL(k_quant_weight<__bf16>, grid, dim3(256), 0, s, static_cast<const __bf16*>(w), wq, scale, K, N,
                       i8_pitch(K));
  return hipGetLastError();
}

namespace {
LinearArgs linear_args(const Linear& l) {
  LinearArgs a;
  a.xq = l.xq;
  a.xs = l.xs;
  a.wq = l.wq;
  a.ws = l.w_scale;
  a.bias = l.bias;
  a.out = l.out;
  a.B = l.B;
  a.n = l.n;
  a.N = l.N;
  a.Kp = i8_pitch(l.K);
  a.len = l.len;
  a.packed = l.packed;
  a.skip_pad = l.skip_pad;
  const size_t es = l.out_f32 ? 4 : 2;
  a.vec = (size_t)l.N * es % 16 == 0 && reinterpret_cast<uintptr_t>(l.out) % 16 == 0;
  return a;
}

template <typename T, bool kVec, int kUnits>
hipError_t run_few(const Linear& l, const void* x, hipStream_t s) {
  const LinearArgs a = linear_args(l);
  const dim3 grid((l.N + 15) / 16, (unsigned)(((long long)l.B * l.n + 15) / 16));
  const T* xt = static_cast<const T*>(x);
  if (l.out_f32) {
    if (l.gelu)
      hipLaunchKernelGGL((k_linear_few<T, kVec, kUnits, float, true>), grid, dim3(256), 0, s, a, xt, l.K);
    else
      hipLaunchKernelGGL((k_linear_few<T, kVec, kUnits, float, false>), grid, dim3(256), 0, s, a, xt, l.K);
  } else if (l.gelu) {
    hipLaunchKernelGGL((k_linear_few<T, kVec, kUnits, __bf16, true>), grid, dim3(256), 0, s, a, xt, l.K);
  } else {
    hipLaunchKernelGGL((k_linear_few<T, kVec, kUnits, __bf16, false>), grid, dim3(256), 0, s, a, xt, l.K);
  }
  return hipGetLastError();
}
template <typename T, bool kVec>
hipError_t run_few(const Linear& l, const void* x, hipStream_t s) {
  return i8_pitch(l.K) <= 1024 ? run_few<T, kVec, 2>(l, x, s) : run_few<T, kVec, 8>(l, x, s);
}
}  // namespace

bool linear_few_ok(long long rows, int K, int N) {
  if (rows > kFewRows || i8_pitch(K) > kFewK) return false;
  const long long wgs = (rows + 15) / 16 * ((N + 15) / 16);
  return wgs <= kFewWgs && wgs * i8_pitch(K) <= kFewWork;
}

hipError_t launch_linear_few(const Linear& l, const void* x, int x_type, hipStream_t s) {
  const bool vec = l.K % 8 == 0 && reinterpret_cast<uintptr_t>(x) % 16 == 0;
  if (x_type == 2) return run_few<int8_t, true>(l, x, s);
  if (x_type == 0) return vec ? run_few<float, true>(l, x, s) : run_few<float, false>(l, x, s);
  return vec ? run_few<__bf16, true>(l, x, s) : run_few<__bf16, false>(l, x, s);
}

hipError_t launch_linear_i8(const Linear& l, hipStream_t s) {
  const LinearArgs a = linear_args(l);
  if (l.out_f32) return l.gelu ? run_linear<float, true>(a, s) : run_linear<float, false>(a, s);
  return l.gelu ? run_linear<__bf16, true>(a, s) : run_linear<__bf16, false>(a, s);
}

}  // namespace sc
