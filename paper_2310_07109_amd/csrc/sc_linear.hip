// Matrix products in 8-bit integers with a scale for each token and channel.
//
//   out[t, n] = act(s_t w_n sum_k q[t, k] wq[n, k] + bias[n])
//
// k_quant_rows    the tokens' 8-bit rows (sc_quant.h), one wavefront a row.
// k_quant_weight  the weights', once per model.
// k_linear        the product on v_mfma_i32_16x16x64_i8: sums of up to 131072
//                 products of 127 x 127 fit an int32, so they are exact in any
//                 order, and a row's result does not depend on the tile that
//                 computed it.  (With random operands the 16x16x64 form sustains
//                 4.0 POP/s here, 32x32x32 3.5: the clock follows the power; with
//                 zeros 4.8 and 4.9.)
// k_linear_few    the same for a few rows: quantisation and product in one launch.
//
// 32768 x 4096 x 1024 on 8-bit rows: 116 us, 2.4 POP/s (a library's 8192^3: 2.0), at
// 1.8 GHz under load, the matrix units busy 0.62 of the cycles.  32768 x 1024 x 4096:
// 20-27 us of quantising (HBM rate) and 152, with GELU 188-202, 0.33 of the cycles: a tile
// has few stages there, and the arithmetic on its results (21 instructions each, an
// exponential among them) and 268 MB of stores stand beside them.
#include <algorithm>

#include "sc_device.h"
#include "sc_internal.h"
#include "sc_pack.h"
#include "sc_quant.h"

namespace sc {
namespace {

typedef __attribute__((ext_vector_type(4))) int i32x4;

// -------------------------------------------------------- activations ----
// gelu(v) = max(v, 0) - |v| Phi(-|v|), with Phi(-a) = exp2(P(a)): log2 Phi(-a)
// is close to a parabola, so a polynomial (fitted here on [0, 9], minimax in the
// relative error of Phi) replaces the rational form and its reciprocal, and a
// negative leading coefficient lets it run on to 0 beyond the fitted range.
// Absolute error 2.4e-7; of a negative value 1e-6 relative down to -3, 2.5e-6 to
// -5, 3e-5 to -9, where it is 1e-18.  One form for both output types: what is
// stored as bf16 is the float32 value rounded once (degree 5 has 1.6e-4 relative and
// 1 % beyond -5, 14 instructions a result instead of 21 and 182 us instead of 202 for
// 32768 x 1024 x 4096).  NaN stays NaN; |v| beyond 16 is cut for the product with Phi = 0.
SC_DEV float gelu_exp2(float v) {
  const float a = __builtin_elementwise_minimum(fabsf(v), 16.f);  // without the quieting that fminf needs
  float p = -4.266044115186496e-11f;
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
  return fmaf(-a, fast_exp2(p), vmax(v, 0.f));
}

template <bool kGelu>
SC_DEV float finish(int acc, float sx, float sw, float bias) {
  const float v = fmaf((float)acc * sx, sw, bias);
  return kGelu ? gelu_exp2(v) : v;
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
// Global accesses of 16 and 8 bytes at any element's address (rows of odd length).
typedef u32x4 __attribute__((aligned(2))) u32x4_any;
typedef __attribute__((ext_vector_type(2), aligned(2))) unsigned u32x2_any;

// Zeros into n bytes at p (a multiple of 2), by one wavefront.
SC_DEV void zero_bytes(char* p, long long n, int lane) {
  for (long long c = 16 * lane; c < n; c += 1024) {
    if (c + 16 <= n) {
      *reinterpret_cast<u32x4_any*>(p + c) = u32x4_any{0, 0, 0, 0};
    } else {
      for (long long i = c; i < n; i += 2) *reinterpret_cast<unsigned short*>(p + i) = 0;
    }
  }
}

// Eight elements from column c on; zeros at and beyond K.  kVec: rows start at dwords
// (the hardware checks every dword of an access against the buffer's end).
template <typename T, bool kVec>
struct Unit8 {
  static constexpr int kWords = (int)sizeof(T) * 2;
  unsigned w[kVec ? kWords : 8];
  SC_DEV void load(__amdgpu_buffer_rsrc_t row, int c) {
    if constexpr (kVec) {
#pragma unroll
      for (int i = 0; i < kWords / 4; ++i) {
        const u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(row, c * (int)sizeof(T) + 16 * i, 0, 0);
#pragma unroll
        for (int q = 0; q < 4; ++q) w[4 * i + q] = v[q];
      }
    } else {
      static_assert(sizeof(T) == 2, "dwords are aligned");
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = __builtin_amdgcn_raw_buffer_load_b16(row, (c + i) * 2, 0, 0);
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

// Rows of a product's output that are padding: zeroed by the launch that quantises its
// input, beside its reads.
struct ZeroRows {
  char* out;        // or null
  long long bytes;  // of a row
  SC_DEV void fill(unsigned row, int lane) const { zero_bytes(out + row * bytes, bytes, lane); }
};

// Rows dealt round-robin over the launch's waves; the next row's loads are in flight
// while a row is quantised.  Row j of sequence b goes to row b n + j, from row xidx[b,
// j] of the sequence when given.  zero_pad: padding rows become zeros (else they are
// left as they are).
template <typename T, bool kVec, int kUnits>
__global__ __launch_bounds__(256) void k_quant_rows(const T* __restrict__ x, int8_t* __restrict__ xq,
                                                    float* __restrict__ scale, int B, int n, int K, int Kp,
                                                    const int* __restrict__ len, const int* __restrict__ xidx,
                                                    int zero_pad, ZeroRows zero) {
  const int lane = threadIdx.x & 63;
  const unsigned rows = (unsigned)B * (unsigned)n, step = gridDim.x * 4;
  // Round k takes place (i + k turn) mod step, as k_norm does.
  const unsigned turn = (unsigned)(0.382f * (float)step);
  struct Row {
    unsigned p;
    bool exists, live;
    __amdgpu_buffer_rsrc_t buf;
  };
  auto at = [&](unsigned p) {
    Row r;
    r.p = p;
    r.exists = r.live = p < rows;
    long long from = p;
    if (r.live && (len || xidx)) {
      const unsigned b = p / (unsigned)n;
      if (len) r.live = (int)(p - b * n) < clampi(scalar_load(len, b), 0, n);
      if (xidx && r.live) from = (long long)b * n + clampi(scalar_load(xidx, p), 0, n - 1);
    }
    r.buf = row_buffer(x + from * K, K, r.live);
    return r;
  };
  unsigned place = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), round = 0;
  auto advance = [&]() {
    round += step;
    place = place + turn < step ? place + turn : place + turn - step;
  };
  Row cur = at(place);
  if constexpr (kUnits > 0) {
    RowHeld<T, kVec, kUnits> next;
    next.load(cur.buf, lane);
    while (round < rows) {
      advance();
      const RowHeld<T, kVec, kUnits> row = next;
      const Row nrow = at(round + place);
      next.load(nrow.buf, lane);
      if (cur.exists && (cur.live || zero_pad)) {
        int8_t* d = xq + (long long)cur.p * Kp;
        const float s = row.quant(Kp, [&](int c, uint2 v) { *reinterpret_cast<uint2*>(d + c) = v; }, lane);
        if (lane == 0) scale[cur.p] = s;
      }
      if (zero.out && cur.exists && !cur.live) zero.fill(cur.p, lane);
      cur = nrow;
    }
  } else {
    for (; round < rows; advance(), cur = at(round + place)) {
      if (zero.out && cur.exists && !cur.live) zero.fill(cur.p, lane);
      if (!cur.exists || (!cur.live && !zero_pad)) continue;
      int8_t* d = xq + (long long)cur.p * Kp;
      const float s = quant_long<T, kVec>(cur.buf, Kp, [&](int c, uint2 v) { *reinterpret_cast<uint2*>(d + c) = v; },
                                          lane);
      if (lane == 0) scale[cur.p] = s;
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
  int skip_pad;  // k_linear: padding rows of out are left as they are (k_linear_few zeroes them)
};

constexpr int kBK = 128;        // bytes of a row per K stage: whole lines (64-byte pieces halve the loads' rate)
constexpr int kLinWgs = 256;    // one workgroup per CU, each taking tiles in turn
constexpr int kLinLds = 147456; // stage buffers: 3 x 48, 4 x 32 or 8 x 16 KB
constexpr int kLinModes = 4;
constexpr int kGroupM = 8;
// k_linear_few: at most kFewRows rows of kFewK bytes, and at most as many workgroups a CU
// as few_per_cu gives.  Every workgroup quantises its 16 rows again, so the limit falls with
// the cost of that.  us in a graph, this kernel and the two launches of the others:
//   bf16 and 8-bit rows, up to 1024 bytes: five.  K 512 N 2048 1 row 4.1 and 7.1, 128 rows
//     (1024 workgroups) 7.0 and 8.1, 192 rows (1536) 8.7 and 8.2; K 768 N 2304 128 rows
//     (1152) 8.9 and 8.9, and one launch and a workspace less on the host (a call 10 us
//     instead of 15); K 1024 N 4096 64 rows (1024) 8.2 and 9.5, 96 rows (1536) 10.2 and 9.4.
//   the same beyond: two, what 70 KB of LDS each let a CU hold.  K 2304 N 768 64 rows 8.6 and
//     12.2, 128 rows (384) 11.8 and 12.4, 192 rows (576) 16.1 and 12.7; K 4096 N 1024 1 row
//     9.5 and 15.3, 128 rows (512) 13.9 and 16.5, 192 rows 19.4 and 16.8.  8-bit rows alike
//     (K 768 N 2304 128 rows 5.9 and 6.3, 192 rows 7.2 and 6.3; K 2304 N 768 192 rows 12.1
//     and 9.2).
//   float32 rows, up to 1024 bytes: three.  K 1023 N 4096 48 rows (768) 9.2 and 9.5, 64 rows
//     (1024) 10.6 and 9.7; K 767 N 2304 96 rows (864) 10.2 and 9.0.  Beyond: one.  K 4095
//     N 1024 64 rows (256) 17.7 and 18.2, 96 rows (384) 20.8 and 18.4.
//   bf16 rows of odd length, an element a load: one.  K 767 N 768 64 rows (192) 6.8 and 9.0,
//     96 rows (288) 10.2 and 9.0; K 2303 N 768 1 row 12.4 and 14.0, 64 rows (192) 16.2 and
//     15.8, 96 rows (288) 28.7 and 15.9.  Rows of even length at an odd address cost as much
//     and keep the limit of their type: sizes alone decide, since the workspace goes by them.
constexpr int kFewRows = 512, kFewK = 4096;

// Tile shapes: BM x BN, waves along M and N, stage buffers.
template <int kM>
struct LinTile;
template <>
struct LinTile<0> { static constexpr int kBM = 256, kBN = 128, kWgM = 4, kWgN = 2, kNBuf = 3; };
template <>
struct LinTile<1> { static constexpr int kBM = 128, kBN = 128, kWgM = 4, kWgN = 2, kNBuf = 4; };
template <>
struct LinTile<2> { static constexpr int kBM = 64, kBN = 64, kWgM = 2, kWgN = 4, kNBuf = 8; };
template <>
struct LinTile<3> { static constexpr int kBM = 256, kBN = 256, kWgM = 2, kWgN = 4, kNBuf = 2; };

struct LinPlan {
  int mode, T, Nt;
};
constexpr int kStreamMin = 5;  // stages that linear_stream needs: its buffers and two
// The mode with the least rounds of workgroups times the cost of a tile: of a stage
// and of what stands beside the stages, in cycles at 2.4 GHz, from full launches (us,
// modes 0 to 3, random operands: 32768 x 4096 x 1024 164, 178, 334, 121; 32768 x 1024 x
// 4096 179, 215, 498, 160; 24165 x 768 x 768, where the tiles do not fill whole rounds,
// 29, 29, 60, 32).
SC_DEV LinPlan lin_plan(int R, int N, int ns) {
  LinPlan p = {0, 0, 0};
  long long best = 1LL << 62;
#pragma unroll
  for (int m = 0; m < kLinModes; ++m) {
    const int bm = m == 0 || m == 3 ? 256 : m == 1 ? 128 : 64, bn = m == 2 ? 64 : m == 3 ? 256 : 128;
    const int stage = m == 0 ? 2170 : m == 1 ? 1240 : m == 2 ? 500 : 3680;
    const int fixed = m == 0 ? 7700 : m == 1 ? 5600 : m == 2 ? 5000 : 16700;
    const int T = (R + bm - 1) / bm, Nt = (N + bn - 1) / bn;
    const long long rounds = ((long long)T * Nt + kLinWgs - 1) / kLinWgs;
    const long long t = rounds * (ns * stage + fixed);
    if (t < best && (m > 0 || ns >= kStreamMin)) {
      best = t;
      p.mode = m;
      p.T = T;
      p.Nt = Nt;
    }
  }
  return p;
}

// 128-byte rows in LDS, 16-byte units swizzled by bits 1-3 of the row: the fragment
// reads (lane l: row l % 16, unit l / 16 of a chunk's four) run at 226 bytes per clock
// and CU, 64-byte rows swizzled by bits 2-3 at 121.
SC_DEV int q_off(int row, int unit) { return row * kBK + 16 * (unit ^ ((row >> 1) & 7)); }

SC_DEV i32x4 lds_read_q(unsigned addr) {
  return *(const __attribute__((address_space(3))) i32x4*)(size_t)addr;
}

// The row numbering (sc_pack.h) with a table of fixed size: the prefix sums of every
// `per`-th sequence, the rest by a scan of at most per - 1 lengths.
constexpr int kCoarse = 512;
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

// A tile's rows and columns, in LDS.
struct LinTables {
  int row[256];  // of xq and out; rows past the last one repeat it
  float xs[256], sw[256], sb[256];
};

// A workgroup's share of the tiles.  They go to the XCDs in contiguous ranges
// (workgroup i runs on XCD i % 8), in groups of kGroupM row tiles by all column
// tiles: what an XCD runs at a time shares rows and weights in its L2.
struct LinShare {
  long long item, last;
  int T, Nt, step;
  SC_DEV LinShare(const LinPlan& pl) : T(pl.T), Nt(pl.Nt), step(gridDim.x >> 3) {
    const long long items = (long long)T * Nt;
    const int xcd = blockIdx.x & 7;
    last = items * (xcd + 1) / 8;
    item = items * xcd / 8 + (blockIdx.x >> 3);
  }
  template <int kBM, int kBN>
  SC_DEV void place(long long it, int& m0, int& n0) const {
    const int per = kGroupM * Nt, gi = (int)(it / per), rem = (int)(it - (long long)gi * per);
    const int gs = min(kGroupM, T - gi * kGroupM);
    m0 = __builtin_amdgcn_readfirstlane((gi * kGroupM + rem % gs) * kBM);
    n0 = __builtin_amdgcn_readfirstlane(rem / gs * kBN);
  }
};

// What the tiles of one mode share: a wave's part of the loads, fragments, products
// and results.
template <int kM, typename O, bool kGelu>
struct LinWave {
  using S = LinTile<kM>;
  static constexpr int BM = S::kBM, BN = S::kBN, kNBuf = S::kNBuf;
  static constexpr int WM = BM / S::kWgM, WN = BN / S::kWgN, FI = WM / 16, FJ = WN / 16, FH = FI / 2;
  static constexpr int XL = BM / 64, WL = BN / 64, kDma = XL + WL;  // loads of a wave and stage, 8 rows each
  static constexpr int kStage = (BM + BN) * kBK;
  static_assert(kNBuf * kStage <= kLinLds && FI % 2 == 0, "stage buffers, halves of the rows");
  // What a wave stores of a whole tile, in instructions: emit for 16 rows and up to two
  // column fragments at a time, one store of a lane's results each (bf16) or one a fragment
  // (float32).
  static constexpr int kEmits = FI * ((FJ + 1) / 2), kStores = sizeof(O) == 4 ? FI * FJ : kEmits;
  const LinearArgs& a;
  const Packed& pk;
  const int R, tid, lane, w, g, lr, wm, wn;
  const unsigned lds0, xa, wa;
  unsigned xoff[XL], woff[WL];
  i32x4 acc[FI][FJ];
  i32x4 xf[2][FH], wf[2][FJ];  // the fragments of half a wave's rows, and of its columns, twice

  SC_DEV LinWave(const LinearArgs& args, char* stage, const Packed& packed, int rows)
      : a(args), pk(packed), R(rows), tid(threadIdx.x), lane(threadIdx.x & 63),
        w(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)), g(lane >> 4), lr(lane & 15),
        wm((w / S::kWgN) * WM), wn((w % S::kWgN) * WN), lds0(lds_addr(stage)), xa(lds0 + q_off(wm + lr, g)),
        wa(lds0 + BM * kBK + q_off(wn + lr, g)) {}

  // Fills a tile's tables: rows m0 + tid, columns n0 + tid.  The scales come by direct
  // loads, in order with the stages': a wait for a stage loaded later covers them.
  SC_DEV void bring(LinTables& d, int m0, int n0) const {
    if (w < BM / 64) {
      const int p = min(m0 + tid, R - 1), row = a.len ? pk.row(p) : p;
      d.row[tid] = row;
      lds_dma4(a.xs, 4u * (unsigned)row, lds_addr(&d.xs[64 * w]));
    }
    if (w < BN / 64) {
      const unsigned c = 4u * (unsigned)min(n0 + tid, a.N - 1);
      lds_dma4(a.ws, c, lds_addr(&d.sw[64 * w]));
      if (a.bias)
        lds_dma4(a.bias, c, lds_addr(&d.sb[64 * w]));
      else
        d.sb[tid] = 0.f;
    }
  }
  SC_DEV void offsets(const LinTables& d, int n0) {
#pragma unroll
    for (int t = 0; t < XL; ++t) {
      const int R0 = (BM / 8) * w + 8 * t, swz = ((lane >> 4) & 3) | ((R0 >> 1) & 4);
      xoff[t] = (unsigned)d.row[R0 + (lane >> 3)] * (unsigned)a.Kp + 16u * ((lane & 7) ^ swz);
    }
#pragma unroll
    for (int t = 0; t < WL; ++t) {
      const int R0 = (BN / 8) * w + 8 * t, swz = ((lane >> 4) & 3) | ((R0 >> 1) & 4);
      woff[t] = (unsigned)min(n0 + R0 + (lane >> 3), a.N - 1) * (unsigned)a.Kp + 16u * ((lane & 7) ^ swz);
    }
  }
  SC_DEV void issue(int s, int bf) const {  // stage s into buffer bf
    const int8_t *xb = a.xq + (size_t)s * kBK, *wb = a.wq + (size_t)s * kBK;
    const unsigned lx = lds0 + (unsigned)bf * kStage, lw = lx + BM * kBK;
#pragma unroll
    for (int t = 0; t < XL; ++t) lds_dma16(xb, xoff[t], lx + ((BM / 8) * w + 8 * t) * kBK);
#pragma unroll
    for (int t = 0; t < WL; ++t) lds_dma16(wb, woff[t], lw + ((BN / 8) * w + 8 * t) * kBK);
  }
  SC_DEV void cols(int p, int bf, int c) {  // chunk c of 64 k of the stage in buffer bf
#pragma unroll
    for (int j = 0; j < FJ; ++j) wf[p][j] = lds_read_q((wa ^ (64u * c)) + (unsigned)bf * kStage + j * (16 * kBK));
  }
  SC_DEV void rows(int h, int bf, int c) {
#pragma unroll
    for (int i = 0; i < FH; ++i)
      xf[h][i] = lds_read_q((xa ^ (64u * c)) + (unsigned)bf * kStage + (h * FH + i) * (16 * kBK));
    __builtin_amdgcn_sched_barrier(0);  // the reads stay ahead of the products that follow
  }
  SC_DEV void mul(int h, int p) {
#pragma unroll
    for (int i = 0; i < FH; ++i)
#pragma unroll
      for (int j = 0; j < FJ; ++j)
        acc[h * FH + i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wf[p][j], xf[h][i], acc[h * FH + i][j], 0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
  }
  SC_DEV void clear() {
#pragma unroll
    for (int i = 0; i < FI; ++i)
#pragma unroll
      for (int j = 0; j < FJ; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
  }
  static SC_DEV int next_buf(int bf) { return bf == kNBuf - 1 ? 0 : bf + 1; }

  // 16 bytes of a row at column col, at any element's address.  Element by element, rows of
  // odd length take 352 us instead of 227 (32768 x 1024 x 4095; 24165 x 768 x 1111 80 and
  // 41), rows of whole units the same (32768 x 1024 x 4096 152 and 152, with GELU 192 and
  // 189).  The barrier keeps the compiler from running several fragments' results ahead.
  SC_DEV void store16(O* row, int col, uint4 v) const {
    constexpr int kE = 16 / sizeof(O);
    __builtin_amdgcn_sched_barrier(0);
    if (col >= a.N) return;
    if (col + kE <= a.N) {
      *reinterpret_cast<u32x4_any*>(row + col) = __builtin_bit_cast(u32x4_any, v);
    } else {
      const O* e = reinterpret_cast<const O*>(&v);
#pragma unroll
      for (int q = 0; q < kE - 1; ++q)
        if (col + q < a.N) row[col + q] = e[q];
    }
  }
  // Stores 16 rows (16 i on) of two column fragments (j, j + 1; one where a wave has but
  // one): element e of a lane is row 16 i + lr, column 16 j + 4 g + e.  As bf16 a lane
  // holds 8 bytes of each fragment; exchanging them between neighbouring lane groups
  // leaves it with 16 bytes of one, and every group of four lanes with 64 bytes of a row.
  SC_DEV void emit(const i32x4 (&v)[FI][FJ], const LinTables& d, int n0, int i, int j) const {
    const int r = wm + 16 * i + lr;
    __builtin_amdgcn_sched_barrier(0);
    const float xs = d.xs[r];
    O* row = static_cast<O*>(a.out) + (long long)d.row[r] * a.N;
    constexpr int kF = FJ == 1 ? 1 : 2;
    unsigned p[kF][2];
#pragma unroll
    for (int f = 0; f < kF; ++f) {
      const int c = wn + 16 * (j + f) + 4 * g;
      const f32x4 ws = *reinterpret_cast<const f32x4*>(d.sw + c), bs = *reinterpret_cast<const f32x4*>(d.sb + c);
      f32x4 o;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = finish<kGelu>(v[i][j + f][e], xs, ws[e], bs[e]);
      if constexpr (sizeof(O) == 4) {
        store16(row, n0 + c, __builtin_bit_cast(uint4, o));
      } else {
        p[f][0] = pack_bf16(o[0], o[1]);
        p[f][1] = pack_bf16(o[2], o[3]);
      }
    }
    if constexpr (sizeof(O) == 2 && kF == 2) {
      const auto lo = __builtin_amdgcn_permlane16_swap(p[0][0], p[1][0], false, false);
      const auto hi = __builtin_amdgcn_permlane16_swap(p[0][1], p[1][1], false, false);
      store16(row, n0 + wn + 16 * (j + (g & 1)) + 8 * (g >> 1),
              make_uint4((unsigned)lo[0], (unsigned)hi[0], (unsigned)lo[1], (unsigned)hi[1]));
    } else if constexpr (sizeof(O) == 2) {
      const int col = n0 + wn + 16 * j + 4 * g;
      if (col + 4 <= a.N) {
        *reinterpret_cast<u32x2_any*>(row + col) = u32x2_any{p[0][0], p[0][1]};
      } else {
        const O* e = reinterpret_cast<const O*>(p[0]);
#pragma unroll
        for (int q = 0; q < 3; ++q)
          if (col + q < a.N) row[col + q] = e[q];
      }
    }
  }
};

// Tiles one after the other: all stage buffers but the one at hand in flight during a
// tile, the next tile's first stages during its results.  The 256 x 256 form holds all 256
// registers and spills four to eight: what it reloads at the head of a tile waits for every
// access before it, the stages and the last results' stores alike.
template <int kM, typename O, bool kGelu>
SC_DEV void linear_tiles(const LinearArgs& a, char* stage, LinTables* tab, const Packed& pk, int R, const LinPlan& pl) {
  using W = LinWave<kM, O, kGelu>;
  constexpr int kNBuf = W::kNBuf, kDma = W::kDma;
  LinShare sh(pl);
  if (sh.item >= sh.last) return;
  W w(a, stage, pk, R);
  const int ns = a.Kp / kBK;
  // The last tile's stores that the first stages, loaded before them, do not wait for.  A
  // count above the stores issued would let a stage be read before it has landed; below, it
  // only waits longer.
  constexpr int kStores = W::kStores;
  static_assert(kStores == (kM == 1 ? 4 : kM == 2 ? 2 : 16) * (sizeof(O) == 4 && kM != 2 ? 2 : 1),
                "128 x 128, 64 x 64 and 256 x 256 tiles: a wave's stores, 16 bytes a lane (64 x 64 bf16: 8)");
  bool stored = false;
  int m0, n0, cur = 0;
  sh.template place<W::BM, W::BN>(sh.item, m0, n0);
  w.bring(tab[0], m0, n0);
  __syncthreads();
  w.offsets(tab[0], n0);
#pragma unroll
  for (int p = 0; p < kNBuf; ++p)
    if (p < ns) w.issue(p, p);
  while (true) {
    w.clear();
    const long long nitem = sh.item + sh.step;
    const bool more = nitem < sh.last;
    int nm0 = 0, nn0 = 0;
    if (more) sh.template place<W::BM, W::BN>(nitem, nm0, nn0);
    if (stored)
      wait_stages<kNBuf, kDma, kStores>(min(ns, kNBuf) - 1);
    else
      wait_stages<kNBuf, kDma>(min(ns, kNBuf) - 1);
    __syncthreads();  // and the last tile's results have left its tables
    if (more) w.bring(tab[cur ^ 1], nm0, nn0);
    int bf = 0;
    w.cols(0, 0, 0);
    w.rows(0, 0, 0);
    // Two chunks a stage, two halves of the rows each: a half's fragments are in flight
    // during the products of the one before, across stages too.  One barrier per stage,
    // before its last products: the next stage has landed, and this one's buffer is
    // refilled, since every wave holds its last fragments.
    for (int s = 0; s + 1 < ns; ++s) {
      const int bn = W::next_buf(bf);
      w.rows(1, bf, 0);
      w.mul(0, 0);
      w.cols(1, bf, 1);
      w.rows(0, bf, 1);
      w.mul(1, 0);
      w.rows(1, bf, 1);
      w.mul(0, 1);
      if (stored && s + 1 < kNBuf)
        wait_stages<kNBuf - 1, kDma, kStores>(min(ns - 2 - s, kNBuf - 2));
      else
        wait_stages<kNBuf - 1, kDma>(min(ns - 2 - s, kNBuf - 2));
      __syncthreads();
      if (s + kNBuf < ns) w.issue(s + kNBuf, bf);
      w.cols(0, bn, 0);
      w.rows(0, bn, 0);
      w.mul(1, 1);
      bf = bn;
    }
    w.rows(1, bf, 0);
    w.mul(0, 0);
    w.cols(1, bf, 1);
    w.rows(0, bf, 1);
    w.mul(1, 0);
    w.rows(1, bf, 1);
    w.mul(0, 1);
    w.mul(1, 1);
    if (more) {
      __syncthreads();  // every wave has read the last stage
      w.offsets(tab[cur ^ 1], nn0);
#pragma unroll
      for (int p = 0; p < kNBuf; ++p)
        if (p < ns) w.issue(p, p);
    }
#pragma unroll
    for (int i = 0; i < W::FI; ++i)
#pragma unroll
      for (int j = 0; j < W::FJ; j += 2) w.emit(w.acc, tab[cur], n0, i, j);
    stored = n0 + W::BN <= a.N;  // a whole tile: every lane's kStores stores
    if (!more) return;
    sh.item = nitem;
    n0 = nn0;
    cur ^= 1;
  }
}

// The same for tiles of enough stages (kStreamMin), as one stream: the next tile's
// stages follow this one's into the buffers without a gap, and a tile's results are
// finished and stored during the next tile's products, an eighth of a wave's part in
// every stage, so that one wave's arithmetic on results runs beside the other
// waves' matrix instructions, and the stores spread over the whole time.
template <typename O, bool kGelu>
SC_DEV void linear_stream(const LinearArgs& a, char* stage, LinTables* tab, const Packed& pk, int R, const LinPlan& pl) {
  using W = LinWave<0, O, kGelu>;
  constexpr int kNBuf = W::kNBuf, kDma = W::kDma, kUnits = W::kEmits;
  static_assert(kStreamMin == kNBuf + 2, "a barrier between the last tile's results and the next tile's tables");
  LinShare sh(pl);
  if (sh.item >= sh.last) return;
  W w(a, stage, pk, R);
  const int ns = a.Kp / kBK;
  int m0, n0, pn0 = 0, bf = 0;
  int tc = 0, tp = 2, tn = 1;  // tables of this tile, the last one and the next one
  sh.template place<W::BM, W::BN>(sh.item, m0, n0);
  w.bring(tab[tc], m0, n0);
  __syncthreads();
  w.offsets(tab[tc], n0);
#pragma unroll
  for (int p = 0; p < kNBuf; ++p) w.issue(p, p);
  wait_vm<(kNBuf - 1) * kDma>();
  __syncthreads();
  w.cols(0, 0, 0);
  w.rows(0, 0, 0);
  i32x4 done[W::FI][W::FJ];  // the last tile's sums
  bool pending = false;
  while (true) {
    w.clear();
    const long long nitem = sh.item + sh.step;
    const bool more = nitem < sh.last;
    int nm0 = 0, nn0 = 0;
    if (more) sh.template place<W::BM, W::BN>(nitem, nm0, nn0);
    // Stage s; unit u of the last tile's results beside it (none: u < 0).
    auto step = [&](int s, int u) {
      const int bn = W::next_buf(bf);
      w.rows(1, bf, 0);
      w.mul(0, 0);
      if (u >= 0) w.emit(done, tab[tp], pn0, u / (W::FJ / 2), 2 * (u % (W::FJ / 2)));
      w.cols(1, bf, 1);
      w.rows(0, bf, 1);
      w.mul(1, 0);
      w.rows(1, bf, 1);
      w.mul(0, 1);
      const bool turn = more && s == ns - kNBuf - 1;  // not the first stage
      if (more || s + 1 < ns) {
        if (more || s + 2 < ns)
          wait_vm<(kNBuf - 2) * kDma>();
        else
          wait_vm<0>();
        __syncthreads();
        // a barrier into the tile the results of the one before last have left their tables
        if (more && s == 0) w.bring(tab[tn], nm0, nn0);
        if (s + kNBuf < ns)
          w.issue(s + kNBuf, bf);
        else if (more)
          w.issue(s + kNBuf - ns, bf);  // the next tile's
        if (turn) w.offsets(tab[tn], nn0);
        w.cols(0, bn, 0);
        w.rows(0, bn, 0);
      }
      w.mul(1, 1);
      bf = bn;
    };
    int s = 0;
    if (pending) {
#pragma unroll
      for (int u = 0; u < kUnits; ++u) {
        if (s < ns) {
          step(s, u);
          ++s;
        } else {
          w.emit(done, tab[tp], pn0, u / (W::FJ / 2), 2 * (u % (W::FJ / 2)));
        }
      }
    }
    for (; s < ns; ++s) step(s, -1);
#pragma unroll
    for (int i = 0; i < W::FI; ++i)
#pragma unroll
      for (int j = 0; j < W::FJ; ++j) done[i][j] = w.acc[i][j];
    pending = true;
    pn0 = n0;
    if (!more) break;
    n0 = nn0;
    sh.item = nitem;
    const int t = tp;
    tp = tc;
    tc = tn;
    tn = t;
    // the tables of the tile before last are free: its results were finished before the
    // barriers of this tile's last stages
  }
#pragma unroll
  for (int u = 0; u < kUnits; ++u) w.emit(done, tab[tc], pn0, u / (W::FJ / 2), 2 * (u % (W::FJ / 2)));
}

template <typename O, bool kGelu>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2))) void k_linear(LinearArgs a) {
  __shared__ __attribute__((aligned(1024))) char stage[kLinLds];
  __shared__ __attribute__((aligned(16))) LinTables tab[3];
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
      linear_stream<O, kGelu>(a, stage, tab, pk, R, pl);
    else if (pl.mode == 1)
      linear_tiles<1, O, kGelu>(a, stage, tab, pk, R, pl);
    else if (pl.mode == 2)
      linear_tiles<2, O, kGelu>(a, stage, tab, pk, R, pl);
    else
      linear_tiles<3, O, kGelu>(a, stage, tab, pk, R, pl);
  }
  if (!a.len || a.skip_pad) return;
  // zeros into the padding rows, an even share a workgroup
  const long long P = (long long)a.B * a.n - R;
  const long long lo = P * blockIdx.x / gridDim.x, end = P * (blockIdx.x + 1) / gridDim.x;
  const int lane = threadIdx.x & 63;
  const long long bytes = a.N * (long long)sizeof(O);
  for (long long q = lo + (threadIdx.x >> 6); q < end; q += 8)
    zero_bytes(static_cast<char*>(a.out) + pk.pad_row(q) * bytes, bytes, lane);
}

template <typename O, bool kGelu>
hipError_t run_linear(const LinearArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((k_linear<O, kGelu>), dim3(kLinWgs), dim3(512), 0, s, a);
  return hipGetLastError();
}

template <typename T, bool kVec>
hipError_t run_quant(const void* x, int8_t* xq, float* scale, int B, int n, int K, int Kp, const int* len,
                     const int* xidx, int zero_pad, ZeroRows z, hipStream_t s) {
  const long long rows = (long long)B * n;
  const dim3 grid((unsigned)std::min<long long>((rows + 3) / 4, 2048)), block(256);
  const T* xt = static_cast<const T*>(x);
  if (Kp <= 1024)
    hipLaunchKernelGGL((k_quant_rows<T, kVec, 2>), grid, block, 0, s, xt, xq, scale, B, n, K, Kp, len, xidx, zero_pad,
                       z);
  else if (Kp <= 4096)
    hipLaunchKernelGGL((k_quant_rows<T, kVec, 8>), grid, block, 0, s, xt, xq, scale, B, n, K, Kp, len, xidx, zero_pad,
                       z);
  else
    hipLaunchKernelGGL((k_quant_rows<T, kVec, 0>), grid, block, 0, s, xt, xq, scale, B, n, K, Kp, len, xidx, zero_pad,
                       z);
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
    // rows held at once, as registers allow (an element a load: 272 with two, one workgroup a CU)
    constexpr int kAtOnce = kUnits == 2 || (kVec && sizeof(T) == 2) ? 4 : kVec ? 2 : 1;
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
  const float v = on ? finish<kGelu>(sum, ss[r], a.ws[col], a.bias ? a.bias[col] : 0.f) : 0.f;
  store_out(static_cast<O*>(a.out) + m * a.N + col, v);
}

}  // namespace

hipError_t launch_quant_rows(const void* x, int f32, int8_t* xq, float* scale, int B, int n, int K, const int* len,
                             const int* xidx, int zero_pad, void* zero_out, long long zero_row, hipStream_t s) {
  const int Kp = i8_pitch(K);
  const ZeroRows z = {static_cast<char*>(zero_out), zero_row};
  const bool vec = K % 2 == 0 && reinterpret_cast<uintptr_t>(x) % 4 == 0;
  if (f32) return run_quant<float, true>(x, xq, scale, B, n, K, Kp, len, xidx, zero_pad, z, s);
  return vec ? run_quant<__bf16, true>(x, xq, scale, B, n, K, Kp, len, xidx, zero_pad, z, s)
             : run_quant<__bf16, false>(x, xq, scale, B, n, K, Kp, len, xidx, zero_pad, z, s);
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
  a.skip_pad = l.skip_pad;
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

namespace {
int few_per_cu(int K, int x_type) {
  const bool longer = i8_pitch(K) > 1024;
  if (x_type == 1 && K % 2 != 0) return 1;
  if (x_type == 0) return longer ? 1 : 3;
  return longer ? 2 : 5;
}
}  // namespace

bool linear_few_ok(long long rows, int K, int N, int x_type) {
  if (rows > kFewRows || i8_pitch(K) > kFewK) return false;
  return (rows + 15) / 16 * ((N + 15) / 16) <= few_per_cu(K, x_type) * kLinWgs;
}

hipError_t launch_linear_few(const Linear& l, const void* x, int x_type, hipStream_t s) {
  const bool vec = l.K % 2 == 0 && reinterpret_cast<uintptr_t>(x) % 4 == 0;
  if (x_type == 2) return run_few<int8_t, true>(l, x, s);
  if (x_type == 0) return run_few<float, true>(l, x, s);
  return vec ? run_few<__bf16, true>(l, x, s) : run_few<__bf16, false>(l, x, s);
}

hipError_t launch_linear_i8(const Linear& l, hipStream_t s) {
  const LinearArgs a = linear_args(l);
  if (l.out_f32) return l.gelu ? run_linear<float, true>(a, s) : run_linear<float, false>(a, s);
  return l.gelu ? run_linear<__bf16, true>(a, s) : run_linear<__bf16, false>(a, s);
}

}  // namespace sc
