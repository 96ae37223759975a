// Matrix products in 8-bit integers with a scale for each token and channel.
//
//   out[t, n] = act(s_t w_n sum_k q[t, k] wq[n, k] + bias[n])
//
// k_quant_rows    the tokens' 8-bit rows (sc_quant.h), one wavefront a row.
// k_quant_weight  the weights', once per model.
// k_linear        the product on v_mfma_i32_16x16x64_i8: sums of up to 131072
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
  const float a = fminf(fabsf(v), 16.f);
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
// Eight elements from column c on; zeros at and beyond K.
template <typename T, bool kVec>
struct Unit8 {
  T v[8];
  SC_DEV void load(const T* row, int c, int K) {
    if (kVec) {
      if (c < K) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i)
          reinterpret_cast<uint4*>(v)[i] = reinterpret_cast<const uint4*>(row + c)[i];
        return;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = (T)0.f;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = c + i < K ? row[c + i] : (T)0.f;
    }
  }
  SC_DEV float amax() const {
    float a = fabsf((float)v[0]);
#pragma unroll
    for (int i = 1; i < 8; ++i) a = vmax(a, fabsf((float)v[i]));
    return a;
  }
  SC_DEV uint2 quant(const RowQuant& r) const {
    unsigned q[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = quant_one<T>(r, (float)v[i]);
    return make_uint2(pack_i8(q[0], q[1], q[2], q[3]) & r.live, pack_i8(q[4], q[5], q[6], q[7]) & r.live);
  }
};

// One wavefront quantises one row of K elements into Kp bytes at dst (global or
// LDS); returns the scale.  A lane holds its kUnits units of eight elements
// (K <= 512 kUnits); kUnits 0 reads the row twice.
template <typename T, bool kVec, int kUnits, typename Dst>
SC_DEV float quant_row(const T* __restrict__ src, int K, int Kp, Dst dst, int lane) {
  if constexpr (kUnits > 0) {
    Unit8<T, kVec> u[kUnits];
    float a = 0.f;
#pragma unroll
    for (int i = 0; i < kUnits; ++i) u[i].load(src, 8 * (lane + 64 * i), K);
#pragma unroll
    for (int i = 0; i < kUnits; ++i) a = vmax(a, u[i].amax());
    const RowQuant r = row_quant(butterfly_max(a));
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
      const int c = 8 * (lane + 64 * i);
      if (c < Kp) dst(c, u[i].quant(r));
    }
    return r.scale;
  } else {
    float a = 0.f;
    for (int c = 8 * lane; c < K; c += 512) {
      Unit8<T, kVec> u;
      u.load(src, c, K);
      a = vmax(a, u.amax());
    }
    const RowQuant r = row_quant(butterfly_max(a));
    for (int c = 8 * lane; c < Kp; c += 512) {
      Unit8<T, kVec> u;
      u.load(src, c, K);
      dst(c, u.quant(r));
    }
    return r.scale;
  }
}

// Rows dealt round-robin over the launch's waves.  packed: row p of the output
// is the p-th surviving row (pack_seq), read through xidx; else rows keep their
// places and padding rows become zeros.
template <typename T, bool kVec, int kUnits>
__global__ __launch_bounds__(256) void k_quant_rows(const T* __restrict__ x, int8_t* __restrict__ xq,
                                                    float* __restrict__ scale, int B, int n, int K, int Kp,
                                                    const int* __restrict__ len, const int* __restrict__ xidx,
                                                    int packed) {
  extern __shared__ int pre[];
  const int lane = threadIdx.x & 63;
  long long rows = (long long)B * n;
  if (packed && len) {
    pack_prefix(pre, len, B, n);
    __syncthreads();
    rows = pre[B];
  }
  for (long long p = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); p < rows;
       p += (long long)gridDim.x * 4) {
    long long from = p;
    bool live = true;
    if (packed) {
      if (len) {
        const int b = pack_seq(pre, B, (int)p);
        from = (long long)b * n + (p - pre[b]);
      }
      if (xidx) from = from / n * n + clampi(xidx[from], 0, n - 1);
    } else if (len) {
      const long long b = p / n;
      live = (int)(p - b * n) < clampi(len[b], 0, n);
    }
    int8_t* d = xq + p * Kp;
    auto dst = [&](int c, uint2 v) { *reinterpret_cast<uint2*>(d + c) = v; };
    float s = 0.f;
    if (live) {
      s = quant_row<T, kVec, kUnits>(x + from * K, K, Kp, dst, lane);
    } else {
      for (int c = 8 * lane; c < Kp; c += 512) dst(c, make_uint2(0, 0));
    }
    if (lane == 0) scale[p] = s;
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

constexpr int kBK = 64;                // bytes of a row per K stage
constexpr int kLinStage = 73728;       // stage buffers
constexpr int kLinModes = 3;
constexpr int kLinBm[kLinModes] = {256, 128, 64}, kLinBn[kLinModes] = {128, 128, 64};
constexpr int kGroupM = 8;
// 256 x 128 tiles from kLinTall of them on, else 128 x 128 tiles from kLinWide of
// them on, else 64 x 64.
constexpr int kLinTall = 512, kLinWide = 256;

struct LinPlan {
  int mode, bm, bn, T, Nt;
};
SC_DEV LinPlan lin_plan(int R, int N) {
  LinPlan p;
  const int nt = (N + 127) / 128;
  if ((long long)((R + 255) / 256) * nt >= kLinTall)
    p.mode = 0;
  else if ((long long)((R + 127) / 128) * nt >= kLinWide)
    p.mode = 1;
  else
    p.mode = 2;
  p.bm = p.mode == 0 ? 256 : p.mode == 1 ? 128 : 64;
  p.bn = p.mode == 2 ? 64 : 128;
  p.T = (R + p.bm - 1) / p.bm;
  p.Nt = (N + p.bn - 1) / p.bn;
  return p;
}

// 64-byte rows in LDS: 16-byte units swizzled by bits 2-3 of the row, so that
// 16 consecutive rows read at one unit hit 16 distinct 16-byte bank groups.
SC_DEV int q_off(int row, int unit) { return row * kBK + 16 * (unit ^ ((row >> 2) & 3)); }

SC_DEV i32x4 lds_read_q(unsigned addr) {
  return *(const __attribute__((address_space(3))) i32x4*)(size_t)addr;
}

template <int kM, typename O, bool kGelu>
SC_DEV void linear_tile(const LinearArgs& a, char* stage, const int* grow, const int* xrow, const float* sw,
                        const float* sb, int n0) {
  constexpr int BM = kLinBm[kM], BN = kLinBn[kM];
  constexpr int WM = BM / 2, WN = BN / 2, FI = WM / 16, FJ = WN / 16;
  constexpr int XL = BM / 64, WL = BN / 64, kDma = XL + WL;
  constexpr int kStage = (BM + BN) * kBK;
  constexpr int kNBuf = kLinStage / kStage < 6 ? kLinStage / kStage : 6;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4,
            lr = lane & 15;
  const int wm = (w >> 1) * WM, wn = (w & 1) * WN;
  const int u = 16 * ((lane & 3) ^ ((lane >> 4) & 3));
  unsigned xoff[XL], woff[WL];
#pragma unroll
  for (int t = 0; t < XL; ++t) xoff[t] = (unsigned)xrow[(BM / 4) * w + 16 * t + (lane >> 2)] * (unsigned)a.Kp + u;
#pragma unroll
  for (int t = 0; t < WL; ++t)
    woff[t] = (unsigned)min(n0 + (BN / 4) * w + 16 * t + (lane >> 2), a.N - 1) * (unsigned)a.Kp + u;
  const unsigned lds0 = lds_addr(stage);
  auto issue = [&](int s, int bf) {
    const int8_t *xb = a.xq + (size_t)s * kBK, *wb = a.wq + (size_t)s * kBK;
    const unsigned lx = lds0 + (unsigned)bf * kStage, lw = lx + BM * kBK;
#pragma unroll
    for (int t = 0; t < XL; ++t) lds_dma16(xb, xoff[t], lx + ((BM / 4) * w + 16 * t) * kBK);
#pragma unroll
    for (int t = 0; t < WL; ++t) lds_dma16(wb, woff[t], lw + ((BN / 4) * w + 16 * t) * kBK);
  };
  i32x4 acc[FI][FJ];
#pragma unroll
  for (int i = 0; i < FI; ++i)
#pragma unroll
    for (int j = 0; j < FJ; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
  const int ns = a.Kp / kBK;
#pragma unroll
  for (int p = 0; p < kNBuf - 1; ++p)
    if (p < ns) issue(p, p);
  const unsigned xa = lds0 + q_off(wm + lr, g), wa = lds0 + BM * kBK + q_off(wn + lr, g);
  int bf = 0;
  for (int s = 0; s < ns; ++s) {
    wait_stages<kNBuf - 1, kDma>(min(ns - 1 - s, kNBuf - 2));
    __syncthreads();
    if (s + kNBuf - 1 < ns) issue(s + kNBuf - 1, bf == 0 ? kNBuf - 1 : bf - 1);
    const unsigned o = (unsigned)bf * kStage;
    i32x4 af[FI], wf[FJ];
#pragma unroll
    for (int j = 0; j < FJ; ++j) wf[j] = lds_read_q(wa + o + j * (16 * kBK));
#pragma unroll
    for (int i = 0; i < FI; ++i) af[i] = lds_read_q(xa + o + i * (16 * kBK));
#pragma unroll
    for (int i = 0; i < FI; ++i)
#pragma unroll
      for (int j = 0; j < FJ; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wf[j], af[i], acc[i][j], 0, 0, 0);
    bf = bf == kNBuf - 1 ? 0 : bf + 1;
  }
  // A lane holds four consecutive columns of a row (row wm + 16 i + lr, columns
  // wn + 16 j + 4 g ..).  The wave's part goes through LDS, 32 rows at a time,
  // and leaves as whole 16-byte units.
  constexpr int es = sizeof(O), kPitch = WN * es + 16, kUr = WN * es / 16, kEpu = 16 / es;
  static_assert(4 * 32 * kPitch <= kLinStage, "staging rows");
  __syncthreads();  // every wave has read the last stage
  char* st = stage + w * (32 * kPitch);
#pragma unroll
  for (int c = 0; c < WM / 32; ++c) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float s = a.xs[xrow[wm + 32 * c + 16 * i + lr]];
#pragma unroll
      for (int j = 0; j < FJ; ++j) {
        const f32x4 ws = *reinterpret_cast<const f32x4*>(sw + wn + 16 * j + 4 * g);
        const f32x4 bs = *reinterpret_cast<const f32x4*>(sb + wn + 16 * j + 4 * g);
        char* d = st + (16 * i + lr) * kPitch + (16 * j + 4 * g) * es;
        f32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = finish<es == 4, kGelu>(acc[2 * c + i][j][e], s, ws[e], bs[e]);
        if constexpr (es == 4) {
          *reinterpret_cast<f32x4*>(d) = v;
        } else {
          *reinterpret_cast<uint2*>(d) = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
        }
      }
    }
#pragma unroll
    for (int t = 0; t < 32 * kUr / 64; ++t) {
      const int r = t * (64 / kUr) + lane / kUr, un = lane % kUr, gr = grow[wm + 32 * c + r];
      const int col = n0 + wn + un * kEpu;
      const uint4 v = *reinterpret_cast<const uint4*>(st + r * kPitch + 16 * un);
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
  }
}

template <typename O, bool kGelu>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void k_linear(LinearArgs a) {
  __shared__ __attribute__((aligned(1024))) char stage[kLinStage];
  __shared__ int grow[256], xrow[256];
  __shared__ __attribute__((aligned(16))) float sw[128], sb[128];
  int* pre = reinterpret_cast<int*>(stage);  // until the first stage lands
  const int tid = threadIdx.x;
  int R = a.B * a.n;
  if (a.len) {
    pack_prefix(pre, a.len, a.B, a.n);
    __syncthreads();
    R = __builtin_amdgcn_readfirstlane(pre[a.B]);
  }
  const LinPlan pl = lin_plan(R, a.N);
  // The items are dealt to the XCDs in contiguous ranges (workgroup i runs on XCD
  // i % 8), and in groups of kGroupM row tiles by all column tiles: what runs at
  // a time on an XCD shares rows and weights in its L2.
  const long long items = (long long)pl.T * pl.Nt;
  const int x = blockIdx.x & 7;
  const long long item = items * x / 8 + (blockIdx.x >> 3);
  if (item < items * (x + 1) / 8) {
    const int per = kGroupM * pl.Nt, gi = (int)(item / per), rem = (int)(item - (long long)gi * per);
    const int gs = min(kGroupM, pl.T - gi * kGroupM);
    const int m0 = (gi * kGroupM + rem % gs) * pl.bm, n0 = rem / gs * pl.bn;
    if (tid < pl.bm) {
      const int p = min(m0 + tid, R - 1);  // rows past the last one read it again
      int gr = p;
      if (a.len) {
        const int b = pack_seq(pre, a.B, p);
        gr = b * a.n + (p - pre[b]);
      }
      grow[tid] = m0 + tid < R ? gr : -1;
      xrow[tid] = a.packed ? p : gr;
    }
    if (tid < pl.bn) {
      const int c = min(n0 + tid, a.N - 1);
      sw[tid] = a.ws[c];
      sb[tid] = a.bias ? a.bias[c] : 0.f;
    }
    __syncthreads();  // the prefix table is dead from here: the stages overwrite it
    if (pl.mode == 0)
      linear_tile<0, O, kGelu>(a, stage, grow, xrow, sw, sb, n0);
    else if (pl.mode == 1)
      linear_tile<1, O, kGelu>(a, stage, grow, xrow, sw, sb, n0);
    else
      linear_tile<2, O, kGelu>(a, stage, grow, xrow, sw, sb, n0);
  }
  if (!a.len || a.skip_pad) return;
  // zeros into the padding rows, an even share a workgroup
  const long long P = (long long)a.B * a.n - R;
  const long long lo = P * blockIdx.x / gridDim.x, hi = P * (blockIdx.x + 1) / gridDim.x;
  if (lo >= hi) return;
  __syncthreads();  // the staging rows have been read
  pack_prefix(pre, a.len, a.B, a.n);
  __syncthreads();
  for (long long q = lo + (tid >> 6); q < hi; q += 4) {
    int l = 0, h = a.B - 1;  // the largest b with b n - pre[b] <= q
    while (l < h) {
      const int mid = (l + h + 1) >> 1;
      if ((long long)mid * a.n - pre[mid] <= q) l = mid;
      else h = mid - 1;
    }
    // row pre[l + 1] - pre[l] + (q - (l n - pre[l])) of sequence l, in place
    O* o = static_cast<O*>(a.out) + (q + pre[l + 1]) * a.N;
    if (a.vec) {
      for (int c = tid & 63; c < a.N / (16 / (int)sizeof(O)); c += 64)
        reinterpret_cast<uint4*>(o)[c] = make_uint4(0, 0, 0, 0);
    } else {
      for (int c = tid & 63; c < a.N; c += 64) o[c] = (O)0.f;
    }
  }
}

template <typename O, bool kGelu>
hipError_t run_linear(const LinearArgs& a, hipStream_t s) {
  const long long items = linear_tiles((long long)a.B * a.n, a.N);
  hipLaunchKernelGGL((k_linear<O, kGelu>), dim3((unsigned)(8 * ((items + 7) / 8))), dim3(256), 0, s, a);
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

// At most the tiles of all rows in each mode: fewer rows take smaller tiles only
// while the larger ones are few.
long long linear_tiles(long long rows, int N) {
  const long long nt = (N + 127) / 128;
  long long items = (rows + 255) / 256 * nt;
  items = std::max(items, std::min<long long>((rows + 127) / 128 * nt, 2 * kLinTall));
  return std::max(items, std::min<long long>((rows + 63) / 64 * ((N + 63) / 64), 4 * kLinWide));
}

hipError_t launch_linear_i8(const Linear& l, hipStream_t s) {
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
  if (l.out_f32) return l.gelu ? run_linear<float, true>(a, s) : run_linear<float, false>(a, s);
  return l.gelu ? run_linear<__bf16, true>(a, s) : run_linear<__bf16, false>(a, s);
}

}  // namespace sc
