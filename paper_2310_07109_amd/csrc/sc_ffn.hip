// The gated feed-forward block, forward: y = (act(x Wg) * (x Wu)) Wd.  The products are in
// sc_ffn.h; the matrix units bound them where there are rows, the weights' bytes where
// there are few.
#include <algorithm>

#include "sc_ffn.h"

namespace sc {
namespace {

// A wavefront a row of one job: the numbering and the zeros of the batch's rows, then every
// copy's rows (one after the other in the same wave, five jobs of an odd-sized batch took
// 11 us for 1503 rows, side by side 8).  The search for a row's place and memory bound it:
// 32768 rows of 1024 to zero or number 6 us.
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
  const bool whole = R == T, rows = a.always || !whole;
  // The packed row of row r, or -1.
  auto packed = [&](long long r) -> long long {
    if (!a.len) return r;
    const int b = (int)(r / a.n), j = (int)(r - (long long)b * a.n), first = pre[b];
    return j < pre[b + 1] - first ? first + j : -1;
  };
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
  const long long step = (long long)gridDim.x * 4;
  long long at = (long long)blockIdx.x * 4 + w;
  if (a.len) {
    for (; at < T; at += step) {
      const long long to = packed(at);
      if (to >= 0) {
        if (lane == 0) a.map[to] = (int)at;
      } else if (a.zero) {
        char* z = a.zero + at * a.zero_bytes;
        for (long long c = 16 * lane; c < a.zero_bytes; c += 1024) {
          if (c + 16 <= a.zero_bytes) *reinterpret_cast<u32x4_any*>(z + c) = u32x4_any{0, 0, 0, 0};
          else
            for (long long i = c; i < a.zero_bytes; i += 2) *reinterpret_cast<unsigned short*>(z + i) = 0;
        }
      }
    }
    at -= T;
  }
#pragma unroll
  for (int i = 0; i < kFfnCopies; ++i) {
    if (i >= a.copies) break;
    const FfnCopy& c = a.copy[i];
    if (c.rows == 0 && !rows) continue;
    const long long count = c.rows == 0 ? T : c.rows;
    for (; at < count; at += step) {
      const long long to = c.rows == 0 ? packed(at) : at;
      if (to >= 0) copy(c, at, to);
    }
    at -= count;
  }
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

// ----------------------------------------------------------- few rows ----
// A few rows are bound by the weights' bytes and by latency: every wave asks for all of
// its part of them at once.  A workgroup takes 16 kMF rows and 32 columns (of Wg and of Wu),
// its waves a share of the contraction each, in chunks of 32.  A lane reads two
// columns of eight successive rows of W and has, with a byte permutation for each pair,
// the fragments of both: nothing goes through LDS but the waves' sums, added in order.
// The columns are dealt so that neighbouring blocks, halves of a line, share an L2.
struct FewArgs {
  const char *x, *w[2];  // rows of ldx bytes, [K, N] with rows of ldw bytes
  __bf16* out;           // rows of ldo elements
  unsigned ldx, ldw, ldo;
  int T, N, K;
  const int* len;        // rows at and beyond a sequence's length become zeros, or null
  int n;
};

// kAhead: chunks of a wave in flight.
template <int kMF, bool kPair, int kAct, int kFewWaves, int kAhead>
__global__ __launch_bounds__(64 * kFewWaves) __attribute__((amdgpu_waves_per_eu(kFewWaves / 4))) void k_ffn_few(FewArgs a) {
  constexpr int kMats = kPair ? 2 : 1, kFrags = kMF * 2 * kMats;
  __shared__ float red[kFewWaves][kFrags * 256];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4,
            lr = lane & 15;
  const int blocks = (a.N + 31) / 32, per = (blocks + 7) / 8, c = ((int)blockIdx.x & 7) * per + ((int)blockIdx.x >> 3);
  if (c >= blocks) return;
  const int n0 = 32 * c, m0 = (int)blockIdx.y * 16 * kMF;
  const u32x4 zero = {0, 0, 0, 0};
  auto buffer = [](const char* p, unsigned bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(p), 0, (int)bytes, 0x00027000);
  };
  const auto bx = buffer(a.x, (unsigned)a.T * a.ldx), b0 = buffer(a.w[0], (unsigned)a.K * a.ldw),
             b1 = buffer(a.w[kMats - 1], (unsigned)a.K * a.ldw);
  const int chunks = (a.K + 31) / 32;
  struct Chunk {
    unsigned w[kMats][8];
    u32x4 x[kMF];
  };
  auto load = [&](Chunk& ch, int i) {
    const int k = 32 * i + 8 * g;  // rows beyond K lie beyond the buffers' ends
    const unsigned at = (unsigned)k * a.ldw + 2u * (n0 + 2 * lr);
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      ch.w[0][r] = __builtin_amdgcn_raw_buffer_load_b32(b0, at + r * a.ldw, 0, 0);
      if constexpr (kPair) ch.w[1][r] = __builtin_amdgcn_raw_buffer_load_b32(b1, at + r * a.ldw, 0, 0);
    }
#pragma unroll
    for (int m = 0; m < kMF; ++m)
      ch.x[m] = __builtin_amdgcn_raw_buffer_load_b128(
          bx, k < a.K ? (unsigned)(m0 + 16 * m + lr) * a.ldx + 2u * k : kBeyond, 0, 0);
  };
  f32x4 acc[kMF][kMats][2];
#pragma unroll
  for (int m = 0; m < kMF; ++m)
#pragma unroll
    for (int q = 0; q < kMats; ++q) acc[m][q][0] = acc[m][q][1] = f32x4{0.f, 0.f, 0.f, 0.f};
  Chunk ch[kAhead];
#pragma unroll
  for (int i = 0; i < kAhead; ++i) load(ch[i], w + kFewWaves * i);
  for (int i = w; i < chunks; i += kFewWaves * kAhead) {
#pragma unroll
    for (int q = 0; q < kAhead; ++q) {
#pragma unroll
      for (int mat = 0; mat < kMats; ++mat)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          u32x4 f = zero;
#pragma unroll
          for (int p = 0; p < 4; ++p)
            f[p] = __builtin_amdgcn_perm(ch[q].w[mat][2 * p + 1], ch[q].w[mat][2 * p], j ? 0x07060302u : 0x05040100u);
#pragma unroll
          for (int m = 0; m < kMF; ++m)
            acc[m][mat][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                __builtin_bit_cast(bf16x8, ch[q].x[m]), __builtin_bit_cast(bf16x8, f), acc[m][mat][j], 0, 0, 0);
        }
      load(ch[q], i + kFewWaves * (kAhead + q));
    }
  }
#pragma unroll
  for (int m = 0; m < kMF; ++m)
#pragma unroll
    for (int q = 0; q < kMats; ++q)
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) red[w][((m * kMats + q) * 2 + j) * 256 + 64 * e + lane] = acc[m][q][j][e];
  __syncthreads();
  // element e of lane (g, lr): row 4 g + e, columns 2 lr and 2 lr + 1
  for (int i = tid; i < kMF * 256; i += 64 * kFewWaves) {
    const int m = i >> 8, e = (i >> 6) & 3, l = i & 63, row = m0 + 16 * m + 4 * (l >> 4) + e, col = n0 + 2 * (l & 15);
    if (row >= a.T || col >= a.N) continue;
    bool live = true;
    if (a.len) {
      const unsigned b = (unsigned)row / (unsigned)a.n;
      live = (int)((unsigned)row - b * a.n) < clampi(a.len[b], 0, a.n);
    }
    float v[kMats][2];
#pragma unroll
    for (int q = 0; q < kMats; ++q)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int at = ((m * kMats + q) * 2 + j) * 256 + 64 * e + l;
        float s = red[0][at];
#pragma unroll
        for (int k = 1; k < kFewWaves; ++k) s += red[k][at];
        v[q][j] = s;
      }
    float o[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) o[j] = live ? (kPair ? act<kAct>(v[0][j]) * v[kMats - 1][j] : v[0][j]) : 0.f;
    *reinterpret_cast<unsigned*>(a.out + (long long)row * a.ldo + col) = pack_bf16(o[0], o[1]);
  }
}

template <int kMF, bool kPair, int kAct, int kWaves, int kAhead>
hipError_t run_few(const FewArgs& a, hipStream_t s) {
  const int blocks = (a.N + 31) / 32, grid = (blocks + 7) / 8 * 8;
  hipLaunchKernelGGL((k_ffn_few<kMF, kPair, kAct, kWaves, kAhead>), dim3(grid, (a.T + 16 * kMF - 1) / (16 * kMF)),
                     dim3(64 * kWaves), 0, s, a);
  return hipGetLastError();
}
template <int kAct>
hipError_t few_gate(const FewArgs& a, hipStream_t s) {
  if (a.T <= 16) return run_few<1, true, kAct, 16, 2>(a, s);
  if (a.T <= 32) return run_few<2, true, kAct, 8, 4>(a, s);
  return run_few<4, true, kAct, 8, 3>(a, s);
}

// The forward of a few rows, where nothing is kept and nothing has to be copied.  us in a
// graph, these two launches and the three of the tiles: 512 x 1536, 1 row 9.6 and 17.1, 128
// rows 16.3 and 17.9; 768 x 2304, 1 row 10.7 and 21.2, 128 rows 19.3 and 22.8; 1024 x 4096,
// 1 row 11.9 and 30.5, 128 rows 27.9 and 33.4.
constexpr int kFewRows = 128;
// Chunks beyond the contraction are asked for, up to 16 waves' last ones: their offsets
// stay below 32 bits, and the buffers give zeros for them.
constexpr long long kFewBeyond = 8192;
bool few_ok(const Ffn& a) {
  return !a.saved && !ffn_odd(a) && (long long)a.B * a.n <= kFewRows &&
         (a.D + kFewBeyond) * 2 * a.F < (1LL << 32) && (a.F + kFewBeyond) * 2 * a.D < (1LL << 32);
}

hipError_t launch_few(const Ffn& a, char* h, hipStream_t s) {
  FewArgs g = {};
  g.x = static_cast<const char*>(a.x);
  g.w[0] = static_cast<const char*>(a.wg);
  g.w[1] = static_cast<const char*>(a.wu);
  g.out = reinterpret_cast<__bf16*>(h);
  g.ldx = 2u * a.D;
  g.ldw = 2u * a.F;
  g.ldo = a.F;
  g.T = a.B * a.n;
  g.N = a.F;
  g.K = a.D;
  const hipError_t e = a.act == kActGelu   ? few_gate<kActGelu>(g, s)
                       : a.act == kActSilu ? few_gate<kActSilu>(g, s)
                                           : few_gate<kActNone>(g, s);
  if (e != hipSuccess) return e;
  FewArgs d = g;
  d.x = h;
  d.w[0] = d.w[1] = static_cast<const char*>(a.wd);
  d.out = static_cast<__bf16*>(a.y);
  d.ldx = 2u * a.F;
  d.ldw = 2u * a.D;
  d.ldo = a.D;
  d.N = a.D;
  d.K = a.F;
  d.len = a.len;
  d.n = a.n;
  return d.T <= 16 ? run_few<1, false, kActNone, 16, 4>(d, s) : run_few<2, false, kActNone, 16, 4>(d, s);
}

template <int kAct>
hipError_t gate(const FfnArgs& g, int tile, hipStream_t s) {
  return g.blocks ? run_ffn<kGateKeep, kAct>(g, tile, s) : run_ffn<kGate, kAct>(g, tile, s);
}

}  // namespace

hipError_t launch_ffn_rows(const void* rows, hipStream_t s) {
  const FfnRows& r = *static_cast<const FfnRows*>(rows);
  const long long T = (long long)r.B * r.n;
  long long jobs = r.len ? T : 0;
  for (int i = 0; i < r.copies; ++i) jobs += r.copy[i].rows == 0 ? T : r.copy[i].rows;
  hipLaunchKernelGGL(k_ffn_rows, dim3((unsigned)std::min<long long>((jobs + 3) / 4, 2048)), dim3(256), 0, s, r);
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
  if (few_ok(a)) return launch_few(a, ws.h, s);
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
