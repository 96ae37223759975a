// The tiled matrix products of the gated feed-forward block, forward and backward.
//
// Six products, one form.  The contraction of an operand lies along its rows in memory
// (x . Wd^T) or across them (x . W, x^T . g): both are staged as they lie, in whole lines,
// by direct loads, and the second kind is transposed on the way from LDS to the fragments
// (ds_read_b64_tr_b16), so no operand is ever laid out anew.
//
//   kGate  g = x Wg, u = x Wu     h = act(g) u; kept for the backward: act(g) and u act'(g)
//   kDown  y = h Wd
//   kDh    dh = dy Wd^T           dg = dh u act'(g), du = dh act(g)
//   kDx    dx = dg Wg^T + du Wu^T, one sum over 2 F
//   kDwd   dWd = h^T dy           over the rows, in slabs
//   kDwgu  dWg = x^T dg, dWu = x^T du
//
// A tile is BM x BN of a workgroup of eight waves; a stage is 64 of the contraction.
// Sums are float32 in ascending order of the contraction, whatever the tile.  What the next
// product reads, h, dg and du, is rounded to bf16, as the matrix units take it (a second bf16
// part of each would be two thirds as many products again in a training step); y and every
// gradient then have two roundings behind them, 0.0023 of their norm off where float32 in
// between would leave 0.0017.
//
// The matrix units bound them, at the clock that their power leaves, and beside them the
// results, which one workgroup a CU does not overlap with products.  32768 rows, D 1024,
// F 2816, least of 20, us (PFLOP/s): gate and its factors 390 (0.97), down 177 (1.07), dh and
// dWd 463 (0.82; apart 333 and 160), dx, dWg and dWu 638 (1.18; apart 296 and 342); gate
// alone, F 4096, 447 (1.23), down 225 (1.22).  dh is as long as its products (160, as dWd's)
// and a copy of its 923 MB of factors and results (180) one after the other.  A library's
// products of such shapes reach 0.86 to 1.46 without the activation.
#pragma once
#include "sc_act.h"
#include "sc_device.h"
#include "sc_internal.h"
#include "sc_pack.h"

namespace sc {
namespace {

typedef __attribute__((ext_vector_type(4))) unsigned u32x4;
typedef __attribute__((ext_vector_type(2))) unsigned u32x2;
typedef u32x4 __attribute__((aligned(2))) u32x4_any;
typedef __attribute__((ext_vector_type(2), aligned(2))) unsigned u32x2_any;
typedef f32x4 __attribute__((aligned(4))) f32x4_any;

constexpr int kGate = 0, kDown = 1, kDh = 2, kDx = 3, kDwd = 4, kDwgu = 5, kGateKeep = 6;  // 6: kGate that keeps the factors
constexpr int kFfnWgs = 256;   // CUs; workgroups take tiles in turn
constexpr int kGroupTiles = 8;  // row tiles that share weights in an XCD's L2

template <int kM>
struct FfnTile;
template <>
struct FfnTile<0> { static constexpr int kBM = 256, kBN = 256, kWgM = 2, kWgN = 4, kNBuf = 2; };
template <>
struct FfnTile<1> { static constexpr int kBM = 128, kBN = 128, kWgM = 2, kWgN = 4, kNBuf = 4; };
template <>
struct FfnTile<2> { static constexpr int kBM = 64, kBN = 64, kWgM = 4, kWgN = 2, kNBuf = 4; };

// One operand: rows of ld bytes.  Those whose row count is the batch's come packed (the
// valid rows, one after the other) or, when no row is padding, from where they are.
struct FfnOperand {
  const char* p[2];
  const char* packed;  // instead of p[0] when rows are padding, or null
  unsigned ld;
  int rows;            // 0: the valid rows
};

struct FfnArgs {
  FfnOperand a, b;
  const int* map;    // packed row -> row of the batch (null: the same)
  const int* count;  // the number of valid rows (null: T)
  int T;
  int M, N, K;       // output rows (kDwd, kDwgu), columns, contraction (not kDwd, kDwgu)
  int map_a;         // a's rows are the batch's: read through map
  void* out[2];      // bf16: h | y | dg, du | dx | dwd | dwg, dwu
  int ld;            // elements of its rows
  char* blocks;      // kGate: the factors for the backward, or null; kDh: to read
  int across;        // blocks of a row of blocks
  float* part;       // kDwd, kDwgu: sums of the slabs (one slab: null)
  int slabs;
};

// -------------------------------------------------------------- loads ----
// One direct load of 16 bytes a lane through a buffer descriptor: zeros beyond its end.
SC_DEV void lds_dma16_buf(u32x4 rsrc, unsigned voff, unsigned lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds"
               :
               : "v"(voff), "s"(rsrc), "s"(__builtin_amdgcn_readfirstlane((int)lds))
               : "memory", "m0");
}
constexpr unsigned kBeyond = 0xfffff000u;  // an offset beyond every descriptor's end

// A descriptor of `bytes` from p + skip on (skip <= bytes), in scalar registers.
SC_DEV u32x4 descriptor(const char* p, unsigned bytes, unsigned skip) {
  const unsigned long long at = uniform64((unsigned long long)(size_t)p + skip);
  return u32x4{(unsigned)at, (unsigned)(at >> 32), (unsigned)__builtin_amdgcn_readfirstlane((int)(bytes - skip)),
               0x00027000u};
}

// Contraction along the rows: 128 bytes a row and stage, 16-byte units swizzled by bits
// 1-3 of the row; lane l reads unit l / 16 of row l % 16.
SC_DEV int row_off(int row, int unit) { return row * 128 + 16 * (unit ^ ((row >> 1) & 7)); }

// Contraction across the rows: 64 rows of kUnits 16-byte units.  A transposing read
// touches, in 32 lanes, rows 0-3 and 8-11 and two units of each; the order of the units
// spreads these over all banks.
template <int kUnits>
SC_DEV int col_swz(int k) {
  if constexpr (kUnits >= 16) return 2 * (k & 3) | (k & 8);
  else if constexpr (kUnits == 8) return (k & 2) | ((k & 8) >> 1);
  else return (k & 8) >> 2;
}

// An operand's part of a stage: kSpan rows of 64 (kAcross: 64 rows of kSpan), a wave's
// share of the loads and its fragments.  kSubs: the operand is that many matrices side by
// side, kSpan / kSubs columns of each.
template <bool kAcross, int kSpan, int kWave, int kSubs>
struct FfnPart {
  static constexpr int kLoads = kSpan / 64, kBytes = kSpan * 128;
  static constexpr int kCols = kSpan / kSubs, kUnits = kCols / 8, kPitch = 2 * kCols;
  static constexpr int kFrags = kWave / 16, kSubFrags = kFrags / kSubs;
  static constexpr int kSubLoads = kSpan / 8 / kSubs;  // of the eight waves, a matrix
  unsigned voff[kLoads];
  unsigned fa;   // address of the first fragment in the part

  // Which load (of a matrix) a wave's t-th is, and of which matrix.
  static SC_DEV int load_sub(int w, int t) { return kSubs == 1 ? 0 : (8 * t + w) / kSubLoads; }
  static SC_DEV int load_at(int w, int t) { return kAcross ? (8 * t + w) % kSubLoads : kLoads * w + t; }

  SC_DEV void init(int lane, int wave_at) {  // wave_at: the wave's first row or column (of a matrix)
    const int g = lane >> 4;
    if constexpr (!kAcross) {
      fa = row_off(wave_at + (lane & 15), g);
    } else {
      const int r = (lane >> 2) & 3, k = 8 * g + r, u = wave_at / 8 + ((lane & 3) >> 1);
      fa = k * kPitch + 16 * (u ^ col_swz<kUnits>(k)) + 8 * (lane & 1);
    }
  }
  // Offsets of a tile whose first row or column is `first`; row(i): bytes to its i-th row.
  template <typename Row>
  SC_DEV void offsets(int lane, int w, int first, unsigned ld, Row row) {
#pragma unroll
    for (int t = 0; t < kLoads; ++t) {
      if constexpr (!kAcross) {
        const int r = 8 * load_at(w, t) + (lane >> 3);
        voff[t] = row(first + r) + 16u * ((lane & 7) ^ ((r >> 1) & 7));
      } else {
        const int k = load_at(w, t) * (64 / kUnits) + lane / kUnits;
        voff[t] = (unsigned)k * ld + 2u * first + 16u * ((lane % kUnits) ^ col_swz<kUnits>(k));
      }
    }
  }
  // kAlong with a contraction that ends inside the stage: units from `limit` on are zeros.
  SC_DEV void issue_one(int t, const u32x4 (&rsrc)[kSubs], unsigned lds, int w, int limit) const {
    const int sub = load_sub(w, t);
    u32x4 d = rsrc[0];
    if constexpr (kSubs == 2) d = sub ? rsrc[1] : rsrc[0];
    const unsigned to = lds + (unsigned)(sub * 128 * kCols + load_at(w, t) * 1024);
    if (!kAcross && limit < 8) {
      const int lane = opaque_lane();
      const int r = 8 * load_at(w, t) + (lane >> 3), unit = (lane & 7) ^ ((r >> 1) & 7);
      lds_dma16_buf(d, unit < limit ? voff[t] : kBeyond, to);
    } else {
      lds_dma16_buf(d, voff[t], to);
    }
  }
  // Fragment i of chunk c (32 of the stage's 64) of the part at LDS address `lds`.
  SC_DEV bf16x8 frag(unsigned lds, int i, int c) const {
    if constexpr (!kAcross) {
      return lds_read16(((fa ^ (64u * c)) + lds) + i * 2048);
    } else {
      const int sub = i / kSubFrags, j = i % kSubFrags;
      const unsigned at = lds + (fa ^ (32u * j)) + sub * 128 * kCols + c * 32 * kPitch;
      const i16x4 lo = lds_read_tr16(at), hi = lds_read_tr16(at + 4 * kPitch);
      return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
  }
};

// ------------------------------------------------------------ results ----
// Float32 rounded to 24 bits (the nearest, halves away from 0: 2^-16 of a value at most, where
// a cut would take up to 2^-15 off every one), four values in three words, and back.  Infinities
// stay, and so do NaNs: bf16's and the hardware's own have no low bits that could carry.
SC_DEV void pack24(const f32x4& v, unsigned* w) {
  const u32x4 u = __builtin_bit_cast(u32x4, v) + 0x80u;
  w[0] = __builtin_amdgcn_perm(u[1], u[0], 0x05030201u);
  w[1] = __builtin_amdgcn_perm(u[2], u[1], 0x06050302u);
  w[2] = __builtin_amdgcn_perm(u[3], u[2], 0x07060503u);
}
SC_DEV f32x4 unpack24(const unsigned* w) {
  const u32x4 u = {w[0] << 8, __builtin_amdgcn_perm(w[1], w[0], 0x0504030cu),
                   __builtin_amdgcn_perm(w[2], w[1], 0x0403020cu), w[2] & 0xffffff00u};
  return __builtin_bit_cast(f32x4, u);
}
// What the backward needs of g and u, its two factors of dh: u act'(g) and act(g), made
// where the exponential is at hand (from g and u themselves the backward's results took 34
// of a tile's 64 us).  Blocks of 16 rows by 32 columns, of a block a lane's twelve words
// (both factors of its columns 4 g on, both of columns 16 + 4 g on) in three planes of 16
// bytes a lane, so that whole lines move.
constexpr int kBlockBytes = 3 * 1024;
SC_DEV char* block_at(char* blocks, int across, int ri, int cb, int lane) {
  return blocks + ((long long)ri * across + cb) * kBlockBytes + 16 * lane;
}
SC_DEV void store_block(char* at, const unsigned (&w)[12]) {
#pragma unroll
  for (int p = 0; p < 3; ++p)
    *reinterpret_cast<u32x4*>(at + 1024 * p) = u32x4{w[4 * p], w[4 * p + 1], w[4 * p + 2], w[4 * p + 3]};
}
// Six words of one half of a block.
SC_DEV void store_half_block(char* at, int half, const unsigned (&w)[6]) {
  if (half == 0) {
    *reinterpret_cast<u32x4*>(at) = u32x4{w[0], w[1], w[2], w[3]};
    *reinterpret_cast<u32x2*>(at + 1024) = u32x2{w[4], w[5]};
  } else {
    *reinterpret_cast<u32x2*>(at + 1024 + 8) = u32x2{w[0], w[1]};
    *reinterpret_cast<u32x4*>(at + 2048) = u32x4{w[2], w[3], w[4], w[5]};
  }
}

// Up to kCount bf16 values of a row from column col on, those below N, at any address.
template <int kCount>
SC_DEV void store_row(__bf16* row, int col, int N, const unsigned (&v)[kCount / 2]) {
  if (col + kCount <= N) {
    if constexpr (kCount == 8) *reinterpret_cast<u32x4_any*>(row + col) = u32x4_any{v[0], v[1], v[2], v[3]};
    else *reinterpret_cast<u32x2_any*>(row + col) = u32x2_any{v[0], v[1]};
  } else {
#pragma unroll
    for (int q = 0; q < kCount - 1; ++q)
      if (col + q < N) row[col + q] = __builtin_bit_cast(__bf16, (unsigned short)(v[q / 2] >> (16 * (q & 1))));
  }
}
// Two fragments of 16 columns from column c on: a lane holds columns 4 g to 4 g + 3 of
// each; exchanged between neighbouring groups, 8 of one.
struct Pair {
  unsigned v[4];
  SC_DEV void set(const f32x4& a, const f32x4& b) {
    const auto lo = __builtin_amdgcn_permlane16_swap(pack_bf16(a[0], a[1]), pack_bf16(b[0], b[1]), false, false);
    const auto hi = __builtin_amdgcn_permlane16_swap(pack_bf16(a[2], a[3]), pack_bf16(b[2], b[3]), false, false);
    v[0] = (unsigned)lo[0];
    v[1] = (unsigned)hi[0];
    v[2] = (unsigned)lo[1];
    v[3] = (unsigned)hi[1];
  }
  SC_DEV void store(__bf16* row, int c, int N, int g) const {
    store_row<8>(row, c + 16 * (g & 1) + 8 * (g >> 1), N, v);
  }
};
SC_DEV void store_pair(__bf16* row, int c, int N, int g, const f32x4& a, const f32x4& b, bool on) {
  Pair p;
  p.set(a, b);
  if (on) p.store(row, c, N, g);
}
SC_DEV void store_one(__bf16* row, int c, int N, int g, const f32x4& a, bool on) {
  const unsigned v[2] = {pack_bf16(a[0], a[1]), pack_bf16(a[2], a[3])};
  if (on) store_row<4>(row, c + 4 * g, N, v);
}

// --------------------------------------------------------------- tile ----
template <int kKind, int kM, int kAct>
struct FfnProduct {
  using S = FfnTile<kM>;
  static constexpr int BM = S::kBM, BN = S::kBN, kNBuf = S::kNBuf;
  static constexpr int WM = BM / S::kWgM, WN = BN / S::kWgN, FI = WM / 16, FJ = WN / 16;
  static constexpr bool kIsGate = kKind == kGate || kKind == kGateKeep;
  static constexpr bool kOverRows = kKind == kDwd || kKind == kDwgu;  // contraction over the batch's rows
  static constexpr bool kAcrossA = kOverRows, kAcrossB = kOverRows || kIsGate || kKind == kDown;
  static constexpr int kSubs = kIsGate ? 2 : 1;
  static constexpr int kH = FI >= 2 ? 2 : 1, FH = FI / kH;  // a wave's rows go in halves
  using A = FfnPart<kAcrossA, BM, WM, 1>;
  using B = FfnPart<kAcrossB, BN, WN, kSubs>;
  static constexpr int kStage = A::kBytes + B::kBytes, kDma = A::kLoads + B::kLoads;

  const FfnArgs& p;
  const int R, lane, w, g, lr, wm, wn;
  const unsigned lds0;
  A a;
  B b;
  f32x4 acc[FI][FJ];
  bf16x8 xf[2][FH], wf[2][FJ];
  // the tile
  struct Tile {
    int m0, n0, sel, slab;  // sel: of two outputs
  };
  int m0, n0, sel, slab, k0, ns, seg;  // k0: first stage; ns: stages, of which a segment has seg
  const char *pa[2], *pb[2];
  unsigned bytes_a, bytes_b;

  SC_DEV FfnProduct(const FfnArgs& args, char* stage, int rows)
      : p(args), R(rows), lane(threadIdx.x & 63), w(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)), g(lane >> 4),
        lr(lane & 15), wm(w / S::kWgN * WM), wn(w % S::kWgN * (WN / kSubs)), lds0(lds_addr(stage)) {
    a.init(lane, wm);
    b.init(lane, wn);
    const bool whole = R == p.T;
    pa[0] = !whole && p.a.packed ? p.a.packed : p.a.p[0];
    pb[0] = !whole && p.b.packed ? p.b.packed : p.b.p[0];
    pa[1] = p.a.p[1];
    pb[1] = p.b.p[1];
    bytes_a = (unsigned)(p.a.rows ? p.a.rows : R) * p.a.ld;
    bytes_b = (unsigned)(p.b.rows ? p.b.rows : R) * p.b.ld;
  }
  SC_DEV int rows() const { return kOverRows ? p.M : R; }
  SC_DEV int tiles_n() const {
    constexpr int bn = BN / kSubs;
    return (p.N + bn - 1) / bn * (both() ? 2 : 1);
  }
  SC_DEV bool both() const { return kKind == kDwgu && p.out[0] && p.out[1]; }
  // Tiles in groups of kGroupTiles row tiles by all column tiles.
  SC_DEV void place(long long item) {
    const int T = (rows() + BM - 1) / BM, Nt = tiles_n();
    slab = kOverRows ? __builtin_amdgcn_readfirstlane((int)(item / ((long long)T * Nt))) : 0;
    const int it = __builtin_amdgcn_readfirstlane((int)(item - (long long)slab * T * Nt));
    const int per = kGroupTiles * Nt, gi = it / per, rem = it - gi * per, gs = min(kGroupTiles, T - gi * kGroupTiles);
    m0 = (gi * kGroupTiles + rem % gs) * BM;
    int nt = rem / gs;
    sel = 0;
    if constexpr (kKind == kDwgu) {
      sel = both() ? nt >= Nt / 2 : p.out[0] == nullptr;
      if (both() && sel) nt -= Nt / 2;
    }
    n0 = nt * (BN / kSubs);
    if constexpr (kOverRows) {
      const int all = (R + 63) / 64;
      k0 = (int)((long long)all * slab / p.slabs);
      ns = (int)((long long)all * (slab + 1) / p.slabs) - k0;
      seg = ns;
    } else {
      k0 = 0;
      seg = (p.K + 63) / 64;
      ns = kKind == kDx ? 2 * seg : seg;
    }
    m0 = __builtin_amdgcn_readfirstlane(m0);
    n0 = __builtin_amdgcn_readfirstlane(n0);
    const int M = rows(), N = p.N, lane = opaque_lane();
    const bool mapped = p.map_a && R != p.T;
    a.offsets(lane, w, m0, p.a.ld, [&](int r) {
      int row = min(r, M - 1);
      if (mapped) row = p.map[row];
      return (unsigned)row * p.a.ld;
    });
    b.offsets(lane, w, n0, p.b.ld, [&](int r) { return (unsigned)min(r, N - 1) * p.b.ld; });
  }
  // A stage's loads, to be issued one by one; zeros past the tile's last stage, so that the
  // number in flight is always the same.
  struct Load {
    u32x4 ra[1], rb[kSubs];
    unsigned at;
    int limit;
  };
  SC_DEV Load stage_load(int s, int bf) const {
    Load l;
    l.at = lds0 + (unsigned)bf * kStage;
    const bool live = s < ns;
    const int second = kKind == kDx && s >= seg, ks = live ? k0 + (second ? s - seg : s) : 0;
    l.limit = kOverRows || ks < seg - 1 ? 8 : (p.K - 64 * ks + 7) / 8;  // units of the stage (operands along the rows)
    const unsigned skip_a = kAcrossA ? (unsigned)ks * 64 * p.a.ld : (unsigned)ks * 128;
    const unsigned skip_b = kAcrossB ? (unsigned)ks * 64 * p.b.ld : (unsigned)ks * 128;
    const unsigned na = live ? bytes_a : skip_a, nb = live ? bytes_b : skip_b;
    l.ra[0] = descriptor(second ? pa[1] : pa[0], na, skip_a);
    l.rb[0] = descriptor((kKind == kDwgu ? sel : second) ? pb[1] : pb[0], nb, skip_b);
    if constexpr (kSubs == 2) l.rb[1] = descriptor(pb[1], nb, skip_b);
    return l;
  }
  SC_DEV void issue_one(const Load& l, int t) const {
    if (t < A::kLoads) a.issue_one(t, l.ra, l.at, w, l.limit);
    else b.issue_one(t - A::kLoads, l.rb, l.at + A::kBytes, w, l.limit);
  }
  SC_DEV void cols(int q, int bf, int c) {
    const unsigned at = lds0 + (unsigned)bf * kStage + A::kBytes;
#pragma unroll
    for (int j = 0; j < FJ; ++j) wf[q][j] = b.frag(at, j, c);
  }
  SC_DEV void rows(int q, int bf, int c, int h) {
    const unsigned at = lds0 + (unsigned)bf * kStage;
#pragma unroll
    for (int i = 0; i < FH; ++i) xf[q][i] = a.frag(at, h * FH + i, c);
    __builtin_amdgcn_sched_barrier(0);
  }
  // A half's products; between(i) after the i-th of its FH rows of fragments.
  template <typename F>
  SC_DEV void mul(int h, int qx, int qw, F between) {
#pragma unroll
    for (int i = 0; i < FH; ++i) {
#pragma unroll
      for (int j = 0; j < FJ; ++j)
        acc[h * FH + i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf[qw][j], xf[qx][i], acc[h * FH + i][j], 0, 0, 0);
      between(i);
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  SC_DEV void mul(int h, int qx, int qw) {
    mul(h, qx, qw, [](int) {});
  }
  static SC_DEV int next_buf(int bf) { return bf == kNBuf - 1 ? 0 : bf + 1; }

  // Stores that every wave issues for a tile without an edge.  While the last tile's are
  // under way, newer than the stages that start() loaded, a stage is waited for past them.
  // A count above what was issued would let a stage be read before it has landed; below, it
  // only waits longer.
  static constexpr int kStores = kKind == kGateKeep ? FI * (FJ == 2 ? 3 : 4)
                                 : kKind == kGate   ? FI
                                 : kKind == kDh     ? FI * FJ
                                                    : FI * FJ / 2;
  static constexpr int kMost(int n) { return n < 63 ? n : 63; }  // the counter's end
  SC_DEV bool whole(const Tile& t) const { return t.m0 + BM <= rows() && t.n0 + BN / kSubs <= p.N; }
  // The tile's sums.  Every half's fragments are in flight during the products of the one
  // before, across stages too; one barrier a stage, before its last products: the next
  // stage has landed, and every wave holds its last fragments of this one, whose buffer is
  // refilled.
  SC_DEV void sums(bool stored) {
#pragma unroll
    for (int i = 0; i < FI; ++i)
#pragma unroll
      for (int j = 0; j < FJ; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (kOverRows && ns == 0) return;
    if (stored)
      wait_vm<kMost((kNBuf - 1) * kDma + kStores)>();
    else
      wait_vm<(kNBuf - 1) * kDma>();
    __syncthreads();
    int bf = 0;
    cols(0, 0, 0);
    rows(0, 0, 0, 0);
    for (int s = 0; s + 1 < ns; ++s) {
      const int bn = next_buf(bf);
#pragma unroll
      for (int q = 0; q + 1 < 2 * kH; ++q) half(q, bf);
      if (stored && s + 1 < kNBuf)
        wait_vm<kMost((kNBuf - 2) * kDma + kStores)>();
      else
        wait_vm<(kNBuf - 2) * kDma>();
      __syncthreads();
      cols(0, bn, 0);
      rows(0, bn, 0, 0);
      // The refill's loads go out among the products (all at once behind the barrier, the
      // matrix units wait for them: dWg, dWu of 32768 x 1024 x 2816 386 us instead of 365;
      // over all halves of the next stage, they land too late: 408).
      const Load next = stage_load(s + kNBuf, bf);
      mul((2 * kH - 1) % kH, 1, 1, [&](int i) {
#pragma unroll
        for (int t = i * kDma / FH; t < (i + 1) * kDma / FH; ++t) issue_one(next, t);
        __builtin_amdgcn_sched_barrier(0);
      });
      bf = bn;
    }
    // the last stage by itself: joined with the others, its products would wait for
    // fragments that the loop has just asked for
#pragma unroll
    for (int q = 0; q + 1 < 2 * kH; ++q) half(q, bf);
    mul((2 * kH - 1) % kH, 1, 1);
  }
  // Half q of a stage (of 2 kH, the last one apart), and the fragments of the next one.
  SC_DEV void half(int q, int bf) {
    if (q + 1 == kH) cols(1, bf, 1);
    rows((q + 1) & 1, bf, (q + 1) / kH, (q + 1) % kH);
    mul(q % kH, q & 1, q / kH);
  }
  SC_DEV void start() {
#pragma unroll
    for (int s = 0; s < kNBuf; ++s) {
      const Load l = stage_load(s, s);
#pragma unroll
      for (int t = 0; t < kDma; ++t) issue_one(l, t);
    }
  }

  SC_DEV Tile tile() const { return {m0, n0, sel, slab}; }
  // Element e of a lane: row 16 i + lr, column 16 j + 4 g + e.
  SC_DEV void emit_h(const Tile& t, int i, int lane) const {
    constexpr int J = FJ / 2;
    const int g = lane >> 4, lr = lane & 15;
    const int r0 = t.m0 + wm + 16 * i, r = r0 + lr, c = t.n0 + wn;
    const bool on = r < R, keep = kKind == kGateKeep && r0 < R && c < 32 * p.across;
    __bf16* row = static_cast<__bf16*>(p.out[0]) + (long long)r * p.ld;
    f32x4 h[J];
    unsigned w[6 * J];
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const f32x4 gt = acc[i][j], up = acc[i][J + j];
      if constexpr (kKind == kGateKeep) {
        f32x4 fg, fu;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float slope;
          fu[e] = act_slope<kAct>(gt[e], slope);
          fg[e] = up[e] * slope;
          h[j][e] = fu[e] * up[e];
        }
        pack24(fg, w + 6 * j);
        pack24(fu, w + 6 * j + 3);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) h[j][e] = act<kAct>(gt[e]) * up[e];
      }
    }
    char* at = block_at(p.blocks, p.across, r0 / 16, c / 32, lane);
    if constexpr (J == 1) {
      if (keep) store_half_block(at, c / 16 & 1, w);
      store_one(row, c, p.N, g, h[0], on);
    } else {
      static_assert(J == 2, "a block a wave and 16 rows");
      if (keep) store_block(at, w);
      store_pair(row, c, p.N, g, h[0], h[1], on);
    }
  }
  // The words of block j (of the wave's FJ / 2) of rows i.
  SC_DEV void load_block(const Tile& t, int i, int j, int lane, unsigned (&w)[12]) const {
    const int r0 = t.m0 + wm + 16 * i, c = t.n0 + wn + 32 * j;
    if (r0 < R && c < 32 * p.across) {
      const char* at = block_at(p.blocks, p.across, r0 / 16, c / 32, lane);
#pragma unroll
      for (int q = 0; q < 3; ++q) {
        const u32x4 v = *reinterpret_cast<const u32x4*>(at + 1024 * q);
#pragma unroll
        for (int e = 0; e < 4; ++e) w[4 * q + e] = v[e];
      }
    } else {
#pragma unroll
      for (int q = 0; q < 12; ++q) w[q] = 0;
    }
  }
  SC_DEV void make_dh(int i, int j, const unsigned (&w)[12], Pair& dg, Pair& du) const {
    f32x4 vg[2], vu[2];
#pragma unroll
    for (int f = 0; f < 2; ++f) {
      const f32x4 fg = unpack24(w + 6 * f), fu = unpack24(w + 6 * f + 3);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        vg[f][e] = acc[i][2 * j + f][e] * fg[e];
        vu[f][e] = acc[i][2 * j + f][e] * fu[e];
      }
    }
    dg.set(vg[0], vg[1]);
    du.set(vu[0], vu[1]);
  }
  SC_DEV void emit_rows(const Tile& t, int i, int lane) const {  // kDown, kDx, kDwd, kDwgu
    const int g = lane >> 4, lr = lane & 15;
    const int r = t.m0 + wm + 16 * i + lr, c = t.n0 + wn;
    const bool on = r < rows();
    if constexpr (kOverRows) {
      if (p.part) {
        float* part = p.part + ((long long)t.sel * p.slabs + t.slab) * p.M * p.N + (long long)r * p.N;
#pragma unroll
        for (int j = 0; j < FJ; ++j) {
          const int col = c + 16 * j + 4 * g;
          if (!on) continue;
          if (col + 4 <= p.N) {
            *reinterpret_cast<f32x4_any*>(part + col) = acc[i][j];
          } else {
#pragma unroll
            for (int e = 0; e < 3; ++e)
              if (col + e < p.N) part[col + e] = acc[i][j][e];
          }
        }
        return;
      }
    }
    long long at = r;
    if (!kOverRows && p.map && R != p.T && on) at = p.map[r];
    __bf16* row = static_cast<__bf16*>(t.sel ? p.out[1] : p.out[0]) + at * p.ld;
#pragma unroll
    for (int j = 0; j < FJ; j += 2) store_pair(row, c + 16 * j, p.N, g, acc[i][j], acc[i][j + 1], on);
  }
  SC_DEV void results(const Tile& t) const {
    const int lane = opaque_lane();
    if constexpr (kKind == kDh) {
      // Units of 16 rows by 32 columns, the factors of kAhead of them in flight.  Loads and
      // stores retire in order, so a load behind a store waits for it: all factors come
      // first, the results in the place of the sums, then all stores (mixed, 358 us for
      // 32768 x 2816 x 1024, 225 without the loads and 250 without the stores).
      constexpr int kJ = FJ / 2, kUnits = FI * kJ, kAhead = kUnits < 4 ? kUnits : 4;
      unsigned w[kAhead][12];
      Pair dg[kUnits], du[kUnits];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) load_block(t, u / kJ, u % kJ, lane, w[u]);
#pragma unroll
      for (int u = 0; u < kUnits; ++u) {
        __builtin_amdgcn_sched_barrier(0);
        make_dh(u / kJ, u % kJ, w[u % kAhead], dg[u], du[u]);
        if (u + kAhead < kUnits) load_block(t, (u + kAhead) / kJ, (u + kAhead) % kJ, lane, w[u % kAhead]);
      }
      const int g = lane >> 4, lr = lane & 15;
#pragma unroll
      for (int u = 0; u < kUnits; ++u) {
        __builtin_amdgcn_sched_barrier(0);
        const int r = t.m0 + wm + 16 * (u / kJ) + lr, c = t.n0 + wn + 32 * (u % kJ);
        if (r >= R) continue;
        dg[u].store(static_cast<__bf16*>(p.out[0]) + (long long)r * p.ld, c, p.N, g);
        du[u].store(static_cast<__bf16*>(p.out[1]) + (long long)r * p.ld, c, p.N, g);
      }
    } else {
#pragma unroll
      for (int i = 0; i < FI; ++i) {
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (kIsGate) emit_h(t, i, lane);
        else emit_rows(t, i, lane);
      }
    }
  }
};

// A workgroup's tiles: `it` and what next() gives, until it is `last` or more.
template <int kKind, int kM, int kAct, typename Next>
SC_DEV void ffn_tiles(const FfnArgs& a, char* stage, int R, long long it, long long last, Next next) {
  if (it >= last) return;
  FfnProduct<kKind, kM, kAct> p(a, stage, R);
  p.place(it);
  p.start();
  bool stored = false;
  while (true) {
    p.sums(stored);
    const auto t = p.tile();
    it = next(it);
    const bool more = it < last;
    if (more) {  // the next tile's first stages are loaded during this one's results
      p.place(it);
      __syncthreads();  // every wave has read the last stage
      p.start();
    }
    p.results(t);
    if (!more) break;
    stored = p.whole(t);
  }
  wait_vm<0>();  // no load may land after the memory has gone to another
}
// The tiles go to the XCDs in contiguous ranges (workgroup i runs on XCD i % 8): what an XCD
// runs at a time shares rows and weights in its L2.
struct FfnShare {
  long long first, last;
  SC_DEV explicit FfnShare(long long items)
      : first(items * (blockIdx.x & 7) / 8), last(items * ((blockIdx.x & 7) + 1) / 8) {}
};
template <int kKind, int kM>
SC_DEV long long ffn_items(const FfnArgs& a, int R) {
  using S = FfnTile<kM>;
  constexpr bool over = kKind == kDwd || kKind == kDwgu, gate = kKind == kGate || kKind == kGateKeep;
  constexpr int bn = S::kBN / (gate ? 2 : 1);
  const int rows = over ? a.M : R;
  return (long long)((rows + S::kBM - 1) / S::kBM) * ((a.N + bn - 1) / bn) * (over ? a.slabs : 1) *
         (kKind == kDwgu && a.out[0] && a.out[1] ? 2 : 1);
}
SC_DEV int ffn_rows_of(const FfnArgs& a) { return a.count ? __builtin_amdgcn_readfirstlane(a.count[0]) : a.T; }

template <int kKind, int kM, int kAct>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2))) void k_ffn(FfnArgs a) {
  using P = FfnProduct<kKind, kM, kAct>;
  __shared__ __attribute__((aligned(1024))) char stage[P::kNBuf * P::kStage];
  const int R = ffn_rows_of(a), step = gridDim.x >> 3;
  const FfnShare share(ffn_items<kKind, kM>(a, R));
  ffn_tiles<kKind, kM, kAct>(a, stage, R, share.first + (blockIdx.x >> 3), share.last,
                             [=](long long it) { return it + step; });
}

// Two products that do not wait for each other in one launch: kSum over the batch's rows, in
// slabs as long as about `ratio` tiles of kRow.  Every workgroup of an XCD takes its share of
// the slabs; those that are left over go to the first workgroups, and the others take `ratio`
// tiles of kRow for each.  Every second workgroup begins with its tiles of kRow, so that the
// results of some are written during the products of others.
//
// With 256 x 256 tiles the state of both products is more than a lane's 256 registers: 9 (dh
// with dWd) and 8 (dx with dWg, dWu) of them lie in scratch, and their reloads wait for loads
// and stores in flight; the four products apart have none there.  The medians of 20, joined
// and apart, are still even or better joined: 32768 rows of 1024 x 2816, 480 us and 345 + 165,
// 657 and 307 + 348; 16384 of 768 x 2048, 176 and 117 + 57, 205 and 109 + 97.
template <int kRow, int kSum, int kM>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2))) void k_ffn_two(FfnArgs a, FfnArgs b, int ratio) {
  using P = FfnProduct<kRow, kM, kActNone>;
  using Q = FfnProduct<kSum, kM, kActNone>;
  static_assert(P::kNBuf * P::kStage == Q::kNBuf * Q::kStage, "one memory for both");
  __shared__ __attribute__((aligned(1024))) char stage[P::kNBuf * P::kStage];
  const int R = ffn_rows_of(a), wgs = gridDim.x >> 3, j = blockIdx.x >> 3;
  const FfnShare row(ffn_items<kRow, kM>(a, R)), sum(ffn_items<kSum, kM>(b, R));
  const int left = (int)((sum.last - sum.first) % wgs), others = wgs - left;
  const long long edge = left ? row.first + (long long)ratio * others : row.first;
  const bool before = left && j >= left;
  for (int turn = 0; turn < 2; ++turn) {
    if ((turn + j) & 1) {
      ffn_tiles<kRow, kM, kActNone>(a, stage, R, before ? row.first + j - left : edge + j, row.last,
                                    [=](long long it) {
                                      if (it >= edge) return it + wgs;
                                      return it + others < edge ? it + others : edge + j;
                                    });
    } else {
      ffn_tiles<kSum, kM, kActNone>(b, stage, R, sum.first + j, sum.last, [=](long long it) { return it + wgs; });
    }
    __syncthreads();
  }
}

template <int kM>
constexpr int kFfnGrid = kM == 2 ? 2 * kFfnWgs : kFfnWgs;
template <int kKind, int kM, int kAct>
hipError_t run_ffn(const FfnArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((k_ffn<kKind, kM, kAct>), dim3(kFfnGrid<kM>), dim3(512), 0, s, a);
  return hipGetLastError();
}
template <int kRow, int kSum, int kM>
hipError_t run_ffn_two(const FfnArgs& a, const FfnArgs& b, int ratio, hipStream_t s) {
  hipLaunchKernelGGL((k_ffn_two<kRow, kSum, kM>), dim3(kFfnGrid<kM>), dim3(512), 0, s, a, b, ratio);
  return hipGetLastError();
}
// What a product costs with tiles of kind m, in ns: rounds of workgroups times the stages of
// a tile and what stands beside them (kDh reads and writes ten bytes for every result).  A CU
// holds two workgroups of 64 x 64 tiles, which take about twice as long together.  From
// launches of every kind, us with tiles of 256, 128 and 64: 2048 rows of 1024 x 2816, gate
// 35, 39, 56, down 65, 27, 25, dh 40, 30, 32, dx 122, 53, 54; 1504 of 504 x 1112, gate 20,
// 12, 18, down 31, 14, 8, dh 25, 14, 11, dx 57, 25, 17; 8192 of 1024 x 4096, gate 157, 263,
// 371, down 106, 102, 146, dh 132, 158, 184, dx 202, 209, 321.
inline long long ffn_fixed(int m, bool dh) {
  return m == 0 ? (dh ? 38000 : 9000) : m == 1 ? (dh ? 11000 : 4000) : (dh ? 3500 : 2500);
}
inline long long ffn_stage(int m, long long tiles) {
  return m == 0 ? (tiles > kFfnWgs / 2 ? 1750 : 1450) : m == 1 ? (tiles > kFfnWgs / 2 ? 700 : 570) : tiles > kFfnWgs ? 560 : 300;
}
inline long long ffn_at_once(int m, long long tiles) { return m == 2 && tiles > kFfnWgs ? 2 * kFfnWgs : kFfnWgs; }
inline long long ffn_tiles_of(int m, long long rows, long long cols) {
  const long long bm = m == 0 ? 256 : m == 1 ? 128 : 64;
  return (rows + bm - 1) / bm * ((cols + bm - 1) / bm);
}
inline long long ffn_cost(int m, long long rows, long long cols, long long stages, int slabs, bool dh) {
  const long long tiles = ffn_tiles_of(m, rows, cols) * slabs, at_once = ffn_at_once(m, tiles);
  return (tiles + at_once - 1) / at_once * ((stages + slabs - 1) / slabs * ffn_stage(m, tiles) + ffn_fixed(m, dh));
}
struct FfnPlan {
  int tile, slabs;
};
// most_slabs > 1: the contraction may be cut; each slab's sums are written and read again.
inline FfnPlan ffn_plan(long long rows, long long cols, long long stages, int most_slabs, bool dh = false) {
  FfnPlan best = {0, 1};
  long long least = 1LL << 62;
  for (int m = 0; m < 3; ++m)
    for (int s = 1; s <= most_slabs && (s == 1 || s * 4 <= stages); ++s) {
      const long long extra = s == 1 ? 0 : 4000 + rows * cols * s * 8 / 5000;  // a launch, and 5 TB/s
      const long long t = ffn_cost(m, rows, cols, stages, s, dh) + extra;
      if (t < least) {
        least = t;
        best = {m, s};
      }
    }
  return best;
}
// One product over rows and one in slabs, of plans of their own, as one launch with tiles of
// kind `tile`, or as two (-1).  Plans of one kind are joined; others where the tiles of a
// launch, dealt evenly with half of the longest at its end, cost less than both rounded up
// and a launch.  The whole backward in a graph, us, joined and not: 512 x 512 x 1536 36.7 and
// 40.7, 1504 x 504 x 1112 42 and 53, 1024 x 768 x 2304 58 and 67, 2048 x 1024 x 2816 126 and
// 146, 16384 x 768 x 2048 377 and 396; of two kinds joined as 256 x 256, 8192 x 768 x 2304
// 310 and 285.
struct FfnSize {
  long long rows, cols, stages;
  bool dh;
};
struct FfnTwoPlan {
  int tile, ratio;  // ratio: tiles of the first that take as long as one of the second
};
inline FfnTwoPlan ffn_plan_two(const FfnSize& a, const FfnPlan& pa, const FfnSize& b, const FfnPlan& pb) {
  const long long launch = 2000;
  long long least = ffn_cost(pa.tile, a.rows, a.cols, a.stages, 1, a.dh) +
                    ffn_cost(pb.tile, b.rows, b.cols, b.stages, pb.slabs, b.dh) + launch;
  FfnTwoPlan best = {-1, 1};
  const bool same = pa.tile == pb.tile;
  for (int m = same ? pa.tile : 1; m < (same ? pa.tile + 1 : 3); ++m) {
    const long long na = ffn_tiles_of(m, a.rows, a.cols), nb = ffn_tiles_of(m, b.rows, b.cols) * pb.slabs, n = na + nb;
    const long long ta = a.stages * ffn_stage(m, n) + ffn_fixed(m, a.dh),
                    tb = (b.stages + pb.slabs - 1) / pb.slabs * ffn_stage(m, n) + ffn_fixed(m, b.dh);
    const long long most = ta > tb ? ta : tb, at_once = ffn_at_once(m, n);
    const long long t = n <= at_once ? most : (na * ta + nb * tb) / at_once + most / 2;
    if (same || t < least) {
      least = t;
      const long long r = (tb + ta / 2) / ta;
      best = {m, (int)(r < 1 ? 1 : r > 1 << 20 ? 1 << 20 : r)};
    }
  }
  return best;
}
template <int kKind, int kAct>
hipError_t run_ffn(const FfnArgs& a, int tile, hipStream_t s) {
  if (tile == 0) return run_ffn<kKind, 0, kAct>(a, s);
  if (tile == 1) return run_ffn<kKind, 1, kAct>(a, s);
  return run_ffn<kKind, 2, kAct>(a, s);
}

template <int kRow, int kSum>
hipError_t run_ffn_two(const FfnArgs& a, const FfnArgs& b, int tile, int ratio, hipStream_t s) {
  if (tile == 0) return run_ffn_two<kRow, kSum, 0>(a, b, ratio, s);
  if (tile == 1) return run_ffn_two<kRow, kSum, 1>(a, b, ratio, s);
  return run_ffn_two<kRow, kSum, 2>(a, b, ratio, s);
}

// -------------------------------------------------------------- sizes ----
inline int up8(int v) { return (v + 7) / 8 * 8; }
// Widths that direct loads of 16 bytes cannot take: those tensors are copied to rows
// rounded up to 8, zeros behind.
inline bool ffn_odd(const Ffn& a) { return a.D % 8 != 0 || a.F % 8 != 0; }

struct FfnSaved {
  char* h;      // [valid rows, Fp] bf16
  char* blocks;  // the factors of dh
  size_t bytes;
};
inline FfnSaved ffn_saved(const Ffn& a, void* base) {
  const size_t T = (size_t)a.B * a.n, Fp = up8(a.F);
  FfnSaved s;
  s.h = static_cast<char*>(base);
  const size_t h = (T * Fp * 2 + 255) / 256 * 256;
  s.blocks = s.h + h;
  s.bytes = h + (T + 15) / 16 * ((Fp + 31) / 32) * kBlockBytes;
  return s;
}

struct FfnCarve {
  char* base;
  size_t off = 0;
  char* take(size_t bytes) {
    char* p = base ? base + off : nullptr;
    off += (bytes + 255) / 256 * 256;
    return p;
  }
};

// What stands before the products: the numbering of the valid rows, zeros into the
// padding rows of an output, and the copies.
struct FfnCopy {
  const char* src;
  char* dst;
  int rows, cols, pitch;  // elements; rows 0: the batch's valid rows
};
constexpr int kFfnCopies = 5;
struct FfnRows {
  const int* len;
  int B, n;
  int* map;    // null without lengths
  int* count;
  char* zero;  // rows of zero_bytes whose padding ones are zeroed, or null
  long long zero_bytes;
  int always;  // the batch's rows are copied even if none is padding
  int copies;
  FfnCopy copy[kFfnCopies];
};
}  // namespace

hipError_t launch_ffn_rows(const void* rows, hipStream_t s);  // an FfnRows

}  // namespace sc
