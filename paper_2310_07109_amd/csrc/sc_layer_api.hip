// C ABI of the layer operators (declared in include/sc_layer.h): argument
// validation on the host and launch sequencing on the caller's stream.
#include <cmath>
#include <cstring>

#include "../../include/sc_layer.h"
#include "sc_api_common.h"
#include "sc_internal.h"

namespace {

bool aligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }
bool float_type(int t) { return t == SC_F32 || t == SC_BF16; }

// A padded batch of rows.
sc_status check_rows(int B, int n) {
  if (B < 1 || n < 1) return SC_EINVAL;
  return (long long)B * n < (1LL << 31) ? SC_OK : SC_EUNSUPPORTED;
}

struct Span {
  const void* p;
  size_t n;
};
template <size_t N>
bool any_overlap(const Span& out, const Span (&others)[N]) {
  for (const Span& o : others)
    if (overlaps(out.p, out.n, o.p, o.n)) return true;
  return false;
}

// ------------------------------------------------------------- rotary ----
sc_status check_rotary(const sc_rotary_desc* d) {
  if (!d) return SC_EINVAL;
  if (d->Hq < 0 || d->Hk < 0 || d->d < 2 || d->d % 2 != 0) return SC_EINVAL;
  if (d->rot_dim < 0 || d->rot_dim > d->d || d->rot_dim % 2 != 0) return SC_EINVAL;
  if (d->layout != SC_ROTARY_HALF && d->layout != SC_ROTARY_INTERLEAVED) return SC_EINVAL;
  if (d->norm != 0 && d->norm != 1) return SC_EINVAL;
  if (d->norm && d->kind != SC_NORM_LAYER && d->kind != SC_NORM_RMS) return SC_EINVAL;
  if (d->norm && (!(d->eps > 0.f) || !std::isfinite(d->eps))) return SC_EINVAL;
  if (!std::isfinite(d->amplitude) || !float_type(d->dtype)) return SC_EINVAL;
  const sc_status st = check_rows(d->B, d->n);
  if (st != SC_OK) return st;
  if (d->d > sc::kRotaryMaxD) return SC_EUNSUPPORTED;
  return (long long)d->Hq + 2LL * d->Hk < (1LL << 15) ? SC_OK : SC_EUNSUPPORTED;
}

// Part i (q, k, v): its heads, its stride, and the bytes that its strided and dense
// tensors span.
struct RotaryPart {
  long long heads, stride;
  size_t strided, dense;
};
// SC_EINVAL for strides that are too short, of the parts present.
sc_status rotary_parts(const sc_rotary_desc* d, const bool (&present)[3], RotaryPart (&parts)[3]) {
  const int64_t strides[3] = {d->q_stride, d->k_stride, d->v_stride};
  const size_t e = elem_size(d->dtype), rows = (size_t)d->B * d->n;
  for (int i = 0; i < 3; ++i) {
    RotaryPart& p = parts[i];
    p.heads = i == 0 ? d->Hq : d->Hk;
    p.stride = strides[i];
    const long long row = p.heads * d->d;
    p.dense = rows * row * e;
    p.strided = 0;
    if (!present[i]) continue;
    if (p.heads < 1 || p.stride < row || p.stride > (1LL << 40)) return SC_EINVAL;
    p.strided = ((rows - 1) * (size_t)p.stride + row) * e;
  }
  return SC_OK;
}

// Whether a strided tensor meets `other`, of `no` bytes.
bool strided_overlap(const void* p, const RotaryPart& part, const void* other, size_t no) {
  return p && other && overlaps(p, part.strided, other, no);
}
// Whether two strided tensors do: parts of the same fused rows lie between one another
// without sharing an element.
bool strided_overlap(const sc_rotary_desc* d, const void* p, const RotaryPart& a, const void* q, const RotaryPart& b) {
  if (!p || !q || !overlaps(p, a.strided, q, b.strided)) return false;
  if (a.stride != b.stride) return true;
  const long long e = (long long)elem_size(d->dtype), row = a.stride * e, wa = a.heads * d->d * e,
                  wb = b.heads * d->d * e;
  long long off = (long long)(reinterpret_cast<uintptr_t>(q) - reinterpret_cast<uintptr_t>(p)) % row;
  if (off < 0) off += row;
  return off < wa || off + wb > row;  // b starts inside a row's part of a, or runs into the next one's
}

sc_status turns_of(const sc_rotary_desc* d, const double* freq, sc::RotaryTurns* t) {
  std::memset(t, 0, sizeof(*t));
  if (d->rot_dim > 0 && !freq) return SC_EINVAL;
  // f / (2 pi) as a sum of two doubles, its fraction in 2^-64 (long double arithmetic takes
  // 4 us of a call for 32 frequencies, this none to speak of).
  constexpr double inv = 0.15915494309189535, inv_low = -9.839338337591243e-18, one = 18446744073709551616.0;
  for (int i = 0; i < d->rot_dim / 2; ++i) {
    const double f = std::fabs(freq[i]), hi = f * inv;
    if (!(f < 1048576.0)) return SC_EINVAL;
    const double low = std::fma(f, inv, -hi) + f * inv_low;
    double x = (hi - std::floor(hi)) * one;
    const double whole = std::floor(x);
    x = (x - whole) + low * one;  // some 2^30 units of 2^-64 at most, signed
    const unsigned long long turn = (unsigned long long)whole + (unsigned long long)(long long)std::floor(x + 0.5);
    t->t[i] = freq[i] < 0.0 ? 0 - turn : turn;
  }
  return SC_OK;
}

sc::Rotary rotary_args(const sc_rotary_desc* d, const void* q, const void* k, const void* v, const float* q_w,
                       const float* k_w, const int32_t* positions) {
  sc::Rotary a;
  std::memset(&a, 0, sizeof(a));
  a.q = q;
  a.k = k;
  a.v = v;
  a.q_stride = d->q_stride;
  a.k_stride = d->k_stride;
  a.v_stride = d->v_stride;
  a.q_w = q_w;
  a.k_w = k_w;
  a.len = d->valid_len;
  a.pos = positions;
  a.B = d->B;
  a.n = d->n;
  a.Hq = d->Hq;
  a.Hk = d->Hk;
  a.d = d->d;
  a.R = d->rot_dim;
  a.interleaved = d->layout == SC_ROTARY_INTERLEAVED;
  a.norm = d->norm;
  a.rms = d->kind == SC_NORM_RMS;
  a.f32 = d->dtype == SC_F32;
  a.eps = d->eps;
  a.amplitude = d->amplitude;
  return a;
}

sc_status rotary_impl(const sc_rotary_desc* d, const double* freq, const void* q, const void* k, const void* v,
                      const float* q_w, const float* k_w, const int32_t* positions, void* q_out, void* k_out,
                      void* v_out, void* stream) {
  sc_status st = check_rotary(d);
  if (st != SC_OK) return st;
  const void* ins[3] = {q, k, v};
  void* outs[3] = {q_out, k_out, v_out};
  const bool present[3] = {q != nullptr, k != nullptr, v != nullptr};
  if (!q && !k && !v) return SC_EINVAL;
  for (int i = 0; i < 3; ++i)
    if ((outs[i] != nullptr) != present[i]) return SC_EINVAL;
  if (!d->norm && (q_w || k_w)) return SC_EINVAL;
  RotaryPart p[3];
  st = rotary_parts(d, present, p);
  if (st != SC_OK) return st;
  const size_t rows = (size_t)d->B * d->n, wb = 4 * (size_t)d->d;
  const Span small[] = {{q_w, wb}, {k_w, wb}, {positions, rows * 4}, {d->valid_len, 4 * (size_t)d->B}};
  for (int i = 0; i < 3; ++i) {
    const Span o{outs[i], p[i].dense};
    if (any_overlap(o, small)) return SC_EINVAL;
    for (int j = 0; j < 3; ++j) {
      const bool same = i == j && outs[i] == ins[j] && p[i].stride == p[i].heads * d->d;  // in place
      if (!same && strided_overlap(ins[j], p[j], outs[i], p[i].dense)) return SC_EINVAL;
      if (j < i && overlaps(outs[i], p[i].dense, outs[j], p[j].dense)) return SC_EINVAL;
    }
  }
  sc::Rotary a = rotary_args(d, q, k, v, q_w, k_w, positions);
  st = turns_of(d, freq, &a.turns);
  if (st != SC_OK) return st;
  a.oq = q_out;
  a.ok = k_out;
  a.ov = v_out;
  return sc::launch_rotary(a, static_cast<hipStream_t>(stream)) == hipSuccess ? SC_OK : SC_EHIP;
}

sc_status rotary_backward_impl(const sc_rotary_desc* d, const double* freq, const void* dq_out, const void* dk_out,
                               const void* dv_out, const void* q, const void* k, const float* q_w, const float* k_w,
                               const int32_t* positions, void* dq, void* dk, void* dv, float* dq_w, float* dk_w,
                               void* workspace, size_t ws_bytes, void* stream) {
  sc_status st = check_rotary(d);
  if (st != SC_OK) return st;
  const void* grads[3] = {dq_out, dk_out, dv_out};
  const void* ins[3] = {d->norm ? q : nullptr, d->norm ? k : nullptr, nullptr};
  void* outs[3] = {dq, dk, dv};
  const bool present[3] = {dq != nullptr, dk != nullptr, dv != nullptr};
  if (!dq && !dk && !dv) return SC_EINVAL;
  for (int i = 0; i < 3; ++i) {
    if ((grads[i] != nullptr) != present[i]) return SC_EINVAL;
    if (d->norm && i < 2 && present[i] && !ins[i]) return SC_EINVAL;
  }
  if (!d->norm && (q_w || k_w || dq_w || dk_w)) return SC_EINVAL;
  if ((dq_w && !dq) || (dk_w && !dk)) return SC_EINVAL;
  RotaryPart p[3];
  st = rotary_parts(d, present, p);
  if (st != SC_OK) return st;
  const size_t need = dq_w || dk_w ? sc_rotary_backward_workspace_size(d) : 0;
  if (need > 0 && (!workspace || ws_bytes < need)) return SC_EWORKSPACE;
  if (need > 0 && !aligned(workspace, 16)) return SC_EINVAL;
  const size_t rows = (size_t)d->B * d->n, wb = 4 * (size_t)d->d;
  const Span small[] = {{q_w, wb}, {k_w, wb}, {positions, rows * 4}, {d->valid_len, 4 * (size_t)d->B}};
  const Span sums[] = {{dq_w, wb}, {dk_w, wb}, {workspace, need}};
  for (int i = 0; i < 3; ++i) {
    if (any_overlap(sums[i], small)) return SC_EINVAL;
    for (int j = 0; j < i; ++j)
      if (overlaps(sums[i].p, sums[i].n, sums[j].p, sums[j].n)) return SC_EINVAL;
    for (int j = 0; j < 3; ++j)
      if (present[j] && (overlaps(sums[i].p, sums[i].n, grads[j], p[j].dense) ||
                         strided_overlap(ins[j], p[j], sums[i].p, sums[i].n) ||
                         strided_overlap(outs[j], p[j], sums[i].p, sums[i].n)))
        return SC_EINVAL;
  }
  for (int i = 0; i < 3; ++i) {
    if (!present[i]) continue;
    for (const Span& s : small)
      if (strided_overlap(outs[i], p[i], s.p, s.n)) return SC_EINVAL;
    for (int j = 0; j < 3; ++j) {
      if (!present[j]) continue;
      const bool same = i == j && outs[i] == grads[j] && p[i].stride == p[i].heads * d->d;  // in place
      if (!same && strided_overlap(outs[i], p[i], grads[j], p[j].dense)) return SC_EINVAL;
      if (ins[j] && strided_overlap(d, outs[i], p[i], ins[j], p[j])) return SC_EINVAL;
      if (j < i && strided_overlap(d, outs[i], p[i], outs[j], p[j])) return SC_EINVAL;
    }
  }
  sc::Rotary a = rotary_args(d, ins[0], ins[1], nullptr, q_w, k_w, positions);
  st = turns_of(d, freq, &a.turns);
  if (st != SC_OK) return st;
  a.gq = dq_out;
  a.gk = dk_out;
  a.gv = dv_out;
  a.oq = dq;
  a.ok = dk;
  a.ov = dv;
  a.dq_w = dq_w;
  a.dk_w = dk_w;
  a.ws = static_cast<float*>(workspace);
  return sc::launch_rotary_backward(a, static_cast<hipStream_t>(stream)) == hipSuccess ? SC_OK : SC_EHIP;
}

// ---------------------------------------------------------------- ffn ----
constexpr int kFfnMaxWidth = 1 << 20;  // 64 rows of a stage stay below 32-bit byte offsets
constexpr long long kFfnMaxBytes = (1LL << 32) - 4096;

sc_status check_ffn(const sc_ffn_desc* d) {
  if (!d) return SC_EINVAL;
  if (d->D < 1 || d->F < 1 || !float_type(d->dtype)) return SC_EINVAL;
  if (d->act != SC_ACT_NONE && d->act != SC_ACT_GELU && d->act != SC_ACT_SILU) return SC_EINVAL;
  const sc_status st = check_rows(d->B, d->n);
  if (st != SC_OK) return st;
  if (d->dtype != SC_BF16 || d->D > kFfnMaxWidth || d->F > kFfnMaxWidth) return SC_EUNSUPPORTED;
  if (d->valid_len && d->B > sc::kPackMaxB) return SC_EUNSUPPORTED;
  const long long T = (long long)d->B * d->n, D = (d->D + 7) / 8 * 8, F = (d->F + 7) / 8 * 8;
  if (2 * T * D >= kFfnMaxBytes || 2 * T * F >= kFfnMaxBytes || 2 * D * F >= kFfnMaxBytes) return SC_EUNSUPPORTED;
  return SC_OK;
}

sc::Ffn ffn_args(const sc_ffn_desc* d, const void* x, const void* wg, const void* wu, const void* wd, void* ws) {
  sc::Ffn a;
  std::memset(&a, 0, sizeof(a));
  a.x = x;
  a.wg = wg;
  a.wu = wu;
  a.wd = wd;
  a.ws = ws;
  a.len = d->valid_len;
  a.B = d->B;
  a.n = d->n;
  a.D = d->D;
  a.F = d->F;
  a.act = d->act;
  return a;
}

sc_status gated_ffn_impl(const sc_ffn_desc* d, const void* x, const void* wg, const void* wu, const void* wd, void* y,
                         void* saved, void* workspace, size_t ws_bytes, void* stream) {
  const sc_status st = check_ffn(d);
  if (st != SC_OK) return st;
  if (!x || !wg || !wu || !wd || !y) return SC_EINVAL;
  const size_t need = sc_gated_ffn_workspace_size(d, saved != nullptr);
  if (need > 0 && (!workspace || ws_bytes < need)) return SC_EWORKSPACE;
  const void* all[] = {x, wg, wu, wd, y, saved, need > 0 ? workspace : nullptr};
  for (const void* p : all)
    if (!aligned(p, 16)) return SC_EINVAL;
  const size_t rows = (size_t)d->B * d->n, xb = rows * d->D * 2, wb = (size_t)d->D * d->F * 2;
  const Span ins[] = {{x, xb}, {wg, wb}, {wu, wb}, {wd, wb}, {d->valid_len, 4 * (size_t)d->B}};
  const Span outs[] = {{y, xb}, {saved, sc_gated_ffn_saved_size(d)}, {workspace, need}};
  for (int i = 0; i < 3; ++i) {
    if (any_overlap(outs[i], ins)) return SC_EINVAL;
    for (int j = 0; j < i; ++j)
      if (overlaps(outs[i].p, outs[i].n, outs[j].p, outs[j].n)) return SC_EINVAL;
  }
  sc::Ffn a = ffn_args(d, x, wg, wu, wd, workspace);
  a.y = y;
  a.saved = saved;
  return sc::launch_ffn(a, static_cast<hipStream_t>(stream)) == hipSuccess ? SC_OK : SC_EHIP;
}

sc_status gated_ffn_backward_impl(const sc_ffn_desc* d, const void* x, const void* wg, const void* wu, const void* wd,
                                  const void* saved, const void* dy, void* dx, void* dwg, void* dwu, void* dwd,
                                  void* workspace, size_t ws_bytes, void* stream) {
  const sc_status st = check_ffn(d);
  if (st != SC_OK) return st;
  if (!x || !wg || !wu || !wd || !saved || !dy) return SC_EINVAL;
  if (!dx && !dwg && !dwu && !dwd) return SC_EINVAL;
  const size_t need = sc_gated_ffn_backward_workspace_size(d);
  if (!workspace || ws_bytes < need) return SC_EWORKSPACE;
  const void* all[] = {x, wg, wu, wd, saved, dy, dx, dwg, dwu, dwd, workspace};
  for (const void* p : all)
    if (!aligned(p, 16)) return SC_EINVAL;
  const size_t rows = (size_t)d->B * d->n, xb = rows * d->D * 2, wb = (size_t)d->D * d->F * 2;
  const Span ins[] = {{x, xb},  {wg, wb}, {wu, wb}, {wd, wb}, {saved, sc_gated_ffn_saved_size(d)},
                      {dy, xb}, {d->valid_len, 4 * (size_t)d->B}};
  const Span outs[] = {{dx, xb}, {dwg, wb}, {dwu, wb}, {dwd, wb}, {workspace, need}};
  for (int i = 0; i < 5; ++i) {
    if (any_overlap(outs[i], ins)) return SC_EINVAL;
    for (int j = 0; j < i; ++j)
      if (overlaps(outs[i].p, outs[i].n, outs[j].p, outs[j].n)) return SC_EINVAL;
  }
  sc::Ffn a = ffn_args(d, x, wg, wu, wd, workspace);
  a.saved = const_cast<void*>(saved);
  a.dy = dy;
  a.dx = dx;
  a.dwg = dwg;
  a.dwu = dwu;
  a.dwd = dwd;
  return sc::launch_ffn_backward(a, static_cast<hipStream_t>(stream)) == hipSuccess ? SC_OK : SC_EHIP;
}

// ------------------------------------------------------------ dropout ----
sc_status check_dropout(const sc_dropout_desc* d) {
  if (!d) return SC_EINVAL;
  if (d->D < 1 || !float_type(d->dtype) || !std::isfinite(d->res_scale)) return SC_EINVAL;
  if (!(d->p >= 0.0) || !(d->p * 65536.0 < 65535.5)) return SC_EINVAL;
  return check_rows(d->B, d->n);
}

sc_status dropout_impl(const sc_dropout_desc* d, const void* x, const int64_t* seed, const void* residual, void* out,
                       void* stream) {
  const sc_status st = check_dropout(d);
  if (st != SC_OK) return st;
  if (!x || !seed || !out || !aligned(seed, 8)) return SC_EINVAL;
  const size_t xb = (size_t)d->B * d->n * d->D * elem_size(d->dtype);
  if ((out != x && overlaps(out, xb, x, xb)) || (out != residual && overlaps(out, xb, residual, xb))) return SC_EINVAL;
  if (overlaps(out, xb, seed, 8) || overlaps(out, xb, d->valid_len, 4 * (size_t)d->B)) return SC_EINVAL;
  sc::Dropout a;
  std::memset(&a, 0, sizeof(a));
  a.x = x;
  a.residual = residual;
  a.out = out;
  a.seed = seed;
  a.len = d->valid_len;
  a.B = d->B;
  a.n = d->n;
  a.D = d->D;
  a.site = d->site;
  a.f32 = d->dtype == SC_F32;
  a.threshold = (unsigned)std::nearbyint(d->p * 65536.0);
  a.scale = (float)(65536.0 / (65536.0 - a.threshold));
  a.res_scale = d->res_scale;
  return sc::launch_dropout(a, static_cast<hipStream_t>(stream)) == hipSuccess ? SC_OK : SC_EHIP;
}

}  // namespace

#ifdef SC_DEBUG
namespace {
template <typename D>
sc_status debug_len(sc_status desc, const D* d, void* stream) {
  return desc == SC_OK && d->valid_len ? debug_rows(d->valid_len, nullptr, d->B, d->n, 0, stream) : SC_OK;
}
}  // namespace
#define SC_DEBUG_LEN(pre, stream, call) SC_DEBUG_RUN(pre, stream, call)
#else
#define SC_DEBUG_LEN(pre, stream, call) return call
#endif

extern "C" {

sc_status sc_rotary_frequencies(int32_t rot_dim, double base, int32_t scaling, double factor, double length,
                                double fast, double slow, double* freq, float* amplitude) {
  if (!freq || !amplitude || rot_dim < 2 || rot_dim % 2 != 0) return SC_EINVAL;
  if (!(base > 1.0) || !std::isfinite(base)) return SC_EINVAL;
  if (scaling < SC_ROTARY_PLAIN || scaling > SC_ROTARY_BANDS) return SC_EINVAL;
  if (scaling != SC_ROTARY_PLAIN && (!(factor >= 1.0) || !std::isfinite(factor))) return SC_EINVAL;
  if (scaling == SC_ROTARY_BANDS && (!(length >= 1.0) || !std::isfinite(length) || !(slow >= 0.0) || !(fast > slow) ||
                                     !std::isfinite(fast)))
    return SC_EINVAL;
  if (rot_dim > sc::kRotaryMaxD) return SC_EUNSUPPORTED;
  if (scaling == SC_ROTARY_BASE && rot_dim > 2) base *= std::pow(factor, rot_dim / (rot_dim - 2.0));
  *amplitude = scaling == SC_ROTARY_BANDS ? (float)(0.1 * std::log(factor) + 1.0) : 1.f;
  for (int i = 0; i < rot_dim / 2; ++i) {
    const double f = std::pow(base, -2.0 * i / rot_dim);
    freq[i] = f;
    if (scaling == SC_ROTARY_LINEAR) freq[i] = f / factor;
    if (scaling == SC_ROTARY_BANDS) {
      const double turns = f * length / 6.283185307179586476925286766559;
      double keep = (turns - slow) / (fast - slow);
      keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
      freq[i] = f * keep + f / factor * (1.0 - keep);
    }
  }
  return SC_OK;
}

sc_status sc_rotary(const sc_rotary_desc* d, const double* freq, const void* q, const void* k, const void* v,
                    const float* q_w, const float* k_w, const int32_t* positions, void* q_out, void* k_out,
                    void* v_out, void* stream) {
  SC_DEBUG_LEN(debug_len(check_rotary(d), d, stream), stream,
               rotary_impl(d, freq, q, k, v, q_w, k_w, positions, q_out, k_out, v_out, stream));
}

size_t sc_rotary_backward_workspace_size(const sc_rotary_desc* d) {
  if (check_rotary(d) != SC_OK || !d->norm) return 0;
  return sc::rotary_backward_floats((long long)d->B * d->n, d->d, d->Hq > d->Hk ? d->Hq : d->Hk) * sizeof(float);
}

sc_status sc_rotary_backward(const sc_rotary_desc* d, const double* freq, const void* dq_out, const void* dk_out,
                             const void* dv_out, const void* q, const void* k, const float* q_w, const float* k_w,
                             const int32_t* positions, void* dq, void* dk, void* dv, float* dq_w, float* dk_w,
                             void* workspace, size_t ws_bytes, void* stream) {
  SC_DEBUG_LEN(debug_len(check_rotary(d), d, stream), stream,
               rotary_backward_impl(d, freq, dq_out, dk_out, dv_out, q, k, q_w, k_w, positions, dq, dk, dv, dq_w, dk_w,
                                    workspace, ws_bytes, stream));
}

size_t sc_gated_ffn_workspace_size(const sc_ffn_desc* d, int32_t save) {
  return check_ffn(d) == SC_OK ? sc::ffn_workspace_bytes(ffn_args(d, nullptr, nullptr, nullptr, nullptr, nullptr), save != 0)
                               : 0;
}

size_t sc_gated_ffn_saved_size(const sc_ffn_desc* d) {
  return check_ffn(d) == SC_OK ? sc::ffn_saved_bytes(ffn_args(d, nullptr, nullptr, nullptr, nullptr, nullptr)) : 0;
}

sc_status sc_gated_ffn(const sc_ffn_desc* d, const void* x, const void* wg, const void* wu, const void* wd, void* y,
                       void* saved, void* workspace, size_t ws_bytes, void* stream) {
  SC_DEBUG_LEN(debug_len(check_ffn(d), d, stream), stream,
               gated_ffn_impl(d, x, wg, wu, wd, y, saved, workspace, ws_bytes, stream));
}

size_t sc_gated_ffn_backward_workspace_size(const sc_ffn_desc* d) {
  return check_ffn(d) == SC_OK
             ? sc::ffn_backward_workspace_bytes(ffn_args(d, nullptr, nullptr, nullptr, nullptr, nullptr))
             : 0;
}

sc_status sc_gated_ffn_backward(const sc_ffn_desc* d, const void* x, const void* wg, const void* wu, const void* wd,
                                const void* saved, const void* dy, void* dx, void* dwg, void* dwu, void* dwd,
                                void* workspace, size_t ws_bytes, void* stream) {
  SC_DEBUG_LEN(debug_len(check_ffn(d), d, stream), stream,
               gated_ffn_backward_impl(d, x, wg, wu, wd, saved, dy, dx, dwg, dwu, dwd, workspace, ws_bytes, stream));
}

sc_status sc_dropout(const sc_dropout_desc* d, const void* x, const int64_t* seed, const void* residual, void* out,
                     void* stream) {
  SC_DEBUG_LEN(debug_len(check_dropout(d), d, stream), stream, dropout_impl(d, x, seed, residual, out, stream));
}

}  // extern "C"
