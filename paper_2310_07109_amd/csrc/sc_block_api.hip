// C ABI of the block operators (declared in include/sc_block.h): argument
// validation on the host and launch sequencing on the caller's stream.
#include <cmath>
#include <cstring>

#include "../../include/sc_block.h"
#include "sc_api_common.h"
#include "sc_internal.h"

namespace {

bool aligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

constexpr int kQuantMaxK = 1 << 29;  // 32-bit byte offsets inside a row

bool float_type(int t) { return t == SC_F32 || t == SC_BF16; }

// A padded batch of rows.
sc_status check_rows(int B, int n) {
  if (B < 1 || n < 1) return SC_EINVAL;
  return (long long)B * n < (1LL << 31) ? SC_OK : SC_EUNSUPPORTED;
}

sc_status check_linear(const sc_linear_desc* d) {
  if (!d) return SC_EINVAL;
  if (d->K < 1 || d->N < 1) return SC_EINVAL;
  if (!float_type(d->x_dtype) && d->x_dtype != SC_I8) return SC_EINVAL;
  if (!float_type(d->out_dtype)) return SC_EINVAL;
  if (d->act != SC_ACT_NONE && d->act != SC_ACT_GELU) return SC_EINVAL;
  const sc_status st = check_rows(d->B, d->n);
  if (st != SC_OK) return st;
  if (d->K > sc::kI8MaxK) return SC_EUNSUPPORTED;
  if (d->valid_len && d->B > sc::kPackMaxB) return SC_EUNSUPPORTED;  // the packed rows' prefix table
  // tile loads address the rows and the weights with 32-bit byte offsets
  const long long rows = (long long)d->B * d->n, pitch = sc::i8_pitch(d->K);
  if (rows * pitch >= (1LL << 32) || d->N * pitch >= (1LL << 32)) return SC_EUNSUPPORTED;
  return SC_OK;
}

struct LinearWs {
  int8_t* xq;
  float* xs;
};
size_t carve_linear(const sc_linear_desc* d, void* base, LinearWs* w) {
  // no rows of its own: they come quantised, or stay in the launch
  if (d->x_dtype == SC_I8 || sc::linear_few_ok((long long)d->B * d->n, d->K, d->N, d->x_dtype)) return 0;
  const size_t rows = (size_t)d->B * d->n;
  Carver c(base);
  LinearWs x;
  x.xq = c.take<int8_t>(rows * sc::i8_pitch(d->K));
  x.xs = c.take<float>(rows);
  if (w) *w = x;
  return c.off;
}

sc_status check_norm(const sc_norm_desc* d) {
  if (!d) return SC_EINVAL;
  if (d->D < 1) return SC_EINVAL;
  if (d->kind != SC_NORM_LAYER && d->kind != SC_NORM_RMS) return SC_EINVAL;
  if ((d->post != 0 && d->post != 1) || (d->pre != 0 && d->pre != 1)) return SC_EINVAL;
  if (d->gate_mode < SC_GATE_NONE || d->gate_mode > SC_GATE_TOKEN) return SC_EINVAL;
  if (!(d->eps > 0.f) || !std::isfinite(d->eps) || !std::isfinite(d->res_scale)) return SC_EINVAL;
  if (!float_type(d->dtype)) return SC_EINVAL;
  const sc_status st = check_rows(d->B, d->n);
  if (st != SC_OK) return st;
  return d->D > sc::kNormMaxD ? SC_EUNSUPPORTED : SC_OK;
}

size_t gate_bytes(const sc_norm_desc* d) {
  const size_t e = elem_size(d->dtype), D = d->D;
  switch (d->gate_mode) {
    case SC_GATE_CHANNEL: return D * sizeof(float);
    case SC_GATE_SEQUENCE: return d->B * D * e;
    case SC_GATE_TOKEN: return (size_t)d->B * d->n * D * e;
    default: return 0;
  }
}

// What both directions read.
sc_status check_norm_inputs(const sc_norm_desc* d, const void* x, const void* t, const void* gate,
                            const float* post_w, const float* post_b, const float* pre_w, const float* pre_b) {
  if (!x) return SC_EINVAL;
  if (!t && (d->post || d->gate_mode != SC_GATE_NONE)) return SC_EINVAL;
  if ((gate != nullptr) != (d->gate_mode != SC_GATE_NONE)) return SC_EINVAL;
  if (!d->post && (post_w || post_b)) return SC_EINVAL;
  if (!d->pre && (pre_w || pre_b)) return SC_EINVAL;
  return SC_OK;
}

sc::Norm norm_args(const sc_norm_desc* d, const void* x, const void* t, const void* gate, const float* post_w,
                   const float* post_b, const float* pre_w, const float* pre_b) {
  sc::Norm a;
  std::memset(&a, 0, sizeof(a));
  a.x = x;
  a.t = t;
  a.gate = gate;
  a.post_w = post_w;
  a.post_b = post_b;
  a.pre_w = pre_w;
  a.pre_b = pre_b;
  a.B = d->B;
  a.n = d->n;
  a.D = d->D;
  a.len = d->valid_len;
  a.rms = d->kind == SC_NORM_RMS;
  a.post = d->post;
  a.pre = d->pre;
  a.gate_mode = d->gate_mode;
  a.f32 = d->dtype == SC_F32;
  a.eps = d->eps;
  a.scale = d->res_scale;
  return a;
}

struct Span {
  const void* p;
  size_t n;
};
// An output against inputs and other outputs.
template <size_t N>
bool any_overlap(const Span& out, const Span (&others)[N]) {
  for (const Span& o : others)
    if (overlaps(out.p, out.n, o.p, o.n)) return true;
  return false;
}

sc_status quantize_rows_impl(int32_t B, int32_t n, int32_t K, const int32_t* valid_len, int32_t dtype, const void* x,
                             int8_t* xq, float* scale, void* stream) {
  if (K < 1 || !float_type(dtype) || !x || !xq || !scale) return SC_EINVAL;
  const sc_status st = check_rows(B, n);
  if (st != SC_OK) return st;
  if (K >= kQuantMaxK) return SC_EUNSUPPORTED;
  const size_t rows = (size_t)B * n, xb = rows * K * elem_size(dtype), qb = rows * sc::i8_pitch(K), sb = rows * 4;
  if (!aligned(xq, 16)) return SC_EINVAL;
  if (overlaps(xq, qb, x, xb) || overlaps(scale, sb, x, xb) || overlaps(xq, qb, scale, sb)) return SC_EINVAL;
  if (valid_len && (overlaps(xq, qb, valid_len, 4 * (size_t)B) || overlaps(scale, sb, valid_len, 4 * (size_t)B)))
    return SC_EINVAL;
  return sc::launch_quant_rows(x, dtype == SC_F32, xq, scale, B, n, K, valid_len, nullptr, 1, nullptr, 0,
                               static_cast<hipStream_t>(stream)) == hipSuccess
             ? SC_OK
             : SC_EHIP;
}

sc_status linear_impl(const sc_linear_desc* d, const void* x, const float* x_scale, const int8_t* wq,
                      const float* w_scale, const float* bias, void* out, void* workspace, size_t ws_bytes,
                      void* stream) {
  const sc_status st = check_linear(d);
  if (st != SC_OK) return st;
  if (!x || !wq || !w_scale || !out || (x_scale != nullptr) != (d->x_dtype == SC_I8)) return SC_EINVAL;
  if (!aligned(wq, 16) || (d->x_dtype == SC_I8 && !aligned(x, 16))) return SC_EINVAL;
  const size_t need = carve_linear(d, nullptr, nullptr);
  if (need > 0 && (!workspace || ws_bytes < need)) return SC_EWORKSPACE;
  if (need > 0 && !aligned(workspace, 16)) return SC_EINVAL;  // it holds 8-bit rows
  const size_t rows = (size_t)d->B * d->n, pitch = sc::i8_pitch(d->K), N = d->N;
  const Span in_x{x, d->x_dtype == SC_I8 ? rows * pitch : rows * d->K * elem_size(d->x_dtype)};
  const Span o{out, rows * N * elem_size(d->out_dtype)}, ws{workspace, need};
  const Span ins[] = {in_x, {x_scale, rows * 4}, {wq, N * pitch}, {w_scale, N * 4}, {bias, N * 4},
                      {d->valid_len, 4 * (size_t)d->B}};
  if (any_overlap(o, ins) || any_overlap(ws, ins) || overlaps(o.p, o.n, ws.p, ws.n)) return SC_EINVAL;
  hipStream_t s = static_cast<hipStream_t>(stream);
  sc::Linear l;
  std::memset(&l, 0, sizeof(l));
  l.xq = static_cast<const int8_t*>(x);
  l.xs = x_scale;
  l.wq = wq;
  l.w_scale = w_scale;
  l.bias = bias;
  l.out = out;
  l.B = d->B;
  l.n = d->n;
  l.K = d->K;
  l.N = d->N;
  l.len = d->valid_len;
  l.gelu = d->act == SC_ACT_GELU;
  l.out_f32 = d->out_dtype == SC_F32;
  if (sc::linear_few_ok((long long)rows, d->K, d->N, d->x_dtype))
    return sc::launch_linear_few(l, x, d->x_dtype, s) == hipSuccess ? SC_OK : SC_EHIP;
  if (d->x_dtype != SC_I8) {
    LinearWs w;
    carve_linear(d, workspace, &w);
    if (sc::launch_quant_rows(x, d->x_dtype == SC_F32, w.xq, w.xs, d->B, d->n, d->K, d->valid_len, nullptr, 0, out,
                              (long long)N * elem_size(d->out_dtype), s) != hipSuccess)
      return SC_EHIP;
    l.skip_pad = 1;  // they are zero already
    l.xq = w.xq;
    l.xs = w.xs;
  }
  return sc::launch_linear_i8(l, s) == hipSuccess ? SC_OK : SC_EHIP;
}

sc_status block_norm_impl(const sc_norm_desc* d, const void* x, const void* t, const void* gate, const float* post_w,
                          const float* post_b, const float* pre_w, const float* pre_b, void* r, void* y, int8_t* yq,
                          float* yscale, void* stream) {
  sc_status st = check_norm(d);
  if (st != SC_OK) return st;
  st = check_norm_inputs(d, x, t, gate, post_w, post_b, pre_w, pre_b);
  if (st != SC_OK) return st;
  if (!r && !y && !yq) return SC_EINVAL;
  if (!d->pre && (y || yq)) return SC_EINVAL;
  if ((yq != nullptr) != (yscale != nullptr) || !aligned(yq, 16)) return SC_EINVAL;
  const size_t rows = (size_t)d->B * d->n, xb = rows * d->D * elem_size(d->dtype), wb = 4 * (size_t)d->D;
  const Span ins[] = {{t, xb},     {gate, gate_bytes(d)}, {post_w, wb}, {post_b, wb},
                      {pre_w, wb}, {pre_b, wb},           {d->valid_len, 4 * (size_t)d->B}};
  const Span outs[] = {{r, xb}, {y, xb}, {yq, rows * sc::i8_pitch(d->D)}, {yscale, rows * 4}};
  for (int i = 0; i < 4; ++i) {
    if (any_overlap(outs[i], ins)) return SC_EINVAL;
    if (!(i == 0 && r == x) && overlaps(outs[i].p, outs[i].n, x, xb)) return SC_EINVAL;
    for (int j = 0; j < i; ++j)
      if (overlaps(outs[i].p, outs[i].n, outs[j].p, outs[j].n)) return SC_EINVAL;
  }
  sc::Norm a = norm_args(d, x, t, gate, post_w, post_b, pre_w, pre_b);
  a.r = r;
  a.y = y;
  a.yq = yq;
  a.yscale = yscale;
  return sc::launch_block_norm(a, static_cast<hipStream_t>(stream)) == hipSuccess ? SC_OK : SC_EHIP;
}

sc_status block_norm_backward_impl(const sc_norm_desc* d, const void* x, const void* t, const void* gate,
                                   const float* post_w, const float* post_b, const float* pre_w, const float* pre_b,
                                   const void* dr, const void* dy, void* dx, void* dt, void* dgate, float* dpost_w,
                                   float* dpost_b, float* dpre_w, float* dpre_b, void* workspace, size_t ws_bytes,
                                   void* stream) {
  sc_status st = check_norm(d);
  if (st != SC_OK) return st;
  st = check_norm_inputs(d, x, t, gate, post_w, post_b, pre_w, pre_b);
  if (st != SC_OK) return st;
  if (!dr && !dy) return SC_EINVAL;
  if (dy && !d->pre) return SC_EINVAL;
  if (!dx && !dt && !dgate && !dpost_w && !dpost_b && !dpre_w && !dpre_b) return SC_EINVAL;
  if ((dt && !t) || (dgate && !gate) || ((dpost_w || dpost_b) && !d->post) || ((dpre_w || dpre_b) && !d->pre))
    return SC_EINVAL;
  sc::Norm a = norm_args(d, x, t, gate, post_w, post_b, pre_w, pre_b);
  const size_t need = sc::block_norm_backward_floats(a) * sizeof(float);
  if (!workspace || ws_bytes < need) return SC_EWORKSPACE;
  if (!aligned(workspace, 16)) return SC_EINVAL;
  const size_t xb = (size_t)d->B * d->n * d->D * elem_size(d->dtype), wb = 4 * (size_t)d->D, gb = gate_bytes(d);
  const Span ins[] = {{x, xb},      {t, xb},     {gate, gb},  {post_w, wb}, {post_b, wb},
                      {pre_w, wb},  {pre_b, wb}, {dr, xb},    {dy, xb},     {d->valid_len, 4 * (size_t)d->B}};
  const Span outs[] = {{dx, xb},      {dt, xb},      {dgate, gb}, {dpost_w, wb}, {dpost_b, wb},
                       {dpre_w, wb},  {dpre_b, wb},  {workspace, need}};
  for (int i = 0; i < 8; ++i) {
    for (const Span& in : ins) {
      if ((i == 0 && dx == in.p && in.p == dr) || (i == 1 && dt == in.p && in.p == dy)) continue;
      if (overlaps(outs[i].p, outs[i].n, in.p, in.n)) return SC_EINVAL;
    }
    for (int j = 0; j < i; ++j)
      if (overlaps(outs[i].p, outs[i].n, outs[j].p, outs[j].n)) return SC_EINVAL;
  }
  a.dr = dr;
  a.dy = dy;
  a.dx = dx;
  a.dt = dt;
  a.dgate = dgate;
  a.dpost_w = dpost_w;
  a.dpost_b = dpost_b;
  a.dpre_w = dpre_w;
  a.dpre_b = dpre_b;
  a.ws = static_cast<float*>(workspace);
  return sc::launch_block_norm_backward(a, static_cast<hipStream_t>(stream)) == hipSuccess ? SC_OK : SC_EHIP;
}

}  // namespace

#ifdef SC_DEBUG
namespace {
// The lengths of a call whose sizes are valid; the entry point reports the rest.
sc_status debug_len(sc_status sizes, int B, int n, const int32_t* valid_len, void* stream) {
  return sizes == SC_OK && valid_len ? debug_rows(valid_len, nullptr, B, n, 0, stream) : SC_OK;
}
template <typename D>
sc_status debug_len(sc_status desc, const D* d, void* stream) {
  return desc == SC_OK ? debug_len(desc, d->B, d->n, d->valid_len, stream) : SC_OK;
}
}  // namespace
#define SC_DEBUG_LEN(pre, stream, call) SC_DEBUG_RUN(pre, stream, call)
#else
#define SC_DEBUG_LEN(pre, stream, call) return call
#endif

extern "C" {

int64_t sc_i8_pitch(int64_t K) { return K < 1 ? 0 : (K + sc::kI8Pitch - 1) / sc::kI8Pitch * sc::kI8Pitch; }

sc_status sc_quantize_rows_i8(int32_t B, int32_t n, int32_t K, const int32_t* valid_len, int32_t dtype,
                              const void* x, int8_t* xq, float* scale, void* stream) {
  SC_DEBUG_LEN(debug_len(check_rows(B, n), B, n, valid_len, stream), stream,
               quantize_rows_impl(B, n, K, valid_len, dtype, x, xq, scale, stream));
}

sc_status sc_quantize_weight_i8(int32_t K, int32_t N, int32_t dtype, const void* w, int8_t* wq, float* scale,
                                void* stream) {
  if (K < 1 || N < 1 || !float_type(dtype) || !w || !wq || !scale) return SC_EINVAL;
  if (!aligned(wq, 16)) return SC_EINVAL;
  if (K >= kQuantMaxK) return SC_EUNSUPPORTED;
  const long long pitch = sc::i8_pitch(K);
  if (N * pitch >= (1LL << 32)) return SC_EUNSUPPORTED;
  const size_t wb = (size_t)K * N * elem_size(dtype), qb = (size_t)N * pitch, sb = 4 * (size_t)N;
  if (overlaps(wq, qb, w, wb) || overlaps(scale, sb, w, wb) || overlaps(wq, qb, scale, sb)) return SC_EINVAL;
  const sc_status st = sc::launch_quant_weight(w, dtype == SC_F32, wq, scale, K, N,
                                               static_cast<hipStream_t>(stream)) == hipSuccess
                           ? SC_OK
                           : SC_EHIP;
#ifdef SC_DEBUG
  return debug_post(st, stream);
#else
  return st;
#endif
}

size_t sc_linear_i8_workspace_size(const sc_linear_desc* d) {
  return check_linear(d) == SC_OK ? carve_linear(d, nullptr, nullptr) : 0;
}

sc_status sc_linear_i8(const sc_linear_desc* d, const void* x, const float* x_scale, const int8_t* wq,
                       const float* w_scale, const float* bias, void* out, void* workspace, size_t ws_bytes,
                       void* stream) {
  SC_DEBUG_LEN(debug_len(check_linear(d), d, stream), stream,
               linear_impl(d, x, x_scale, wq, w_scale, bias, out, workspace, ws_bytes, stream));
}

sc_status sc_block_norm(const sc_norm_desc* d, const void* x, const void* t, const void* gate, const float* post_w,
                        const float* post_b, const float* pre_w, const float* pre_b, void* r, void* y, int8_t* yq,
                        float* yscale, void* stream) {
  SC_DEBUG_LEN(debug_len(check_norm(d), d, stream), stream,
               block_norm_impl(d, x, t, gate, post_w, post_b, pre_w, pre_b, r, y, yq, yscale, stream));
}

size_t sc_block_norm_backward_workspace_size(const sc_norm_desc* d) {
  if (check_norm(d) != SC_OK) return 0;
  return sc::block_norm_backward_floats(norm_args(d, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr)) *
         sizeof(float);
}

sc_status sc_block_norm_backward(const sc_norm_desc* d, const void* x, const void* t, const void* gate,
                                 const float* post_w, const float* post_b, const float* pre_w, const float* pre_b,
                                 const void* dr, const void* dy, void* dx, void* dt, void* dgate, float* dpost_w,
                                 float* dpost_b, float* dpre_w, float* dpre_b, void* workspace, size_t ws_bytes,
                                 void* stream) {
  SC_DEBUG_LEN(debug_len(check_norm(d), d, stream), stream,
               block_norm_backward_impl(d, x, t, gate, post_w, post_b, pre_w, pre_b, dr, dy, dx, dt, dgate, dpost_w,
                                        dpost_b, dpre_w, dpre_b, workspace, ws_bytes, stream));
}

}  // extern "C"
