// Entry points of the layers around the attention (evo.h): argument checks and
// launches.  What the device arrays hold is not known here; the kernels bound
// every access themselves.
#include <hip/hip_runtime.h>

#include <cmath>

#include "evo_host.hpp"
#include "evo_layers.hpp"

namespace evo {
namespace {

constexpr int kMaxWidth = 16384;         // of a normalised row
// Rows of a norm: up to 256, 512 or 1024 threads each, of fewer than 2^32 that a launch
// may have.
constexpr int max_norm_rows(int d) { return (1 << (d <= 2048 ? 24 : d <= 4096 ? 23 : 22)) - 1; }
constexpr int kMaxFeatures = 1 << 20;    // rows and columns of weights
constexpr int kMaxLinearRows = 1 << 20;

#define TRY(expr)                  \
  do {                             \
    const int rc_ = (expr);        \
    if (rc_ != EVO_OK) return rc_; \
  } while (0)

bool aligned(const void* p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
int elt(int dtype) { return dtype == EVO_BF16 ? 2 : 4; }

int check_dtype(const char* name, int dtype) {
  if (dtype != EVO_FP32 && dtype != EVO_BF16) return fail(EVO_E_INVALID, "bad %s %d", name, dtype);
  return EVO_OK;
}

int check_matrix(const char* name, const evo_matrix* m, int dtype, int64_t rows, int columns, bool written) {
  if (!m || !m->data) return fail(EVO_E_INVALID, "%s is NULL", name);
  if (!aligned(m->data, elt(dtype))) return fail(EVO_E_INVALID, "%s is not aligned to its type", name);
  if (rows > 1 && m->row_stride < (written ? columns : 0))
    return fail(EVO_E_INVALID, "%s: row stride %lld", name, (long long)m->row_stride);
  return EVO_OK;
}

MatrixView view(const evo_matrix* m) { return m ? MatrixView{(char*)m->data, m->row_stride} : MatrixView{nullptr, 0}; }
bool is_wide(const MatrixView& v, int dtype) { return !v.p || (aligned(v.p, 16) && v.row * elt(dtype) % 16 == 0); }

int launched(hipError_t e) {
  if (e != hipSuccess) return fail(EVO_E_HIP, "launch failed: %s", hipGetErrorString(e));
  return EVO_OK;
}

int check_floats(const char* name, const float* p) {
  if (!aligned(p, 4)) return fail(EVO_E_INVALID, "%s is not aligned to its type", name);
  return EVO_OK;
}

int check_norm(const evo_block_norm_desc* n) {
  if (!n) return fail(EVO_E_INVALID, "desc is NULL");
  TRY(check_dtype("stream_dtype", n->stream_dtype));
  TRY(check_dtype("block_dtype", n->block_dtype));
  if (n->stream_dtype == EVO_BF16 && n->block_dtype == EVO_FP32)
    return fail(EVO_E_UNSUPPORTED, "a bf16 stream works with bf16 blocks");
  if (n->d < 1) return fail(EVO_E_INVALID, "d %d", n->d);
  if (n->d > kMaxWidth) return fail(EVO_E_UNSUPPORTED, "d %d: up to %d", n->d, kMaxWidth);
  for (int kind : {n->post, n->pre})
    if (kind < EVO_NORM_NONE || kind > EVO_NORM_LAYER) return fail(EVO_E_INVALID, "bad norm %d", kind);
  if (!std::isfinite(n->alpha)) return fail(EVO_E_INVALID, "alpha must be finite");
  if (!(n->eps >= 0.f) || std::isinf(n->eps)) return fail(EVO_E_INVALID, "eps must be finite and at least 0");
  if (!n->post && (n->post_gain || n->post_bias)) return fail(EVO_E_INVALID, "post_gain or post_bias without post's norm");
  if (!n->pre && (n->pre_gain || n->pre_bias || n->scale.data || n->shift.data))
    return fail(EVO_E_INVALID, "pre_gain, pre_bias, scale or shift without pre's norm");
  TRY(check_floats("post_gain", n->post_gain));
  TRY(check_floats("post_bias", n->post_bias));
  TRY(check_floats("pre_gain", n->pre_gain));
  TRY(check_floats("pre_bias", n->pre_bias));
  return EVO_OK;
}

int check_linear_sizes(int dtype, int n_rows, int n_in, int n_out) {
  TRY(check_dtype("dtype", dtype));
  if (n_out < 1 || n_in < 1) return fail(EVO_E_INVALID, "weights of %d by %d", n_out, n_in);
  if (n_out > kMaxFeatures || n_in > kMaxFeatures)
    return fail(EVO_E_UNSUPPORTED, "weights of %d by %d: up to 2^20 each", n_out, n_in);
  if (n_rows < 0) return fail(EVO_E_INVALID, "%d rows", n_rows);
  if (n_rows > kMaxLinearRows) return fail(EVO_E_UNSUPPORTED, "%d rows: up to 2^20", n_rows);
  return EVO_OK;
}

void set_linear_sizes(LinearArgs* a, int n_rows, int n_in, int n_out) {
  a->n_rows = n_rows;
  a->n_in = n_in;
  a->n_out = n_out;
  a->chunks = (n_in + 127) / 128;
}

// Compute units of the current device (see evo_memory.hip's).
int compute_units() {
  int dev = 0, n = 0;
  if (hipGetDevice(&dev) != hipSuccess) return 256;
  if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n < 1) return 256;
  return n;
}

}  // namespace
}  // namespace evo

using namespace evo;

extern "C" {

int evo_block_norm(const evo_block_norm_desc* desc, int32_t n_rows, const evo_matrix* x, const evo_matrix* y,
                   const evo_matrix* x_out, const evo_matrix* h, void* hip_stream) {
  clear_error();
  TRY(check_norm(desc));
  if (n_rows < 0) return fail(EVO_E_INVALID, "%d rows", n_rows);
  if (n_rows > max_norm_rows(desc->d))
    return fail(EVO_E_UNSUPPORTED, "%d rows of %d: up to %d (2^24 - 1 up to 2048, 2^23 - 1 up to 4096, 2^22 - 1)", n_rows, desc->d, max_norm_rows(desc->d));
  const evo_block_norm_desc& n = *desc;
  if (!y && (n.post || n.gate.data)) return fail(EVO_E_INVALID, "post's norm or a gate without y");
  if (!n.pre != !h) return fail(EVO_E_INVALID, n.pre ? "h is NULL" : "h without pre's norm");
  if (!x_out && !h) return fail(EVO_E_INVALID, "neither x_out nor h");
  const bool mods = n.gate.data || n.scale.data || n.shift.data;
  if (mods) {
    if (n.n_mods < 1) return fail(EVO_E_INVALID, "n_mods %d", n.n_mods);
    if (!n.mod_rows && n_rows % n.n_mods)
      return fail(EVO_E_INVALID, "without mod_rows %d rows must be a multiple of n_mods %d", n_rows, n.n_mods);
    if (n.gate.data) TRY(check_matrix("gate", &n.gate, n.block_dtype, n.n_mods, n.d, false));
    if (n.scale.data) TRY(check_matrix("scale", &n.scale, n.block_dtype, n.n_mods, n.d, false));
    if (n.shift.data) TRY(check_matrix("shift", &n.shift, n.block_dtype, n.n_mods, n.d, false));
    if (!aligned(n.mod_rows, 4)) return fail(EVO_E_INVALID, "mod_rows is not aligned to its type");
  } else if (n.mod_rows) {
    return fail(EVO_E_INVALID, "mod_rows without gate, scale or shift");
  }
  if (n_rows) {
    TRY(check_matrix("x", x, n.stream_dtype, n_rows, n.d, false));
    if (y) TRY(check_matrix("y", y, n.block_dtype, n_rows, n.d, false));
    if (x_out) TRY(check_matrix("x_out", x_out, n.stream_dtype, n_rows, n.d, true));
    if (h) TRY(check_matrix("h", h, n.block_dtype, n_rows, n.d, true));
  }
  if (!n_rows) return EVO_OK;
  NormArgs a = {};
  a.x = view(x);
  a.y = view(y);
  a.x_out = view(x_out);
  a.h = view(h);
  a.gate = view(&n.gate);
  a.scale = view(&n.scale);
  a.shift = view(&n.shift);
  a.post_gain = n.post_gain;
  a.post_bias = n.post_bias;
  a.pre_gain = n.pre_gain;
  a.pre_bias = n.pre_bias;
  a.mod_rows = n.mod_rows;
  a.n_rows = n_rows;
  a.d = n.d;
  a.n_mods = mods ? n.n_mods : 0;
  a.post = n.post;
  a.pre = n.pre;
  a.alpha = n.alpha;
  a.eps = n.eps;
  a.inv_d = 1.f / (float)n.d;
  a.by_mod = Divisor::of(mods && !n.mod_rows ? n_rows / n.n_mods : 1);
  bool wide = n.d % 8 == 0;
  for (const MatrixView* v : {&a.x, &a.x_out}) wide = wide && is_wide(*v, n.stream_dtype);
  for (const MatrixView* v : {&a.y, &a.h, &a.gate, &a.scale, &a.shift}) wide = wide && is_wide(*v, n.block_dtype);
  for (const float* g : {n.post_gain, n.post_bias, n.pre_gain, n.pre_bias}) wide = wide && aligned(g, 16);
  return launched(launch_block_norm(n.stream_dtype, n.block_dtype, wide, a, (hipStream_t)hip_stream));
}

int evo_coded_linear(const evo_weights4* w, int32_t dtype, int32_t n_rows, const evo_matrix* x, const float* bias,
                     int32_t activation, const evo_matrix* out, void* hip_stream) {
  clear_error();
  if (!w) return fail(EVO_E_INVALID, "weights are NULL");
  TRY(check_linear_sizes(dtype, n_rows, w->n_in, w->n_out));
  if (!w->codes || !w->scales) return fail(EVO_E_INVALID, "codes or scales are NULL");
  if (!aligned(w->codes, 16)) return fail(EVO_E_INVALID, "codes must be 16-byte aligned");
  if (activation < EVO_ACT_NONE || activation > EVO_ACT_GELU) return fail(EVO_E_INVALID, "bad activation %d", activation);
  TRY(check_floats("bias", bias));
  if (!n_rows) return EVO_OK;
  TRY(check_matrix("x", x, dtype, n_rows, w->n_in, false));
  TRY(check_matrix("out", out, dtype, n_rows, w->n_out, true));
  LinearArgs a = {};
  a.codes = (const uint8_t*)w->codes;
  a.scales = (const uint8_t*)w->scales;
  a.x = view(x);
  a.out = view(out);
  a.bias = bias;
  set_linear_sizes(&a, n_rows, w->n_in, w->n_out);
  a.act = activation;
  a.wide_out = is_wide(a.out, dtype);
  return launched(launch_linear4(dtype, compute_units(), a, (hipStream_t)hip_stream));
}

int evo_debug_linear_plan(int32_t dtype, int32_t n_rows, int32_t n_in, int32_t n_out, int32_t n_cu, int32_t* out) {
  clear_error();
  TRY(check_linear_sizes(dtype, n_rows, n_in, n_out));
  if (n_rows < 1 || n_cu < 1 || !out) return fail(EVO_E_INVALID, "bad argument");
  LinearArgs a = {};
  set_linear_sizes(&a, n_rows, n_in, n_out);
  return describe_linear4(dtype, n_cu, a, out);
}

}  // extern "C"
