// Entry points of the long memories (evo.h): argument checks and launches.
// What the device arrays hold is not known here; the kernels bound every
// access themselves.
#include <hip/hip_runtime.h>

#include <atomic>
#include <chrono>
#include <cmath>

#include "evo_host.hpp"
#include "evo_memory.hpp"

namespace evo {
namespace {

constexpr int64_t kMaxPositions = 1 << 30;
constexpr int64_t kMaxItems = (1ll << 31) - 1;

#define TRY(expr)                  \
  do {                             \
    const int rc_ = (expr);        \
    if (rc_ != EVO_OK) return rc_; \
  } while (0)

bool aligned(const void* p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
int elt(int dtype) { return dtype == EVO_BF16 ? 2 : 4; }

int check_dtype(int dtype) {
  if (dtype != EVO_FP32 && dtype != EVO_BF16) return fail(EVO_E_INVALID, "bad dtype %d", dtype);
  return EVO_OK;
}

int check_head_dim(int dh) {
  if (dh < 1) return fail(EVO_E_INVALID, "head_dim %d", dh);
  if (dh != 32 && dh != 64 && dh != 128) return fail(EVO_E_UNSUPPORTED, "head_dim %d: 32, 64 and 128 are compiled", dh);
  return EVO_OK;
}

// what a cache's shape says, without its pointers
int check_shape(const evo_kv_cache* c) {
  if (!c) return fail(EVO_E_INVALID, "cache is NULL");
  if (c->format < EVO_CACHE_FP32 || c->format > EVO_CACHE_FP8) return fail(EVO_E_INVALID, "bad cache format %d", c->format);
  TRY(check_head_dim(c->head_dim));
  if (c->n_pages < 1 || c->n_kv_heads < 1)
    return fail(EVO_E_INVALID, "cache of %d pages, %d heads", c->n_pages, c->n_kv_heads);
  if ((int64_t)c->n_pages * c->n_kv_heads > kMaxItems) return fail(EVO_E_UNSUPPORTED, "pages * heads above 2^31");
  if (c->page_size < 1) return fail(EVO_E_INVALID, "page_size %d", c->page_size);
  if (c->page_size < 64 || c->page_size > 1024 || (c->page_size & (c->page_size - 1)))
    return fail(EVO_E_UNSUPPORTED, "page_size %d: 64, 128, 256, 512 and 1024 are supported", c->page_size);
  return EVO_OK;
}

int check_cache(const evo_kv_cache* c) {
  TRY(check_shape(c));
  if (!c->k || !c->v) return fail(EVO_E_INVALID, "the cache's k or v is NULL");
  const bool coded = is_coded(c->format);
  if (coded && (!c->k_scale || !c->v_scale)) return fail(EVO_E_INVALID, "an 8-bit cache needs k_scale and v_scale");
  if (!aligned(c->k, 16) || !aligned(c->v, 16) || (coded && (!aligned(c->k_scale, 16) || !aligned(c->v_scale, 16))))
    return fail(EVO_E_INVALID, "the cache's arrays must be 16-byte aligned");
  return EVO_OK;
}

int check_pair(int dtype, int format) {
  if ((format == EVO_CACHE_FP32 && dtype != EVO_FP32) || (format == EVO_CACHE_BF16 && dtype != EVO_BF16))
    return fail(EVO_E_UNSUPPORTED, "a %s cache works with %s rows", format == EVO_CACHE_FP32 ? "fp32" : "bf16",
                format == EVO_CACHE_FP32 ? "fp32" : "bf16");
  return EVO_OK;
}

int check_rows(const evo_kv_rows* r, const evo_kv_cache* c, int heads, bool pointers) {
  if (!r) return fail(EVO_E_INVALID, "rows is NULL");
  if (r->n_seqs < 1 || r->n_rows < 0 || r->max_rows < 0 || r->max_pages < 1)
    return fail(EVO_E_INVALID, "%d sequences, %d rows (at most %d each), %d pages each", r->n_seqs, r->n_rows, r->max_rows,
                r->max_pages);
  if (r->n_rows > (int64_t)r->n_seqs * r->max_rows)
    return fail(EVO_E_INVALID, "%d rows do not fit %d sequences of at most %d", r->n_rows, r->n_seqs, r->max_rows);
  if (!r->cu_rows && r->n_rows != (int64_t)r->n_seqs * r->max_rows)
    return fail(EVO_E_INVALID, "without cu_rows n_rows must be n_seqs * max_rows");
  if (pointers && !r->page_table) return fail(EVO_E_INVALID, "page_table is NULL");
  if ((int64_t)r->max_pages * c->page_size > kMaxPositions)
    return fail(EVO_E_UNSUPPORTED, "max_pages * page_size above 2^30");
  if (((int64_t)r->n_rows + r->n_seqs) * heads > kMaxItems) return fail(EVO_E_UNSUPPORTED, "rows * heads above 2^31");
  return EVO_OK;
}

int check_heads(const char* name, const evo_heads* h, int dtype, int n_rows, int n_heads, int dh, bool written) {
  if (!n_rows) return EVO_OK;
  if (!h || !h->data) return fail(EVO_E_INVALID, "%s is NULL", name);
  if (!aligned(h->data, elt(dtype))) return fail(EVO_E_INVALID, "%s is not aligned to its type", name);
  const int64_t least = written ? dh : 0;
  if ((n_rows > 1 && h->row_stride < least) || (n_heads > 1 && h->head_stride < least))
    return fail(EVO_E_INVALID, "%s: strides %lld and %lld", name, (long long)h->row_stride, (long long)h->head_stride);
  return EVO_OK;
}

int check_norm_rope(const evo_norm_rope* n, int dh) {
  if (!n) return fail(EVO_E_INVALID, "norm_rope is NULL");
  if (std::isnan(n->eps) || std::isinf(n->eps)) return fail(EVO_E_INVALID, "eps must be finite");
  if (n->rotary_dim < 0 || n->rotary_dim > dh || n->rotary_dim % 16)
    return fail(EVO_E_INVALID, "rotary_dim %d: a multiple of 16 up to head_dim %d", n->rotary_dim, dh);
  if (!n->rotary_dim) return EVO_OK;
  if (n->pairs != EVO_PAIRS_HALVES && n->pairs != EVO_PAIRS_ADJACENT) return fail(EVO_E_INVALID, "bad pairs %d", n->pairs);
  if (!n->table || n->n_positions < 1) return fail(EVO_E_INVALID, "a rotation needs its table");
  if (!aligned(n->table, 16)) return fail(EVO_E_INVALID, "the table must be 16-byte aligned");
  return EVO_OK;
}

HeadsView view(const evo_heads* h) {
  HeadsView v = {};
  if (h) v = HeadsView{(char*)h->data, h->row_stride, h->head_stride};
  return v;
}
bool is_wide(const HeadsView& v, int dtype) {
  return !v.p || (aligned(v.p, 16) && v.row * elt(dtype) % 16 == 0 && v.head * elt(dtype) % 16 == 0);
}

CacheView view(const evo_kv_cache* c) {
  int shift = 0;
  while ((1 << shift) < c->page_size) ++shift;
  return CacheView{c->k, c->v, c->k_scale, c->v_scale, c->n_pages, shift, c->n_kv_heads};
}
RowsView view(const evo_kv_rows* r) {
  // sequences that are all full need no cu_rows
  const bool full = r->n_rows == (int64_t)r->n_seqs * r->max_rows;
  return RowsView{full ? nullptr : r->cu_rows, r->page_table, r->n_seqs, r->n_rows, r->max_rows, r->max_pages,
                  Divisor::of(r->max_rows ? r->max_rows : 1)};
}

void set_norm_rope(RowsArgs* a, const evo_norm_rope* n) {
  a->norm = n->eps >= 0.f;
  a->eps = n->eps;
  a->q_gain = n->q_gain;
  a->k_gain = n->k_gain;
  a->half = n->rotary_dim / 2;
  a->adjacent = n->pairs == EVO_PAIRS_ADJACENT;
  a->n_positions = n->n_positions;
  a->table = n->table;
}

int launched(hipError_t e) {
  if (e != hipSuccess) return fail(EVO_E_HIP, "launch failed: %s", hipGetErrorString(e));
  return EVO_OK;
}

// Compute units of the current device (256 where there is none, so that a plan
// can be made on a machine without a GPU).
int compute_units() {
  constexpr int kDevices = 64;
  static std::atomic<int> known[kDevices];
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kDevices) return 256;
  int n = known[dev].load(std::memory_order_relaxed);
  if (n) return n;
  if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n < 1) return 256;
  known[dev].store(n, std::memory_order_relaxed);
  return n;
}

int check_attention(const evo_kv_cache* c, const evo_kv_rows* r, const evo_attention* t, bool pointers) {
  if (pointers) TRY(check_cache(c));
  else TRY(check_shape(c));
  if (!t) return fail(EVO_E_INVALID, "attention is NULL");
  TRY(check_dtype(t->dtype));
  TRY(check_pair(t->dtype, c->format));
  if (t->n_heads < 1 || t->n_heads % c->n_kv_heads)
    return fail(EVO_E_INVALID, "n_heads %d is not a multiple of the cache's %d", t->n_heads, c->n_kv_heads);
  TRY(check_rows(r, c, t->n_heads, pointers));
  if (r->n_rows >= kMaxPositions) return fail(EVO_E_UNSUPPORTED, "rows above 2^30");
  if (t->causal != 0 && t->causal != 1) return fail(EVO_E_INVALID, "causal must be 0 or 1");
  if (t->window < 0 || t->window > kMaxPositions) return fail(EVO_E_INVALID, "window %d", t->window);
  if (t->max_length < 0) return fail(EVO_E_INVALID, "max_length %d", t->max_length);
  if (!std::isfinite(t->scale)) return fail(EVO_E_INVALID, "scale must be finite");
  if (!(t->cap >= 0.f) || std::isinf(t->cap)) return fail(EVO_E_INVALID, "cap must be finite and at least 0");
  if (pointers && !t->lengths) return fail(EVO_E_INVALID, "lengths is NULL");
  return EVO_OK;
}

AttPlan plan_of(const evo_kv_cache* c, const RowsView& r, const evo_attention* t) {
  const int64_t most = (int64_t)r.max_pages * c->page_size;
  const int64_t length = t->max_length ? (t->max_length < most ? t->max_length : most) : most;
  return plan_attention(t->dtype, c->format, c->head_dim, t->n_heads, c->n_kv_heads, r, (int)length, compute_units());
}
int64_t bytes_of(const AttPlan& p) {
  return (p.part_floats + p.ml_floats) * (int64_t)sizeof(float) + p.flags * (int64_t)sizeof(unsigned long long);
}

// A number that no other call of this process has, and that memory which holds
// anything is not likely to hold (steps of an odd constant over 64 bits, from
// the clock; 0 is what cleared flags hold).
unsigned long long call_number() {
  static std::atomic<unsigned long long> next{
      (unsigned long long)std::chrono::high_resolution_clock::now().time_since_epoch().count() * 0x9e3779b97f4a7c15ull};
  const unsigned long long n = next.fetch_add(0x9e3779b97f4a7c15ull, std::memory_order_relaxed);
  return n ? n : call_number();
}

}  // namespace
}  // namespace evo

using namespace evo;

extern "C" {

int evo_qk_norm_rope(const evo_norm_rope* nr, int32_t dtype, int32_t head_dim, int32_t n_rows, int32_t n_heads,
                     int32_t n_kv_heads, const evo_heads* q, const evo_heads* k, const int32_t* positions,
                     const evo_heads* q_out, const evo_heads* k_out, void* hip_stream) {
  clear_error();
  TRY(check_dtype(dtype));
  TRY(check_head_dim(head_dim));
  TRY(check_norm_rope(nr, head_dim));
  if (n_rows < 0 || n_heads < 0 || n_kv_heads < 0 || (int64_t)n_heads + n_kv_heads < 1)
    return fail(EVO_E_INVALID, "%d rows, %d and %d heads", n_rows, n_heads, n_kv_heads);
  if (n_rows * ((int64_t)n_heads + n_kv_heads) > kMaxItems) return fail(EVO_E_UNSUPPORTED, "rows * heads above 2^31");
  RowsArgs a = {};
  if (n_heads) {
    TRY(check_heads("q", q, dtype, n_rows, n_heads, head_dim, false));
    TRY(check_heads("q_out", q_out, dtype, n_rows, n_heads, head_dim, true));
    a.q = view(q);
    a.qo = view(q_out);
  }
  if (n_kv_heads) {
    TRY(check_heads("k", k, dtype, n_rows, n_kv_heads, head_dim, false));
    TRY(check_heads("k_out", k_out, dtype, n_rows, n_kv_heads, head_dim, true));
    a.k = view(k);
    a.ko = view(k_out);
  }
  if (nr->rotary_dim && !positions) return fail(EVO_E_INVALID, "positions is NULL");
  if (!n_rows) return EVO_OK;
  set_norm_rope(&a, nr);
  a.n_heads = n_heads;
  a.n_kv_heads = n_kv_heads;
  a.positions = positions;
  a.rows.n_rows = n_rows;
  a.wide = is_wide(a.q, dtype) && is_wide(a.k, dtype) && is_wide(a.qo, dtype) && is_wide(a.ko, dtype);
  return launched(launch_rows(dtype, -1, head_dim, a, (hipStream_t)hip_stream));
}

int evo_cache_write(const evo_kv_cache* cache, const evo_kv_rows* rows, int32_t dtype, const int32_t* starts,
                    const evo_heads* k, const evo_heads* v, void* hip_stream) {
  clear_error();
  TRY(check_cache(cache));
  TRY(check_dtype(dtype));
  TRY(check_pair(dtype, cache->format));
  TRY(check_rows(rows, cache, cache->n_kv_heads, true));
  if (!starts) return fail(EVO_E_INVALID, "starts is NULL");
  TRY(check_heads("k", k, dtype, rows->n_rows, cache->n_kv_heads, cache->head_dim, false));
  TRY(check_heads("v", v, dtype, rows->n_rows, cache->n_kv_heads, cache->head_dim, false));
  if (!rows->n_rows) return EVO_OK;
  RowsArgs a = {};
  a.k = view(k);
  a.v = view(v);
  a.n_kv_heads = cache->n_kv_heads;
  a.starts = starts;
  a.cache = view(cache);
  a.rows = view(rows);
  a.wide = is_wide(a.k, dtype) && is_wide(a.v, dtype);
  return launched(launch_rows(dtype, cache->format, cache->head_dim, a, (hipStream_t)hip_stream));
}

int evo_cache_read(const evo_kv_cache* cache, const evo_kv_rows* rows, int32_t dtype, const int32_t* starts,
                   const evo_heads* k_out, const evo_heads* v_out, void* hip_stream) {
  clear_error();
  TRY(check_cache(cache));
  TRY(check_dtype(dtype));
  TRY(check_pair(dtype, cache->format));
  TRY(check_rows(rows, cache, cache->n_kv_heads, true));
  if (!starts) return fail(EVO_E_INVALID, "starts is NULL");
  TRY(check_heads("k_out", k_out, dtype, rows->n_rows, cache->n_kv_heads, cache->head_dim, true));
  TRY(check_heads("v_out", v_out, dtype, rows->n_rows, cache->n_kv_heads, cache->head_dim, true));
  if (!rows->n_rows) return EVO_OK;
  RowsArgs a = {};
  a.ko = view(k_out);
  a.v = view(v_out);
  a.n_kv_heads = cache->n_kv_heads;
  a.starts = starts;
  a.cache = view(cache);
  a.rows = view(rows);
  a.wide = is_wide(a.ko, dtype) && is_wide(a.v, dtype);
  return launched(launch_cache_read(dtype, cache->format, cache->head_dim, a, (hipStream_t)hip_stream));
}

int evo_qkv_write(const evo_kv_cache* cache, const evo_kv_rows* rows, const evo_norm_rope* nr, int32_t dtype,
                  int32_t n_heads, const int32_t* starts, const evo_heads* q, const evo_heads* k, const evo_heads* v,
                  const evo_heads* q_out, void* hip_stream) {
  clear_error();
  TRY(check_cache(cache));
  TRY(check_dtype(dtype));
  TRY(check_pair(dtype, cache->format));
  TRY(check_norm_rope(nr, cache->head_dim));
  if (n_heads < 1) return fail(EVO_E_INVALID, "n_heads %d", n_heads);
  const int64_t heads = (int64_t)n_heads + cache->n_kv_heads;
  if (heads > (1 << 20)) return fail(EVO_E_UNSUPPORTED, "%lld heads", (long long)heads);
  TRY(check_rows(rows, cache, (int)heads, true));
  if (!starts) return fail(EVO_E_INVALID, "starts is NULL");
  TRY(check_heads("q", q, dtype, rows->n_rows, n_heads, cache->head_dim, false));
  TRY(check_heads("k", k, dtype, rows->n_rows, cache->n_kv_heads, cache->head_dim, false));
  TRY(check_heads("v", v, dtype, rows->n_rows, cache->n_kv_heads, cache->head_dim, false));
  TRY(check_heads("q_out", q_out, dtype, rows->n_rows, n_heads, cache->head_dim, true));
  if (!rows->n_rows) return EVO_OK;
  RowsArgs a = {};
  set_norm_rope(&a, nr);
  a.q = view(q);
  a.k = view(k);
  a.v = view(v);
  a.qo = view(q_out);
  a.n_heads = n_heads;
  a.n_kv_heads = cache->n_kv_heads;
  a.starts = starts;
  a.cache = view(cache);
  a.rows = view(rows);
  a.wide = is_wide(a.q, dtype) && is_wide(a.k, dtype) && is_wide(a.v, dtype) && is_wide(a.qo, dtype);
  return launched(launch_rows(dtype, cache->format, cache->head_dim, a, (hipStream_t)hip_stream));
}

int64_t evo_chunk_attention_workspace(const evo_kv_cache* cache, const evo_kv_rows* rows, const evo_attention* att) {
  clear_error();
  TRY(check_attention(cache, rows, att, false));
  if (!rows->n_rows) return 0;
  return bytes_of(plan_of(cache, view(rows), att));
}

int evo_chunk_attention(const evo_kv_cache* cache, const evo_kv_rows* rows, const evo_attention* att,
                        const evo_heads* q, const evo_heads* out, float* lse, void* workspace, size_t workspace_bytes,
                        void* hip_stream) {
  clear_error();
  TRY(check_attention(cache, rows, att, true));
  TRY(check_heads("q", q, att->dtype, rows->n_rows, att->n_heads, cache->head_dim, false));
  TRY(check_heads("out", out, att->dtype, rows->n_rows, att->n_heads, cache->head_dim, true));
  if (!rows->n_rows) return EVO_OK;
  AttArgs a = {};
  a.rows = view(rows);
  const AttPlan p = plan_of(cache, a.rows, att);
  const int64_t need = bytes_of(p);
  if (need > 0 && (!workspace || workspace_bytes < (size_t)need || !aligned(workspace, 16)))
    return fail(EVO_E_INVALID, "the workspace must hold %lld bytes, 16-byte aligned", (long long)need);
  if (((int64_t)p.n_tiles * cache->n_kv_heads + 8ll * p.tiles_per_seq) * p.n_split > kMaxItems) return fail(EVO_E_UNSUPPORTED, "too many row tiles");
  a.q = view(q);
  a.out = view(out);
  a.lse = lse;
  a.cache = view(cache);
  a.lengths = att->lengths;
  a.starts = att->starts;
  a.prefix = att->prefix;
  a.slopes = att->slopes;
  a.n_heads = att->n_heads;
  a.group = att->n_heads / cache->n_kv_heads;
  a.causal = att->causal;
  a.window = att->window;
  a.scale = att->scale;
  // (scores below 2^-100 are 0 to their exponential: a smaller cap's reciprocal
  // would leave the range of floats)
  a.cap = att->cap > 0.f ? std::fmax(att->cap, 0x1p-100f) : 0.f;
  a.inv_cap = a.cap > 0.f ? 1.f / a.cap : 0.f;
  a.wide = is_wide(a.q, att->dtype) && is_wide(a.out, att->dtype);
  a.tiles_per_seq = p.tiles_per_seq;
  a.n_tiles = p.n_tiles;
  a.n_split = p.n_split;
  a.by_group = Divisor::of(a.group);
  a.by_kv_heads = Divisor::of(cache->n_kv_heads);
  a.by_tiles = Divisor::of(p.tiles_per_seq ? p.tiles_per_seq : 1);
  a.by_eight = Divisor::of(8ll * (p.tiles_per_seq ? p.tiles_per_seq : 1));
  a.by_split = Divisor::of(p.n_split);
  a.part = (float*)workspace;
  a.part_ml = (float*)workspace + p.part_floats;
  if (p.flags) {
    a.flags = (unsigned long long*)(a.part_ml + p.ml_floats);
    a.number = call_number();
  }
  return launched(launch_attention(att->dtype, cache->format, cache->head_dim, p, a, (hipStream_t)hip_stream));
}

}  // extern "C"
