// Host side of the paged key-value cache: the C entry points of
// include/rwttt_kv.h.  Every argument is checked here, before any launch.

#include <cmath>
#include <new>
#include <vector>

#include "rwttt_kv_rows.h"
#include "rwttt_kv_kernels.h"

struct rwttt_kv {
  rwttt_kv_config cfg;
  rwttt::KvShape shape;
  std::vector<void*> k, v, bounds;   // [n_layers], or empty
  int32_t last_hip = 0;
};

namespace {

bool misaligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }
bool device16(const void* p) { return p && !misaligned(p, 16); }
size_t type_bytes(int32_t t) { return t == RWTTT_F32 ? 4 : t == RWTTT_BF16 ? 2 : 1; }

rwttt_status check_shape(const rwttt_kv_config* c) {
  if (!c || c->reserved != 0) return RWTTT_E_INVALID;
  if (c->n_owners == 0 || c->n_owners > RWTTT_KV_MAX_OWNERS || c->n_layers == 0) return RWTTT_E_INVALID;
  if (c->page_rows < 16 || c->page_rows > 256 || (c->page_rows & (c->page_rows - 1))) return RWTTT_E_INVALID;
  if (c->n_pages == 0 || uint64_t(c->n_pages) * c->page_rows > 0x7fffffffu) return RWTTT_E_INVALID;
  if (c->max_pages == 0 || uint64_t(c->max_pages) * c->page_rows > RWTTT_KV_MAX_ROWS) return RWTTT_E_INVALID;
  if (c->n_kv_heads == 0 || c->n_kv_heads > 512 || c->n_heads == 0 || c->n_heads % c->n_kv_heads)
    return RWTTT_E_INVALID;
  if (c->n_heads / c->n_kv_heads > 128) return RWTTT_E_INVALID;
  if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return RWTTT_E_INVALID;
  if (c->io_dtype != RWTTT_F32 && c->io_dtype != RWTTT_BF16) return RWTTT_E_INVALID;
  if (c->cache_dtype != RWTTT_F32 && c->cache_dtype != RWTTT_BF16 && c->cache_dtype != RWTTT_FP8 &&
      c->cache_dtype != RWTTT_FP4)
    return RWTTT_E_INVALID;
  if (c->cache_dtype == RWTTT_F32 && c->io_dtype != RWTTT_F32) return RWTTT_E_INVALID;
  return RWTTT_OK;
}

rwttt::KvShape shape_of(const rwttt_kv_config* c) {
  rwttt::KvShape h;
  h.n_owners = int(c->n_owners);
  h.n_pages = int(c->n_pages);
  h.page_shift = __builtin_ctz(c->page_rows);
  h.max_pages = int(c->max_pages);
  h.kv_heads = int(c->n_kv_heads);
  h.group = int(c->n_heads / c->n_kv_heads);
  h.head_dim = int(c->head_dim);
  h.io_bf16 = c->io_dtype == RWTTT_BF16;
  h.cache = c->cache_dtype;
  return h;
}

size_t workspace_of(const rwttt_kv_config* c) { return rwttt::kv_workspace_bytes(shape_of(c)); }

bool layers_ok(void* const* p, uint32_t n) {
  if (p)
    for (uint32_t l = 0; l < n; ++l)
      if (!device16(p[l])) return false;
  return true;
}

// An array of an extend.
struct Ints {
  const int32_t* p;
  uint64_t n;
};

bool overlap(const Ints& a, const Ints& b) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
  return x < y ? y - x < a.n * sizeof(int32_t) && b.n != 0 : x - y < b.n * sizeof(int32_t) && a.n != 0;
}

// A row of `heads` heads and the stride between rows, in elements of the io
// type: whole 16-byte pieces that do not overlap.
bool stride_ok(const rwttt_kv* kv, uint64_t stride, uint32_t heads) {
  const uint64_t row = uint64_t(heads) * kv->cfg.head_dim;
  return stride >= row && stride < (uint64_t(1) << 40) && (stride * type_bytes(kv->cfg.io_dtype)) % 16 == 0;
}

// n rows of queries or keys, elements of the io type.
struct Rows {
  const void* p;
  uint64_t stride, row;
};

// Whether some of n rows of a are also some of b's; rows side by side within one
// stride do not meet.
bool overlap(const Rows& a, const Rows& b, uint64_t n, uint64_t bytes) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
  const uint64_t span_a = ((n - 1) * a.stride + a.row) * bytes, span_b = ((n - 1) * b.stride + b.row) * bytes;
  if (x < y ? y - x >= span_a : x - y >= span_b) return false;
  if (a.stride != b.stride) return true;
  const uint64_t step = a.stride * bytes, apart = x < y ? (y - x) % step : (x - y) % step;
  const uint64_t lower = (x < y ? a.row : b.row) * bytes, upper = (x < y ? b.row : a.row) * bytes;
  return apart < lower || step - apart < upper;
}

// An array that a call reads.
struct Span {
  const void* p;
  uint64_t bytes;
};

// Whether some of n rows are also the array's; between two rows it may lie.
bool overlap(const Rows& a, uint64_t n, uint64_t bytes, const Span& b) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
  if (!b.p || y < x) return b.p && x - y < b.bytes;
  if (y - x >= ((n - 1) * a.stride + a.row) * bytes) return false;
  const uint64_t step = a.stride * bytes, at = (y - x) % step;
  return at < a.row * bytes || step - at < b.bytes;
}

// Bytes of a layer's keys or values.
uint64_t layer_bytes(const rwttt_kv_config& c) {
  const uint64_t n = uint64_t(c.n_pages) * c.n_kv_heads * c.page_rows * c.head_dim;
  return c.cache_dtype == RWTTT_F32    ? n * 4
         : c.cache_dtype == RWTTT_BF16 ? n * 2
         : c.cache_dtype == RWTTT_FP8  ? n
                                       : n / 32 * 17;
}

rwttt_status hip_result(rwttt_kv* kv, hipError_t e) {
  if (e == hipSuccess) return RWTTT_OK;
  kv->last_hip = static_cast<int32_t>(e);
  return RWTTT_E_HIP;
}

// The arguments select and attend share.
bool queries_ok(const rwttt_kv* kv, uint32_t layer, const void* q, uint64_t q_stride, const int32_t* lengths,
                const int32_t* rows, uint32_t n) {
  if (!kv || layer >= kv->cfg.n_layers || !kv->cfg.table) return false;
  if (!device16(q) || !stride_ok(kv, q_stride, kv->cfg.n_heads)) return false;
  if (!device16(lengths) || misaligned(rows, 16)) return false;
  return rows ? n <= RWTTT_KV_MAX_OWNERS : n == kv->cfg.n_owners;
}

const float* head_scale(const rwttt_kv* kv, const float* p, uint32_t layer) {
  return p ? p + size_t(layer) * kv->cfg.n_kv_heads : nullptr;
}

}  // namespace

extern "C" {

rwttt_status rwttt_kv_workspace_bytes(const rwttt_kv_config* cfg, size_t* bytes) {
  const rwttt_status s = check_shape(cfg);
  if (s != RWTTT_OK) return s;
  if (!bytes) return RWTTT_E_INVALID;
  *bytes = workspace_of(cfg);
  return RWTTT_OK;
}

rwttt_status rwttt_kv_create(const rwttt_kv_config* cfg, rwttt_kv** out) {
  const rwttt_status s = check_shape(cfg);
  if (s != RWTTT_OK) return s;
  if (!out) return RWTTT_E_INVALID;
  const void* plain[] = {cfg->table, cfg->ring, cfg->k_scale, cfg->v_scale, cfg->bound_step};
  for (const void* p : plain)
    if (misaligned(p, 16)) return RWTTT_E_INVALID;
  if ((cfg->k == nullptr) != (cfg->v == nullptr)) return RWTTT_E_INVALID;
  if (!layers_ok(cfg->k, cfg->n_layers) || !layers_ok(cfg->v, cfg->n_layers) ||
      !layers_ok(cfg->bounds, cfg->n_layers))
    return RWTTT_E_INVALID;
  if (cfg->bounds && !cfg->bound_step) return RWTTT_E_INVALID;
  if (cfg->cache_dtype != RWTTT_FP8 && (cfg->k_scale || cfg->v_scale)) return RWTTT_E_INVALID;
  if (cfg->workspace) {
    if (misaligned(cfg->workspace, 256)) return RWTTT_E_INVALID;
    if (cfg->workspace_bytes < workspace_of(cfg)) return RWTTT_E_CAPACITY;
  }
  rwttt_kv* kv = new (std::nothrow) rwttt_kv;
  if (!kv) return RWTTT_E_CAPACITY;
  kv->cfg = *cfg;
  try {
    if (cfg->k) {
      kv->k.assign(cfg->k, cfg->k + cfg->n_layers);
      kv->v.assign(cfg->v, cfg->v + cfg->n_layers);
    }
    if (cfg->bounds) kv->bounds.assign(cfg->bounds, cfg->bounds + cfg->n_layers);
  } catch (const std::bad_alloc&) {
    delete kv;
    return RWTTT_E_CAPACITY;
  }
  kv->cfg.k = kv->cfg.v = kv->cfg.bounds = nullptr;
  kv->shape = shape_of(cfg);
  *out = kv;
  return RWTTT_OK;
}

rwttt_status rwttt_kv_destroy(rwttt_kv* kv) {
  if (!kv) return RWTTT_E_INVALID;
  delete kv;
  return RWTTT_OK;
}

rwttt_status rwttt_kv_extend(rwttt_kv* kv, const int32_t* have, const int32_t* want, const int32_t* pos,
                             int32_t* new_pos, int32_t* lengths, int32_t* start, int32_t* slots,
                             int32_t* owners, int32_t* positions, uint32_t cap, int32_t* result,
                             void* stream) {
  if (!kv || !kv->cfg.table || !kv->cfg.ring) return RWTTT_E_INVALID;
  if (cap > 0x7fffffffu) return RWTTT_E_INVALID;
  const uint64_t n = kv->cfg.n_owners;
  const Ints in[] = {{have, n}, {want, n}, {pos, 2}};
  const Ints out[] = {{new_pos, 2},     {lengths, n},  {start, n + 1},
                      {result, 4},      {slots, cap},  {owners, cap},
                      {positions, cap}, {kv->cfg.table, n * kv->cfg.max_pages}, {kv->cfg.ring, kv->cfg.n_pages}};
  for (const Ints& a : in)
    if (!device16(a.p)) return RWTTT_E_INVALID;
  for (const Ints& a : out) {
    if (a.n == 0 && !a.p) continue;      // no map entries, no maps
    if (!device16(a.p)) return RWTTT_E_INVALID;
    for (const Ints& b : in)
      if (overlap(a, b)) return RWTTT_E_INVALID;
    for (const Ints* b = out; b != &a; ++b)
      if (overlap(a, *b)) return RWTTT_E_INVALID;
  }
  const rwttt::KvExtendLaunch L{kv->shape, have,  want,  pos,    kv->cfg.table, kv->cfg.ring, new_pos, lengths,
                                start,     slots, owners, positions, result,      cap};
  return hip_result(kv, rwttt::launch_kv_extend(L, static_cast<hipStream_t>(stream)));
}

rwttt_status rwttt_kv_append(rwttt_kv* kv, uint32_t layer, const void* k, uint64_t k_stride, const void* v,
                             uint64_t v_stride, const int32_t* slots, uint32_t n, void* stream) {
  if (!kv || layer >= kv->cfg.n_layers || kv->k.empty()) return RWTTT_E_INVALID;
  if (n == 0) return RWTTT_OK;
  if (n > (1u << 24) || !device16(k) || !device16(v) || !device16(slots)) return RWTTT_E_INVALID;
  if (!stride_ok(kv, k_stride, kv->cfg.n_kv_heads) || !stride_ok(kv, v_stride, kv->cfg.n_kv_heads))
    return RWTTT_E_INVALID;
  rwttt::KvAppendLaunch L;
  L.s = kv->shape;
  L.k_new = k;
  L.v_new = v;
  L.k_stride = k_stride;
  L.v_stride = v_stride;
  L.k = kv->k[layer];
  L.v = kv->v[layer];
  L.bounds = kv->bounds.empty() ? nullptr : static_cast<int8_t*>(kv->bounds[layer]);
  L.k_scale = head_scale(kv, kv->cfg.k_scale, layer);
  L.v_scale = head_scale(kv, kv->cfg.v_scale, layer);
  L.step = head_scale(kv, kv->cfg.bound_step, layer);
  L.slots = slots;
  L.n = n;
  return hip_result(kv, rwttt::launch_kv_append(L, static_cast<hipStream_t>(stream)));
}

rwttt_status rwttt_kv_gather(rwttt_kv* kv, uint32_t layer, const int32_t* owners, const int32_t* positions,
                             const int32_t* lengths, uint32_t n, void* k, uint64_t k_stride, void* v,
                             uint64_t v_stride, void* stream) {
  if (!kv || layer >= kv->cfg.n_layers || kv->k.empty() || !kv->cfg.table) return RWTTT_E_INVALID;
  if (n == 0) return RWTTT_OK;
  if (n > (1u << 24) || !device16(owners) || !device16(positions) || !device16(lengths)) return RWTTT_E_INVALID;
  if (!k && !v) return RWTTT_E_INVALID;
  const uint32_t heads = kv->cfg.n_kv_heads;
  if (k && (misaligned(k, 16) || !stride_ok(kv, k_stride, heads))) return RWTTT_E_INVALID;
  if (v && (misaligned(v, 16) || !stride_ok(kv, v_stride, heads))) return RWTTT_E_INVALID;
  const uint64_t row = uint64_t(heads) * kv->cfg.head_dim;
  const uint64_t io_bytes = type_bytes(kv->cfg.io_dtype);
  if (k && v && overlap(Rows{k, k_stride, row}, Rows{v, v_stride, row}, n, io_bytes)) return RWTTT_E_INVALID;
  const Span read[] = {{owners, n * 4ull},
                       {positions, n * 4ull},
                       {lengths, kv->cfg.n_owners * 4ull},
                       {kv->cfg.table, uint64_t(kv->cfg.n_owners) * kv->cfg.max_pages * 4},
                       {kv->k[layer], layer_bytes(kv->cfg)},
                       {kv->v[layer], layer_bytes(kv->cfg)},
                       {head_scale(kv, kv->cfg.k_scale, layer), heads * 4ull},
                       {head_scale(kv, kv->cfg.v_scale, layer), heads * 4ull}};
  for (const Span& a : read)
    if ((k && overlap(Rows{k, k_stride, row}, n, io_bytes, a)) || (v && overlap(Rows{v, v_stride, row}, n, io_bytes, a)))
      return RWTTT_E_INVALID;
  rwttt::KvGatherLaunch L;
  L.s = kv->shape;
  L.k = kv->k[layer];
  L.v = kv->v[layer];
  L.k_scale = head_scale(kv, kv->cfg.k_scale, layer);
  L.v_scale = head_scale(kv, kv->cfg.v_scale, layer);
  L.table = kv->cfg.table;
  L.owners = owners;
  L.positions = positions;
  L.lengths = lengths;
  L.n = n;
  L.k_out = k;
  L.v_out = v;
  L.k_stride = k_stride;
  L.v_stride = v_stride;
  return hip_result(kv, rwttt::launch_kv_gather(L, static_cast<hipStream_t>(stream)));
}

rwttt_status rwttt_kv_select(rwttt_kv* kv, uint32_t layer, const void* q, uint64_t q_stride,
                             const int32_t* lengths, const int32_t* rows, uint32_t n, uint32_t first,
                             uint32_t last, uint32_t keep, int32_t* pages, void* stream) {
  if (!queries_ok(kv, layer, q, q_stride, lengths, rows, n) || kv->bounds.empty()) return RWTTT_E_INVALID;
  if (keep == 0 || keep > kv->cfg.max_pages + RWTTT_KV_MAX_SELECT || uint64_t(first) + last > keep)
    return RWTTT_E_INVALID;
  if (!device16(pages)) return RWTTT_E_INVALID;
  if (kv->cfg.max_pages > RWTTT_KV_MAX_SELECT) return RWTTT_E_CAPACITY;
  if (n == 0) return RWTTT_OK;
  const rwttt::KvSelectLaunch L{kv->shape,      q,       q_stride, static_cast<const int8_t*>(kv->bounds[layer]),
                                kv->cfg.table, lengths, rows,     n,
                                first,          last,    keep,     pages,
                                kv->cfg.workspace};
  return hip_result(kv, rwttt::launch_kv_select(L, static_cast<hipStream_t>(stream)));
}

rwttt_status rwttt_kv_attend(rwttt_kv* kv, uint32_t layer, const void* q, uint64_t q_stride,
                             const int32_t* lengths, const int32_t* rows, uint32_t n, float scale,
                             uint32_t window, const int32_t* pages, uint32_t keep, void* out,
                             uint64_t out_stride, float* lse, void* stream) {
  if (!queries_ok(kv, layer, q, q_stride, lengths, rows, n) || kv->k.empty() || !kv->cfg.workspace)
    return RWTTT_E_INVALID;
  if (!device16(out) || !stride_ok(kv, out_stride, kv->cfg.n_heads) || misaligned(lse, 16))
    return RWTTT_E_INVALID;
  if (misaligned(pages, 16) || (pages ? keep == 0 || window != 0 : keep != 0)) return RWTTT_E_INVALID;
  if (window > RWTTT_KV_MAX_ROWS) window = 0;           // wider than any cache: all rows
  if (keep > kv->cfg.max_pages + RWTTT_KV_MAX_SELECT) return RWTTT_E_INVALID;
  if (n == 0) return RWTTT_OK;
  rwttt::KvAttendLaunch L;
  L.s = kv->shape;
  L.q = q;
  L.k = kv->k[layer];
  L.v = kv->v[layer];
  L.k_scale = head_scale(kv, kv->cfg.k_scale, layer);
  L.v_scale = head_scale(kv, kv->cfg.v_scale, layer);
  L.q_stride = q_stride;
  L.out_stride = out_stride;
  L.table = kv->cfg.table;
  L.lengths = lengths;
  L.rows = rows;
  L.pages = pages;
  L.n = n;
  L.n_layers = kv->cfg.n_layers;
  L.window = window;
  L.keep = keep;
  L.scale = scale;
  L.out = out;
  L.lse = lse;
  L.workspace = kv->cfg.workspace;
  return hip_result(kv, rwttt::launch_kv_attend(L, static_cast<hipStream_t>(stream)));
}

rwttt_status rwttt_kv_turns(uint32_t turning, double base, int32_t scaling, double factor, double low, double high,
                            double context, uint64_t* turns) {
  if (!turns || turning == 0 || turning % 2 || turning > 256 || !std::isfinite(base) || base <= 1.0)
    return RWTTT_E_INVALID;
  if (scaling < RWTTT_ROTARY_PLAIN || scaling > RWTTT_ROTARY_PARTS) return RWTTT_E_INVALID;
  if (scaling != RWTTT_ROTARY_PLAIN && (!std::isfinite(factor) || factor <= 0.0)) return RWTTT_E_INVALID;
  if (scaling == RWTTT_ROTARY_BASE && turning == 2) return RWTTT_E_INVALID;
  if (scaling == RWTTT_ROTARY_PARTS && (!std::isfinite(low) || !std::isfinite(high) || !std::isfinite(context) ||
                                        context <= 0.0 || high <= low))
    return RWTTT_E_INVALID;
  // long double: 64 bits of mantissa, as many as a turn is divided into
  const long double two_pi = 6.283185307179586476925286766559005768L, d = turning, f = factor;
  const long double b = scaling == RWTTT_ROTARY_BASE ? base * powl(f, d / (d - 2)) : static_cast<long double>(base);
  for (uint32_t i = 0; i < turning / 2; ++i) {
    long double t = powl(b, -2.0L * i / d) / two_pi;            // turns a position
    if (scaling == RWTTT_ROTARY_LINEAR) t /= f;
    if (scaling == RWTTT_ROTARY_PARTS) {
      long double r = (context * t - low) / (static_cast<long double>(high) - low);
      r = r < 0 ? 0 : r > 1 ? 1 : r;
      t = t * (r + (1 - r) / f);
    }
    t -= floorl(t);                                             // whole turns do not count
    const long double units = rintl(ldexpl(t, 64));
    turns[i] = units >= 0x1p64L ? 0 : static_cast<uint64_t>(units);
  }
  return RWTTT_OK;
}

rwttt_status rwttt_kv_rotate(rwttt_kv* kv, const rwttt_kv_rotary* rotary, const int32_t* positions, uint32_t n,
                             const void* q, uint64_t q_stride, void* q_out, uint64_t q_out_stride, const void* k,
                             uint64_t k_stride, void* k_out, uint64_t k_out_stride, void* stream) {
  if (!kv || !rotary) return RWTTT_E_INVALID;
  const rwttt_kv_config& c = kv->cfg;
  if (rotary->turning == 0 || rotary->turning % 2 || rotary->turning > c.head_dim) return RWTTT_E_INVALID;
  if (rotary->layout != RWTTT_ROTARY_HALF && rotary->layout != RWTTT_ROTARY_INTERLEAVED) return RWTTT_E_INVALID;
  if (!std::isfinite(rotary->gain) || (rotary->inverse != 0 && rotary->inverse != 1) || !device16(rotary->turns))
    return RWTTT_E_INVALID;
  if (n == 0) return RWTTT_OK;
  if (n > (1u << 24) || !device16(positions) || (!q && !k)) return RWTTT_E_INVALID;
  const uint64_t bytes = type_bytes(c.io_dtype);
  struct Side {
    const void* in;
    uint64_t stride;
    void* out;
    uint64_t out_stride;
    uint32_t heads;
  };
  const Side sides[] = {{q, q_stride, q_out, q_out_stride, c.n_heads}, {k, k_stride, k_out, k_out_stride, c.n_kv_heads}};
  for (const Side& a : sides) {
    if ((a.in == nullptr) != (a.out == nullptr)) return RWTTT_E_INVALID;
    if (!a.in) continue;
    if (misaligned(a.in, 16) || misaligned(a.out, 16) || !stride_ok(kv, a.stride, a.heads) ||
        !stride_ok(kv, a.out_stride, a.heads))
      return RWTTT_E_INVALID;
  }
  for (const Side& a : sides)
    for (const Side& b : sides) {
      if (!a.in || !b.in) continue;
      const uint64_t row_a = uint64_t(a.heads) * c.head_dim, row_b = uint64_t(b.heads) * c.head_dim;
      const Rows out{a.out, a.out_stride, row_a};
      const bool itself = &a == &b && a.in == a.out && a.stride == a.out_stride;
      if (!itself && overlap(out, Rows{b.in, b.stride, row_b}, n, bytes)) return RWTTT_E_INVALID;
      if (&a != &b && overlap(out, Rows{b.out, b.out_stride, row_b}, n, bytes)) return RWTTT_E_INVALID;
    }
  const Span read[] = {{positions, n * 4ull}, {rotary->turns, rotary->turning / 2 * 8ull}};
  for (const Side& a : sides)
    for (const Span& b : read)
      if (a.in && overlap(Rows{a.out, a.out_stride, uint64_t(a.heads) * c.head_dim}, n, bytes, b)) return RWTTT_E_INVALID;
  rwttt::KvRotateLaunch L;
  L.io_bf16 = kv->shape.io_bf16;
  L.head_dim = kv->shape.head_dim;
  L.turning = int(rotary->turning);
  L.interleaved = rotary->layout == RWTTT_ROTARY_INTERLEAVED;
  L.inverse = rotary->inverse;
  L.gain = rotary->gain;
  L.turns = rotary->turns;
  L.positions = positions;
  L.n = n;
  L.q = {q, q_out, q_stride, q_out_stride, q ? int(c.n_heads) : 0};
  L.k = {k, k_out, k_stride, k_out_stride, k ? int(c.n_kv_heads) : 0};
  return hip_result(kv, rwttt::launch_kv_rotate(L, static_cast<hipStream_t>(stream)));
}

int32_t rwttt_kv_last_hip_error(const rwttt_kv* kv) { return kv ? kv->last_hip : 0; }

}  // extern "C"
