// C ABI of the key/value cache and the attention over it: host-side
// validation and dispatch.  Every check happens before anything is enqueued.
#include <cmath>

#include "kv.h"

namespace grinqh {

static int resolve_kv(const grinqh_kv_desc* d, KvCache* c) {
  if (!d) return fail(GRINQH_EINVAL, "desc is NULL");
  if (d->format < GRINQH_KV_F16 || d->format > GRINQH_KV_I8)
    return fail(GRINQH_EINVAL, "format=%d is not a known cache format", d->format);
  if (d->heads < 1 || d->heads > 1024) return fail(GRINQH_EINVAL, "heads=%d outside 1..1024", d->heads);
  if (d->head_dim != 64 && d->head_dim != 128)
    return fail(GRINQH_EUNSUPPORTED, "head_dim=%d: only 64 and 128 are implemented", d->head_dim);
  if (d->page < 1 || d->page > (1 << 20) || (d->page & (d->page - 1)))
    return fail(GRINQH_EINVAL, "page=%d is not a power of two in 1..2^20", d->page);
  if (d->n_pages < 1) return fail(GRINQH_EINVAL, "n_pages=%d must be positive", d->n_pages);
  *c = KvCache{};
  c->format = d->format; c->H = d->heads; c->D = d->head_dim; c->n_pages = d->n_pages;
  c->shift = __builtin_ctz((unsigned)d->page);
  // a slot index times the row's bytes stays far inside 64 bits
  if ((__int128)d->n_pages * d->heads * d->page > ((__int128)1 << 52))
    return fail(GRINQH_ESIZE, "the cache's %d pages of %d tokens and %d heads overflow", d->n_pages, d->page, d->heads);
  return GRINQH_OK;
}

static int check_cache(const grinqh_kv_cache* in, KvCache* c) {
  if (!in || !in->k || !in->v) return fail(GRINQH_EINVAL, "the cache and its k and v must not be NULL");
  if (((uintptr_t)in->k | (uintptr_t)in->v) & 15u) return fail(GRINQH_EINVAL, "the cache's k and v must be 16-byte aligned");
  if (c->format == GRINQH_KV_I8) {
    if (!in->k_scale || !in->v_scale) return fail(GRINQH_EINVAL, "an 8-bit cache needs k_scale and v_scale");
    if (((uintptr_t)in->k_scale | (uintptr_t)in->v_scale) & 3u) return fail(GRINQH_EINVAL, "scales must be 4-byte aligned");
  } else if (in->k_scale || in->v_scale) {
    return fail(GRINQH_EINVAL, "k_scale and v_scale must be NULL for a 16-bit cache");
  }
  c->k = (char*)in->k; c->v = (char*)in->v; c->ks = in->k_scale; c->vs = in->v_scale;
  return GRINQH_OK;
}

static int check_batch(const grinqh_kv_batch* in, KvBatch* b) {
  if (!in) return fail(GRINQH_EINVAL, "batch is NULL");
  if (in->B < 0 || in->B > 65535) return fail(GRINQH_EINVAL, "B=%d outside 0..65535", in->B);
  if (in->rows < 0 || in->rows > (1 << 24)) return fail(GRINQH_EINVAL, "rows=%d outside 0..2^24", in->rows);
  *b = KvBatch{in->block_table, in->seq_lens, in->row_offsets, in->B, in->table_width, in->rows};
  if (!b->B || !b->rows) return GRINQH_OK;
  if (in->table_width < 1) return fail(GRINQH_EINVAL, "table_width=%d must be positive", in->table_width);
  if (!b->table || !b->lens || !b->offs)
    return fail(GRINQH_EINVAL, "block_table, seq_lens and row_offsets must not be NULL");
  if (((uintptr_t)b->table | (uintptr_t)b->lens | (uintptr_t)b->offs) & 3u)
    return fail(GRINQH_EINVAL, "block_table, seq_lens and row_offsets must be 4-byte aligned");
  return GRINQH_OK;
}

static int check_rows(const char* name, const grinqh_rows* in, int size, int rows, int heads, int dim, bool written,
                      DenseRows* r) {
  if (!in || !in->data) return fail(GRINQH_EINVAL, "%s must not be NULL", name);
  if ((uintptr_t)in->data & 15u) return fail(GRINQH_EINVAL, "%s must be 16-byte aligned", name);
  // the stride of an axis of one entry says nothing
  const int64_t rs = rows > 1 ? in->row_stride : 0, hs = heads > 1 ? in->head_stride : 0, most = (int64_t)1 << 36;
  if (rs < 0 || hs < 0 || rs > most || hs > most) return fail(GRINQH_EINVAL, "%s: strides outside 0..2^36", name);
  if ((rs * size) % 16 || (hs * size) % 16) return fail(GRINQH_EINVAL, "%s: strides must be multiples of 16 bytes", name);
  // rows of heads, or heads of rows, one after the other
  const bool apart = (hs >= dim || heads == 1) && (rs >= (heads - 1) * hs + dim || rows == 1);
  const bool heads_first = (rs >= dim || rows == 1) && (hs >= (rows - 1) * rs + dim || heads == 1);
  if (written && !apart && !heads_first) return fail(GRINQH_EINVAL, "%s: rows that are written must not overlap", name);
  *r = DenseRows{(char*)in->data, (long)rs, (long)hs};
  return GRINQH_OK;
}

static int type_size(int type) { return type == GRINQH_F32 ? 4 : 2; }

static int resolve_attend(const KvCache& c, const grinqh_attend_desc* d, Attend* a) {
  if (!d) return fail(GRINQH_EINVAL, "attend is NULL");
  if (d->heads < 1 || d->heads % c.H || d->heads > 65535)
    return fail(GRINQH_EINVAL, "query heads=%d must be a positive multiple of the cache's %d, at most 65535", d->heads, c.H);
  if (d->type != GRINQH_F16 && d->type != GRINQH_BF16)
    return fail(GRINQH_EUNSUPPORTED, "type=%d: q and out are GRINQH_F16 or GRINQH_BF16", d->type);
  if ((c.format == GRINQH_KV_F16 && d->type != GRINQH_F16) || (c.format == GRINQH_KV_BF16 && d->type != GRINQH_BF16))
    return fail(GRINQH_EUNSUPPORTED, "type=%d: a 16-bit cache is read by queries of its own type", d->type);
  if (!(d->scale > 0) || !std::isfinite(d->scale)) return fail(GRINQH_EINVAL, "scale must be positive and finite");
  if (d->window < 0 || d->sinks < 0) return fail(GRINQH_EINVAL, "window=%d and sinks=%d must not be negative", d->window, d->sinks);
  if (d->max_rows < 1 || d->max_len < 1)
    return fail(GRINQH_EINVAL, "max_rows=%d and max_len=%d must be positive", d->max_rows, d->max_len);
  // no length passes kMaxTokens: a window of that many tokens hides nothing
  const int window = d->window < kMaxTokens ? d->window : 0;
  const int sinks = window ? (int)(d->sinks < kMaxTokens ? d->sinks : kMaxTokens) : 0;
  *a = Attend{d->heads, d->heads / c.H, d->type, d->scale, window, sinks, d->max_rows, d->max_len};
  return GRINQH_OK;
}

// The arguments that writing and reading share.
static int dense_checks(const grinqh_kv_desc* desc, const grinqh_kv_cache* cache, const grinqh_kv_batch* batch, int type,
                        const grinqh_rows* k, const grinqh_rows* v, bool written, KvCache* c, KvBatch* b, DenseRows* kr,
                        DenseRows* vr) {
  int st = resolve_kv(desc, c);
  if (st) return st;
  if (type < GRINQH_F16 || type > GRINQH_F32) return fail(GRINQH_EINVAL, "type=%d is not a known type", type);
  if ((st = check_cache(cache, c)) || (st = check_batch(batch, b))) return st;
  if (!b->B || !b->rows) return GRINQH_OK;
  if ((st = check_rows("k", k, type_size(type), b->rows, c->H, c->D, written, kr))) return st;
  return check_rows("v", v, type_size(type), b->rows, c->H, c->D, written, vr);
}

}  // namespace grinqh

using namespace grinqh;

extern "C" {

int grinqh_kv_bytes(const grinqh_kv_desc* desc, size_t* value_bytes, size_t* scale_bytes) {
  clear_error();
  KvCache c;
  int st = resolve_kv(desc, &c);
  if (st) return st;
  if (!value_bytes || !scale_bytes) return fail(GRINQH_EINVAL, "output pointers are NULL");
  const size_t slots = ((size_t)c.n_pages * c.H) << c.shift;
  *value_bytes = slots * c.D * (c.format == GRINQH_KV_I8 ? 1 : 2);
  *scale_bytes = c.format == GRINQH_KV_I8 ? slots * 4 : 0;
  return GRINQH_OK;
}

int grinqh_kv_write(const grinqh_kv_desc* desc, const grinqh_kv_cache* cache, const grinqh_kv_batch* batch, int type,
                    const grinqh_rows* k, const grinqh_rows* v, void* stream) {
  clear_error();
  KvCache c;
  KvBatch b;
  DenseRows kr, vr;
  int st = dense_checks(desc, cache, batch, type, k, v, false, &c, &b, &kr, &vr);
  if (st || !b.B || !b.rows) return st;
  return launch_kv_write(c, b, type, kr, vr, (hipStream_t)stream);
}

int grinqh_kv_read(const grinqh_kv_desc* desc, const grinqh_kv_cache* cache, const grinqh_kv_batch* batch, int type,
                   const grinqh_rows* k, const grinqh_rows* v, void* stream) {
  clear_error();
  KvCache c;
  KvBatch b;
  DenseRows kr, vr;
  int st = dense_checks(desc, cache, batch, type, k, v, true, &c, &b, &kr, &vr);
  if (st || !b.B || !b.rows) return st;
  return launch_kv_read(c, b, type, kr, vr, (hipStream_t)stream);
}

// Rows times heads, and the rows of a kv head rounded up to a workgroup's, fit 32 bits.
static int check_attend_rows(const Attend& a, int rows) {
  if ((int64_t)rows * a.heads > (1 << 30))
    return fail(GRINQH_ESIZE, "rows=%d of %d heads are more than 2^30", rows, a.heads);
  return GRINQH_OK;
}

int grinqh_attend_workspace_bytes(const grinqh_kv_desc* desc, const grinqh_attend_desc* attend, int32_t B, int32_t rows,
                                  size_t* bytes) {
  clear_error();
  KvCache c;
  Attend a;
  int st = resolve_kv(desc, &c);
  if (st || (st = resolve_attend(c, attend, &a))) return st;
  if (B < 0 || B > 65535) return fail(GRINQH_EINVAL, "B=%d outside 0..65535", B);
  if (rows < 0 || rows > (1 << 24)) return fail(GRINQH_EINVAL, "rows=%d outside 0..2^24", rows);
  if ((st = check_attend_rows(a, rows))) return st;
  if (!bytes) return fail(GRINQH_EINVAL, "bytes is NULL");
  *bytes = B && rows ? attend_workspace(c, a, B, rows) : 0;
  return GRINQH_OK;
}

int grinqh_attend(const grinqh_kv_desc* desc, const grinqh_kv_cache* cache, const grinqh_kv_batch* batch,
                  const grinqh_attend_desc* attend, const grinqh_rows* q, const grinqh_rows* out, float* lse,
                  void* workspace, size_t ws_bytes, void* stream) {
  clear_error();
  KvCache c;
  KvBatch b;
  Attend a;
  DenseRows qr, outr;
  int st = resolve_kv(desc, &c);
  if (st || (st = resolve_attend(c, attend, &a)) || (st = check_cache(cache, &c)) || (st = check_batch(batch, &b))) return st;
  if (!b.B || !b.rows) return GRINQH_OK;
  if ((st = check_attend_rows(a, b.rows))) return st;
  if ((st = check_rows("q", q, 2, b.rows, a.heads, c.D, false, &qr))) return st;
  if ((st = check_rows("out", out, 2, b.rows, a.heads, c.D, true, &outr))) return st;
  if ((uintptr_t)lse & 3u) return fail(GRINQH_EINVAL, "lse must be 4-byte aligned");
  const size_t need = attend_workspace(c, a, b.B, b.rows);
  if (need && !workspace) return fail(GRINQH_EINVAL, "workspace is NULL, %zu bytes are needed", need);
  if (need && ((uintptr_t)workspace & 15u)) return fail(GRINQH_EINVAL, "workspace must be 16-byte aligned");
  if (ws_bytes < need) return fail(GRINQH_ESIZE, "workspace of %zu bytes, %zu are needed", ws_bytes, need);
  return launch_attend(c, b, a, qr, outr, lse, workspace, (hipStream_t)stream);
}

}  // extern "C"
