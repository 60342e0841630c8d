// Host side of the dense attention and cache entry points: argument checks,
// workspace layout and launches.
#include <math.h>

#include <algorithm>

#include "dense.h"
#include "kernels.h"

namespace park {

static bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

// Checks a view of [B][H][N][d] elements of `es` bytes and gives its strides in
// bytes (0 for dimensions of at most one element).
static park_status check_rows(const park_rows* t, int B, int H, int N, int d, size_t es, bool out,
                              const char* what, RowsArg* r) {
  if (!t) return fail(PARK_ERR_INVALID_ARG, "%s is NULL", what);
  *r = {(char*)t->data, 0, 0, 0};
  if (H == 0 || N == 0) return PARK_OK;
  if (!t->data) return fail(PARK_ERR_INVALID_ARG, "%s has no data", what);
  if (!aligned16(t->data)) return fail(PARK_ERR_INVALID_ARG, "%s is not 16-byte aligned", what);
  const int64_t stride[3] = {t->batch, t->head, t->row};
  const int64_t size[3] = {B, H, N};
  int64_t bytes[3];
  for (int i = 0; i < 3; ++i) {
    bytes[i] = 0;
    if (size[i] <= 1) continue;
    if (stride[i] < 0 || stride[i] >= (int64_t)1 << 46)
      return fail(PARK_ERR_INVALID_ARG, "%s: stride %lld", what, (long long)stride[i]);
    bytes[i] = stride[i] * (int64_t)es;
    if (bytes[i] & 15)
      return fail(PARK_ERR_INVALID_ARG, "%s: stride %lld is no multiple of 16 bytes", what,
                  (long long)stride[i]);
  }
  if (size[2] > 1 && stride[2] >= (int64_t)1 << 25)
    return fail(PARK_ERR_UNSUPPORTED, "%s: row stride %lld is not below 2^25", what,
                (long long)stride[2]);
  if (out) {
    // each dimension, from the smallest stride, steps past all before it
    int order[3] = {0, 1, 2};
    std::sort(order, order + 3, [&](int x, int y) { return bytes[x] < bytes[y]; });
    int64_t span = d * (int64_t)es;
    for (int i : order) {
      if (size[i] <= 1) continue;
      if (bytes[i] < span) return fail(PARK_ERR_INVALID_ARG, "%s overlaps itself", what);
      span += (size[i] - 1) * bytes[i];
    }
  }
  r->b = bytes[0];
  r->h = bytes[1];
  r->r = bytes[2];
  return PARK_OK;
}

static park_status check_array(const void* p, const char* what) {
  if (!p) return fail(PARK_ERR_INVALID_ARG, "%s is NULL", what);
  if (!aligned16(p)) return fail(PARK_ERR_INVALID_ARG, "%s is not 16-byte aligned", what);
  return PARK_OK;
}

static park_status check_optional(const void* p, const char* what) {
  if (p && !aligned16(p)) return fail(PARK_ERR_INVALID_ARG, "%s is not 16-byte aligned", what);
  return PARK_OK;
}

static park_status check_attn_dims(const park_attn_dims* m) {
  if (!m) return fail(PARK_ERR_INVALID_ARG, "dims is NULL");
  if (m->B < 1 || m->Hq < 1 || m->Hkv < 1 || m->Nq < 0 || m->Nk < 0)
    return fail(PARK_ERR_INVALID_ARG, "need B, Hq, Hkv >= 1 and Nq, Nk >= 0");
  if (m->Hq % m->Hkv)
    return fail(PARK_ERR_INVALID_ARG, "Hkv = %d does not divide Hq = %d", m->Hkv, m->Hq);
  if (m->d != 64 && m->d != 128)
    return fail(PARK_ERR_UNSUPPORTED, "head dimension %d not supported (64 or 128)", m->d);
  if (m->dtype != PARK_F32 && m->dtype != PARK_BF16)
    return fail(PARK_ERR_INVALID_ARG, "unknown dtype %d", m->dtype);
  if (m->out_dtype != PARK_F32 && m->out_dtype != PARK_BF16)
    return fail(PARK_ERR_INVALID_ARG, "unknown out_dtype %d", m->out_dtype);
  const int64_t most = (int64_t)1 << 30;
  if ((int64_t)m->Nq * (m->Hq / m->Hkv) >= most || m->Nk >= most)
    return fail(PARK_ERR_UNSUPPORTED, "Nq Hq / Hkv and Nk must be below 2^30");
  // (a launch has below 2^32 threads, 256 for every 32 rows at the most)
  const int64_t heads = (int64_t)m->B * m->Hkv;
  if (heads * (dense_tiles((int64_t)m->Nq * (m->Hq / m->Hkv)) + 1) > (int64_t)1 << 24 ||
      heads * (dense_tiles(m->Nk) + 1) > (int64_t)1 << 24 || (int64_t)m->B * m->Hq >= (int64_t)1 << 24)
    return fail(PARK_ERR_UNSUPPORTED,
                "more than 2^24 tiles of 32 rows over all heads, or B Hq not below 2^24");
  return PARK_OK;
}

static park_status check_opts(const park_attn_opts* o, int Nq, int Nk) {
  if (!o) return fail(PARK_ERR_INVALID_ARG, "opts is NULL");
  if (!(o->scale > 0.0 && o->scale <= 1048576.0) || (float)o->scale < 1e-30f)
    return fail(PARK_ERR_INVALID_ARG, "scale %g must be in [1e-30, 2^20]", o->scale);
  if (o->softcap != 0.0 && !(o->softcap >= 1e-30 && o->softcap <= 1e30))
    return fail(PARK_ERR_INVALID_ARG, "softcap %g must be 0 or in [1e-30, 1e30]", o->softcap);
  if (o->softcap > o->scale * 0x1p126)  // (scale / softcap is a float of its full precision)
    return fail(PARK_ERR_INVALID_ARG, "softcap %g is above 2^126 scale (%g)", o->softcap, o->scale);
  if (o->causal != 0 && o->causal != 1)
    return fail(PARK_ERR_INVALID_ARG, "causal = %d must be 0 or 1", o->causal);
  if (o->q_pos <= -(1 << 30) || o->q_pos >= (1 << 30))
    return fail(PARK_ERR_INVALID_ARG, "q_pos = %d out of range", o->q_pos);
  if (o->prefix && !o->causal) return fail(PARK_ERR_INVALID_ARG, "prefix without causal");
  PARK_TRY(check_optional(o->slopes, "slopes"));
  PARK_TRY(check_optional(o->prefix, "prefix"));
  PARK_TRY(check_optional(o->q_doc, "q_doc"));
  PARK_TRY(check_optional(o->k_doc, "k_doc"));
  if (Nq > 0 && Nk > 0 && (o->q_doc == nullptr) != (o->k_doc == nullptr))
    return fail(PARK_ERR_INVALID_ARG, "q_doc and k_doc come together");
  return PARK_OK;
}

static park_status check_space(void* ws, size_t ws_bytes, size_t need) {
  if (need == 0) return PARK_OK;
  PARK_TRY(check_array(ws, "workspace"));
  if (ws_bytes < need)
    return fail(PARK_ERR_WORKSPACE, "workspace of %zu bytes is smaller than the %zu required",
                ws_bytes, need);
  return PARK_OK;
}

static DenseArgs dense_args(const park_attn_dims& m, const park_attn_opts& o) {
  DenseArgs a = {};
  a.B = m.B;
  a.Hkv = m.Hkv;
  a.G = m.Hq / m.Hkv;
  a.Nq = m.Nq;
  a.Nk = m.Nk;
  a.R = m.Nq * a.G;
  // the least multiplier above 2^(31 + gshift) / G, 2^(gshift - 1) < G <= 2^gshift
  while ((1 << a.gshift) < a.G) ++a.gshift;
  a.gmul = (uint32_t)((((uint64_t)1 << (31 + a.gshift)) + a.G - 1) / a.G);
  a.causal = o.causal;
  a.q_pos = o.q_pos;
  a.prefix = o.prefix;
  a.slopes = o.slopes;
  a.scale = (float)o.scale;
  a.cap = (float)o.softcap;
  const double arg = o.softcap > 0.0 ? o.scale / o.softcap : 0.0;
  a.cap_arg = (float)arg;
  a.cap_exp = (float)(2.8853900817779268 * arg);
  a.cap_small = (float)(0.3125 / fabs(arg));
  a.out_f32 = m.out_dtype == PARK_F32;
  return a;
}

static int64_t held_tiles(int64_t heads, int64_t rows) {
  return (rows + DENSE_ROWS - 1) / DENSE_ROWS * heads;
}
static int64_t packed_rows(const park_attn_dims& m) { return (int64_t)m.Nq * (m.Hq / m.Hkv); }
static int64_t heads_of(const park_attn_dims& m) { return (int64_t)m.B * m.Hkv; }

static void carve_splits(Carver& cv, const park_attn_dims& m, DenseArgs& a) {
  const size_t rows = a.split.rows(packed_rows(m) <= DENSE_FEW ? 32 : DENSE_ROWS);
  if (!rows) return;
  a.part = cv.take<float>(rows * m.d);
  a.ml = cv.take<float2>(rows);
}

// forward: document tiles of the keys, then the split tiles' sums
static size_t carve_forward(Carver& cv, const park_attn_dims& m, const park_attn_opts& o, bool docs,
                            DenseArgs& a) {
  if (docs) a.k_tiles = cv.take<DocTile>((size_t)m.B * dense_tiles(m.Nk));
  a.split = dense_fwd_split(packed_rows(m), heads_of(m), dense_tiles(m.Nk), m.d, m.dtype, false, docs,
                            o.causal != 0);
  carve_splits(cv, m, a);
  return cv.off;
}

static size_t carve_backward(Carver& cv, const park_attn_dims& m, const park_attn_opts& o, bool docs,
                             DenseArgs& a, DenseGrad& g) {
  const int64_t R = packed_rows(m);
  const bool f32 = m.dtype == PARK_F32, causal = o.causal != 0;
  g.rows = cv.take<float>((size_t)heads_of(m) * dense_tiles(R) * DENSE_RF * 32);
  if (docs) {
    a.k_tiles = cv.take<DocTile>((size_t)m.B * dense_tiles(m.Nk));
    g.q_tiles = cv.take<DocTile>((size_t)m.B * dense_tiles(R));
  }
  // (dQ of 64-wide rows: three workgroups a CU; 8 heads of 4500 rows 182 -> 125 us)
  g.qsplit = dense_split(held_tiles(heads_of(m), R), dense_tiles(m.Nk), f32, docs, causal,
                         !f32 && m.d == 64 ? 3 : 2, 3);
  g.ksplit = dense_split(held_tiles(heads_of(m), m.Nk), dense_tiles(R), f32, docs, causal, 2, 3);
  // (one after the other)
  const size_t rows = std::max(g.qsplit.rows(DENSE_ROWS), 2 * g.ksplit.rows(DENSE_ROWS));
  if (rows) g.part = cv.take<float>(rows * m.d);
  return cv.off;
}

static park_status check_cache(const park_kv_cache* c) {
  if (!c) return fail(PARK_ERR_INVALID_ARG, "cache is NULL");
  if (c->n_pages < 1 || c->Hkv < 1)
    return fail(PARK_ERR_INVALID_ARG, "need n_pages >= 1 and Hkv >= 1");
  if (c->page != 16 && c->page != 32 && c->page != 64 && c->page != 128)
    return fail(PARK_ERR_UNSUPPORTED, "pages of %d tokens not supported (16, 32, 64 or 128)", c->page);
  if (c->d != 64 && c->d != 128)
    return fail(PARK_ERR_UNSUPPORTED, "head dimension %d not supported (64 or 128)", c->d);
  return PARK_OK;
}

static park_status check_cache_data(const park_kv_cache* c) {
  PARK_TRY(check_array(c->k, "cache k"));
  PARK_TRY(check_array(c->v, "cache v"));
  PARK_TRY(check_array(c->k_exp, "cache k_exp"));
  PARK_TRY(check_array(c->v_exp, "cache v_exp"));
  return check_optional(c->status, "cache status");
}

// Splits of the cache: as many as fill the chip at the longest sequence, and
// enough that the pages of one fit its table.
static park_status cache_splits(const park_kv_cache& c, const park_attn_dims& m, int max_pages,
                                DenseSplit* split) {
  const int64_t tiles = dense_tiles((int64_t)max_pages * c.page);
  DenseSplit sp =
      dense_fwd_split(packed_rows(m), heads_of(m), tiles, m.d, m.dtype, true, true, false);
  auto pages = [&](int64_t k) { return (tiles + k - 1) / k * 32 / c.page + 2; };
  if (pages(sp.whole ? 1 : sp.n) > DENSE_PAGES) {
    sp = {0, (int)(sp.whole + sp.rest), sp.n};
    while (sp.n < DENSE_MAXSPLIT && pages(sp.n) > DENSE_PAGES) ++sp.n;
    if (pages(sp.n) > DENSE_PAGES)
      return fail(PARK_ERR_UNSUPPORTED, "max_pages = %d pages of %d tokens exceed %d pages a part",
                  max_pages, c.page, DENSE_PAGES);
  }
  // (a launch joins them, up to 32 lanes a row)
  if ((int64_t)sp.rest * (packed_rows(m) > DENSE_FEW ? DENSE_ROWS : 32) > (int64_t)1 << 25)
    return fail(PARK_ERR_UNSUPPORTED, "more than 2^25 rows take their pages in parts");
  *split = sp;
  return PARK_OK;
}

static park_status check_cache_dims(const park_kv_cache* c, const park_attn_dims* m, int max_pages,
                                    park_attn_dims* out) {
  PARK_TRY(check_cache(c));
  if (!m) return fail(PARK_ERR_INVALID_ARG, "dims is NULL");
  *out = *m;
  out->Nk = 0;
  PARK_TRY(check_attn_dims(out));
  if (m->Hkv != c->Hkv || m->d != c->d)
    return fail(PARK_ERR_INVALID_ARG, "dims have Hkv = %d, d = %d, the cache %d, %d", m->Hkv, m->d,
                c->Hkv, c->d);
  if (m->dtype != PARK_BF16) return fail(PARK_ERR_UNSUPPORTED, "queries of a cache are bf16");
  if (max_pages < 1 || (int64_t)max_pages * c->page >= (int64_t)1 << 30)
    return fail(PARK_ERR_INVALID_ARG, "max_pages = %d (at least 1, below 2^30 tokens)", max_pages);
  return PARK_OK;
}

}  // namespace park

using namespace park;

extern "C" {

park_status park_attention_workspace_size(const park_attn_dims* dims, const park_attn_opts* opts,
                                          int32_t backward, size_t* bytes) {
  clear_error();
  PARK_TRY(check_attn_dims(dims));
  if (!opts || !bytes) return fail(PARK_ERR_INVALID_ARG, "opts or bytes is NULL");
  DenseArgs a = {};
  DenseGrad g = {};
  Carver cv(nullptr);
  const bool docs = opts->q_doc && dims->Nq > 0 && dims->Nk > 0;
  *bytes = backward ? carve_backward(cv, *dims, *opts, docs, a, g)
                    : carve_forward(cv, *dims, *opts, docs, a);
  return PARK_OK;
}

park_status park_attention(const park_rows* Q, const park_rows* K, const park_rows* V,
                           const park_attn_dims* m, const park_attn_opts* o, const park_rows* O,
                           float* lse, void* ws, size_t ws_bytes, void* stream) {
  clear_error();
  PARK_TRY(check_attn_dims(m));
  PARK_TRY(check_opts(o, m->Nq, m->Nk));
  DenseArgs a = dense_args(*m, *o);
  const size_t es = elem_size(m->dtype);
  PARK_TRY(check_rows(Q, m->B, m->Hq, m->Nq, m->d, es, false, "Q", &a.q));
  PARK_TRY(check_rows(K, m->B, m->Hkv, m->Nk, m->d, es, false, "K", &a.k));
  PARK_TRY(check_rows(V, m->B, m->Hkv, m->Nk, m->d, es, false, "V", &a.v));
  PARK_TRY(check_rows(O, m->B, m->Hq, m->Nq, m->d, elem_size(m->out_dtype), true, "O", &a.o));
  PARK_TRY(check_optional(lse, "lse"));
  const bool docs = o->q_doc && m->Nq > 0 && m->Nk > 0;
  Carver size(nullptr);
  DenseArgs unused = a;
  PARK_TRY(check_space(ws, ws_bytes, carve_forward(size, *m, *o, docs, unused)));
  if (m->Nq == 0) return PARK_OK;
  Carver cv(ws);
  carve_forward(cv, *m, *o, docs, a);
  a.lse = lse;
  hipStream_t st = (hipStream_t)stream;
  if (docs) {
    a.q_doc = o->q_doc;
    a.k_doc = o->k_doc;
    PARK_TRY(launch_doc_tiles({a.k_doc, m->Nk, 1, (DocTile*)a.k_tiles}, nullptr, m->B, st));
  }
  return launch_dense_fwd(a, m->d, m->dtype, false, st);
}

park_status park_attention_backward(const park_rows* dO, const park_rows* Q, const park_rows* K,
                                    const park_rows* V, const park_rows* O, const float* lse,
                                    const float* dlse, const park_attn_dims* m,
                                    const park_attn_opts* o, const park_rows* dQ,
                                    const park_rows* dK, const park_rows* dV, void* ws,
                                    size_t ws_bytes, void* stream) {
  clear_error();
  PARK_TRY(check_attn_dims(m));
  PARK_TRY(check_opts(o, m->Nq, m->Nk));
  DenseArgs a = dense_args(*m, *o);
  DenseGrad g = {};
  const size_t es = elem_size(m->dtype);
  PARK_TRY(check_rows(dO, m->B, m->Hq, m->Nq, m->d, es, false, "dO", &g.dout));
  PARK_TRY(check_rows(Q, m->B, m->Hq, m->Nq, m->d, es, false, "Q", &a.q));
  PARK_TRY(check_rows(K, m->B, m->Hkv, m->Nk, m->d, es, false, "K", &a.k));
  PARK_TRY(check_rows(V, m->B, m->Hkv, m->Nk, m->d, es, false, "V", &a.v));
  PARK_TRY(check_rows(O, m->B, m->Hq, m->Nq, m->d, elem_size(m->out_dtype), false, "O", &a.o));
  PARK_TRY(check_rows(dQ, m->B, m->Hq, m->Nq, m->d, es, true, "dQ", &g.dq));
  PARK_TRY(check_rows(dK, m->B, m->Hkv, m->Nk, m->d, es, true, "dK", &g.dk));
  PARK_TRY(check_rows(dV, m->B, m->Hkv, m->Nk, m->d, es, true, "dV", &g.dv));
  if (m->Nq > 0) PARK_TRY(check_array(lse, "lse"));
  PARK_TRY(check_optional(dlse, "dlse"));
  const bool docs = o->q_doc && m->Nq > 0 && m->Nk > 0;
  Carver size(nullptr);
  DenseArgs a2 = a;
  DenseGrad g2 = g;
  PARK_TRY(check_space(ws, ws_bytes, carve_backward(size, *m, *o, docs, a2, g2)));
  Carver cv(ws);
  carve_backward(cv, *m, *o, docs, a, g);
  g.lse = lse;
  g.dlse = dlse;
  g.o_f32 = m->out_dtype == PARK_F32;
  hipStream_t st = (hipStream_t)stream;
  if (docs) {
    a.q_doc = o->q_doc;
    a.k_doc = o->k_doc;
    const DocIds q = {a.q_doc, m->Nq, a.G, (DocTile*)g.q_tiles};
    PARK_TRY(launch_doc_tiles({a.k_doc, m->Nk, 1, (DocTile*)a.k_tiles}, &q, m->B, st));
  }
  return launch_dense_bwd(a, g, m->d, m->dtype, st);
}

park_status park_cache_append(const park_kv_cache* c, const park_rows* K, const park_rows* V,
                              int32_t B, int32_t N, int32_t dtype, const int32_t* block_table,
                              int32_t max_pages, const int32_t* lens, const int32_t* n_new,
                              void* stream) {
  clear_error();
  PARK_TRY(check_cache(c));
  PARK_TRY(check_cache_data(c));
  if (B < 1 || N < 0) return fail(PARK_ERR_INVALID_ARG, "need B >= 1 and N >= 0");
  if (dtype != PARK_F32 && dtype != PARK_BF16)
    return fail(PARK_ERR_INVALID_ARG, "unknown dtype %d", dtype);
  if (max_pages < 1 || (int64_t)max_pages * c->page >= (int64_t)1 << 30 || N >= 1 << 30)
    return fail(PARK_ERR_INVALID_ARG, "max_pages = %d, N = %d (tokens are below 2^30)", max_pages, N);
  const int64_t slots = ((int64_t)N + 2 * c->page - 2) / c->page;
  if ((int64_t)B * c->Hkv * slots >= (int64_t)1 << 24)
    return fail(PARK_ERR_UNSUPPORTED, "B Hkv (N / page + 2) must be below 2^24");
  CacheAppend a = {};
  PARK_TRY(check_rows(K, B, c->Hkv, N, c->d, elem_size(dtype), false, "K", &a.k));
  PARK_TRY(check_rows(V, B, c->Hkv, N, c->d, elem_size(dtype), false, "V", &a.v));
  PARK_TRY(check_array(block_table, "block_table"));
  PARK_TRY(check_array(lens, "lens"));
  PARK_TRY(check_optional(n_new, "n_new"));
  if (N == 0) return PARK_OK;
  a.pk = c->k;
  a.pv = c->v;
  a.k_exp = c->k_exp;
  a.v_exp = c->v_exp;
  a.table = block_table;
  a.lens = lens;
  a.n_new = n_new;
  a.B = B;
  a.Hkv = c->Hkv;
  a.N = N;
  a.d = c->d;
  a.dtype = dtype;
  a.page_shift = __builtin_ctz(c->page);
  a.n_pages = c->n_pages;
  a.max_pages = max_pages;
  a.status = c->status;
  return launch_cache_append(a, (hipStream_t)stream);
}

park_status park_cache_workspace_size(const park_kv_cache* c, const park_attn_dims* dims,
                                      int32_t max_pages, size_t* bytes) {
  clear_error();
  if (!bytes) return fail(PARK_ERR_INVALID_ARG, "bytes is NULL");
  park_attn_dims m;
  PARK_TRY(check_cache_dims(c, dims, max_pages, &m));
  DenseArgs a = {};
  PARK_TRY(cache_splits(*c, m, max_pages, &a.split));
  Carver cv(nullptr);
  carve_splits(cv, m, a);
  *bytes = cv.off;
  return PARK_OK;
}

park_status park_cache_attention(const park_rows* Q, const park_kv_cache* c,
                                 const int32_t* block_table, int32_t max_pages,
                                 const int32_t* lens, const int32_t* q_lens,
                                 const park_attn_dims* dims, const park_attn_opts* o,
                                 const park_rows* O, float* lse, void* ws, size_t ws_bytes,
                                 void* stream) {
  clear_error();
  park_attn_dims m;
  PARK_TRY(check_cache_dims(c, dims, max_pages, &m));
  PARK_TRY(check_cache_data(c));
  PARK_TRY(check_opts(o, m.Nq, 0));
  if (o->q_doc || o->k_doc) return fail(PARK_ERR_UNSUPPORTED, "a cache takes no documents");
  DenseArgs a = dense_args(m, *o);
  PARK_TRY(check_rows(Q, m.B, m.Hq, m.Nq, m.d, 2, false, "Q", &a.q));
  PARK_TRY(check_rows(O, m.B, m.Hq, m.Nq, m.d, elem_size(m.out_dtype), true, "O", &a.o));
  PARK_TRY(check_optional(lse, "lse"));
  PARK_TRY(check_array(block_table, "block_table"));
  PARK_TRY(check_array(lens, "lens"));
  PARK_TRY(check_optional(q_lens, "q_lens"));
  PARK_TRY(cache_splits(*c, m, max_pages, &a.split));
  Carver size(nullptr);
  DenseArgs unused = a;
  carve_splits(size, m, unused);
  PARK_TRY(check_space(ws, ws_bytes, size.off));
  if (m.Nq == 0) return PARK_OK;
  Carver cv(ws);
  carve_splits(cv, m, a);
  a.lse = lse;
  a.k.p = (char*)c->k;
  a.v.p = (char*)c->v;
  a.k_exp = c->k_exp;
  a.v_exp = c->v_exp;
  a.table = block_table;
  a.lens = lens;
  a.q_lens = q_lens;
  a.page_shift = __builtin_ctz(c->page);
  a.n_pages = c->n_pages;
  a.max_pages = max_pages;
  a.status = c->status;
  return launch_dense_fwd(a, m.d, PARK_BF16, true, (hipStream_t)stream);
}

}  // extern "C"
