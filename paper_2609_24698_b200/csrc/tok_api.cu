// C-ABI front end of the token-level and page operators: argument validation on the host, then their kernels.
#include <math.h>

#include "kernels.h"

namespace tsv {

static inline bool al(const void* p, int n) { return ((uintptr_t)p & (n - 1)) == 0; }

static bool tok_shape_ok(const tsv_tok_shape* s) {
  if (s->dtype != TSV_FP32 && s->dtype != TSV_BF16) return false;
  if (s->B < 1 || s->B > 1 << 20 || s->H < 1 || s->H > 256 || s->Hk < 1 || s->H % s->Hk) return false;
  if (s->d < 8 || s->d > 512 || s->d % 8) return false;
  if (s->window < 1 || s->n_sink < 0 || s->max_n < 1 || s->max_n > 1 << 22) return false;      // (rows of a sequence: below 2^31)
  return s->max_L >= 1 && s->max_L <= (int64_t)1 << 30;
}

static tsv_tok_shape resolved(const tsv_tok_shape* s) {
  tsv_tok_shape r = *s;
  if (!(r.sm_scale > 0.f)) r.sm_scale = (float)(1.0 / sqrt((double)r.d));
  return r;
}

static int check_batch(const tsv_tok_batch* b) {
  if (!b || !b->row0 || !b->n) return TSV_ERR_NULL;
  return b->rows < 0 || b->rows > (int64_t)1 << 40 ? TSV_ERR_SHAPE : TSV_OK;
}

// A strided vector array: NULL is the caller's matter.
static int check_rows(const tsv_tok_shape* s, const void* p, int64_t ld, int heads) {
  const int ve = s->dtype == TSV_BF16 ? 8 : 4;
  if (!al(p, 16)) return TSV_ERR_ALIGN;
  if (ld < (int64_t)heads * s->d) return TSV_ERR_SHAPE;
  return ld % ve ? TSV_ERR_ALIGN : TSV_OK;
}

// Do heads of rows rows, ld elements apart, share bytes with [out, out + bytes)?
static bool meets(const tsv_tok_shape* s, const void* out, int64_t bytes, const void* p, int64_t ld, int heads, int64_t rows) {
  const int64_t es = s->dtype == TSV_BF16 ? 2 : 4, span = ((rows - 1) * ld + (int64_t)heads * s->d) * es;
  const char *a = (const char*)out, *b = (const char*)p;
  return p && a < b + span && b < a + bytes;
}

// Do two arrays of `rows` rows share an element?  Of `heads` vectors each, ld elements from row to row; rows of one and the same stride may lie
// between each other's (column ranges of one array), others not.
static bool rows_meet(const tsv_tok_shape* s, const void* p, int64_t ld, int heads, const void* q, int64_t qld, int qheads, int64_t rows) {
  if (!p || !q || rows < 1) return false;
  const int64_t es = s->dtype == TSV_BF16 ? 2 : 4, w = (int64_t)heads * s->d * es, qw = (int64_t)qheads * s->d * es;
  if (!meets(s, p, (rows - 1) * ld * es + w, q, qld, qheads, rows)) return false;
  if (ld != qld || rows == 1) return true;
  const int64_t stride = ld * es;
  int64_t m = ((int64_t)(uintptr_t)q - (int64_t)(uintptr_t)p) % stride;
  if (m < 0) m += stride;
  return m < w || m + qw > stride;                       // (q's rows begin m bytes behind p's)
}

static int check_tok_cache(const tsv_tok_cache* c, const tsv_tok_shape* s) {
  if (!c || !c->L || !c->k) return TSV_ERR_NULL;
  if (!al(c->k, 16) || !al(c->v, 16)) return TSV_ERR_ALIGN;
  if (c->page_table) {
    if (c->page_tokens < 1 || c->page_tokens > 1 << 20 || c->max_pages < 1 || c->rows < 1) return TSV_ERR_SHAPE;
  } else if (c->rows < (int64_t)s->B * ((int64_t)s->n_sink + s->window)) return TSV_ERR_SHAPE;
  return TSV_OK;
}

// (Without rows there need be no arrays of them: the calls only look the batch over.)
static int check_kv(const tsv_tok_shape* s, const tsv_tok_cache* c, const tsv_tok_batch* b, const tsv_tok_rows* in) {
  if (!in) return TSV_ERR_NULL;
  if (b->rows == 0) return TSV_OK;
  if (!in->k || !in->v != !c->v) return TSV_ERR_NULL;
  int r = check_rows(s, in->k, in->k_ld, s->Hk);
  if (!r && in->v) r = check_rows(s, in->v, in->v_ld, s->Hk);
  return r;
}

static int check_pool(const tsv_page_pool* p) {
  if (!p || !p->page_table || !p->ref) return TSV_ERR_NULL;
  if (p->slots < 1 || p->max_pages < 1 || p->max_pages > 1 << 20 || p->n_pages < 1 || p->n_pages > 1 << 28 || p->page_tokens < 1) return TSV_ERR_SHAPE;
  if (p->n_planes < 0 || p->n_rows < 0 || p->n_planes > 1 << 16 || p->n_rows > 1 << 16) return TSV_ERR_SHAPE;
  if ((p->n_planes && !p->planes) || (p->n_rows && !p->rows)) return TSV_ERR_NULL;
  for (int i = 0; i < p->n_planes; ++i) {
    if (!p->planes[i].base) return TSV_ERR_NULL;
    if (!al(p->planes[i].base, 16) || p->planes[i].bytes % 16) return TSV_ERR_ALIGN;
    if (p->planes[i].bytes < 1 || p->planes[i].bytes > 1 << 30) return TSV_ERR_SHAPE;
  }
  for (int i = 0; i < p->n_rows; ++i) {
    if (!p->rows[i].base) return TSV_ERR_NULL;
    if (!al(p->rows[i].base, 4) || p->rows[i].bytes % 4) return TSV_ERR_ALIGN;
    if (p->rows[i].bytes < 1 || p->rows[i].bytes > 1 << 30) return TSV_ERR_SHAPE;
  }
  return TSV_OK;
}

static int check_list(const tsv_page_pool* p, int n, const int32_t* a, const int32_t* b, const int32_t* c, const int32_t* status) {
  const int r = check_pool(p);
  if (r) return r;
  if (n < 0) return TSV_ERR_SHAPE;
  if (n > TSV_MAX_PAGE_LIST) return TSV_ERR_LIMIT;
  return n && (!a || !b || !c || !status) ? TSV_ERR_NULL : TSV_OK;
}

static int check_ws(const void* ws, size_t have, size_t need) {
  return !ws || !al(ws, 256) || have < need ? TSV_ERR_WORKSPACE : TSV_OK;
}

}  // namespace tsv

using namespace tsv;

extern "C" {

int qk_norm_rope(const tsv_tok_shape* shape, const int32_t* L, const tsv_tok_batch* batch, const tsv_tok_rows* in, const float* wq, const float* wk,
                 float eps, const float* inv_freq, int32_t rot, int32_t first, int32_t pairs, void* q_out, int64_t ldq, void* k_out, int64_t ldk,
                 int32_t* status, void* stream) {
  if (!shape || !L || !in || !status) return TSV_ERR_NULL;
  if (!tok_shape_ok(shape)) return TSV_ERR_SHAPE;
  int r;
  if ((r = check_batch(batch))) return r;
  if (!in->q && !in->k && batch->rows) return TSV_ERR_NULL;
  if ((in->q && !q_out) || (in->k && !k_out) || (rot && !inv_freq)) return TSV_ERR_NULL;
  if (rot < 0 || rot % 16 || first < 0 || first % 8 || first > shape->d - rot) return TSV_ERR_SHAPE;
  if (in->q && ((r = check_rows(shape, in->q, in->q_ld, shape->H)) || (r = check_rows(shape, q_out, ldq, shape->H)))) return r;
  if (in->k && ((r = check_rows(shape, in->k, in->k_ld, shape->Hk)) || (r = check_rows(shape, k_out, ldk, shape->Hk)))) return r;
  const int64_t n = batch->rows;
  const bool q = in->q && n, k = in->k && n;
  // (an output may be its input, row by row; anything else of the call that it shares a row with would be read after it is written)
  if (q && !(q_out == in->q && (ldq == in->q_ld || n == 1)) && rows_meet(shape, q_out, ldq, shape->H, in->q, in->q_ld, shape->H, n)) return TSV_ERR_SHAPE;
  if (k && !(k_out == in->k && (ldk == in->k_ld || n == 1)) && rows_meet(shape, k_out, ldk, shape->Hk, in->k, in->k_ld, shape->Hk, n)) return TSV_ERR_SHAPE;
  if (q && k && (rows_meet(shape, q_out, ldq, shape->H, in->k, in->k_ld, shape->Hk, n) || rows_meet(shape, k_out, ldk, shape->Hk, in->q, in->q_ld, shape->H, n) ||
                 rows_meet(shape, q_out, ldq, shape->H, k_out, ldk, shape->Hk, n))) return TSV_ERR_SHAPE;
  return launch_rope(*shape, L, *batch, *in, wq, wk, eps, inv_freq, rot, first, pairs != 0, q_out, ldq, k_out, ldk, status, (cudaStream_t)stream);
}

size_t tsv_tok_workspace_bytes(const tsv_tok_shape* shape, int64_t rows) {
  if (!shape || !tok_shape_ok(shape) || rows < 0 || rows > (int64_t)1 << 40) return 0;
  return tok_attn_workspace(*shape, rows);
}

int window_sink_attn(const tsv_tok_shape* shape, const tsv_tok_cache* cache, const tsv_tok_batch* batch, const tsv_tok_rows* in, void* out,
                     void* workspace, size_t workspace_bytes, int32_t* status, void* stream) {
  if (!shape || !status || !in || !batch || (batch->rows && (!out || !in->q))) return TSV_ERR_NULL;
  if (!tok_shape_ok(shape)) return TSV_ERR_SHAPE;
  int r;
  if ((r = check_tok_cache(cache, shape)) || (r = check_batch(batch)) || (r = check_kv(shape, cache, batch, in))) return r;
  if (batch->rows && (r = check_rows(shape, in->q, in->q_ld, shape->H))) return r;
  if (!al(out, 16)) return TSV_ERR_ALIGN;
  if ((r = check_ws(workspace, workspace_bytes, tok_attn_workspace(*shape, batch->rows)))) return r;
  if (const int64_t n = batch->rows) {
    const int64_t bytes = n * shape->H * shape->d * (shape->dtype == TSV_BF16 ? 2 : 4);
    if (meets(shape, out, bytes, in->q, in->q_ld, shape->H, n) || meets(shape, out, bytes, in->k, in->k_ld, shape->Hk, n) ||
        meets(shape, out, bytes, in->v, in->v_ld, shape->Hk, n)) return TSV_ERR_SHAPE;
  }
  return launch_tok_attn(resolved(shape), *cache, *batch, *in, out, (char*)workspace, status, (cudaStream_t)stream);
}

int token_commit(const tsv_tok_shape* shape, const tsv_tok_cache* cache, const tsv_tok_batch* batch, const tsv_tok_rows* in, const int32_t* path,
                 int32_t path_ld, const int32_t* count, int32_t* status, void* stream) {
  if (!shape || !status) return TSV_ERR_NULL;
  if (!tok_shape_ok(shape)) return TSV_ERR_SHAPE;
  int r;
  if ((r = check_tok_cache(cache, shape)) || (r = check_batch(batch)) || (r = check_kv(shape, cache, batch, in))) return r;
  if (path && path_ld < 1) return TSV_ERR_SHAPE;
  return launch_token_commit(*shape, *cache, *batch, *in, path, path_ld, count, status, (cudaStream_t)stream);
}

size_t tsv_pages_workspace_bytes(const tsv_page_pool* pool) { return check_pool(pool) ? 0 : pages_workspace(*pool); }

int pages_assign(const tsv_page_pool* pool, int32_t n, const int32_t* slot, const int32_t* first, const int32_t* last, void* workspace,
                 size_t workspace_bytes, int32_t* status, void* stream) {
  int r;
  if ((r = check_list(pool, n, slot, first, last, status)) || (r = check_ws(workspace, workspace_bytes, pages_workspace(*pool)))) return r;
  return n ? launch_pages_assign(*pool, n, slot, first, last, (char*)workspace, status, (cudaStream_t)stream) : TSV_OK;
}

int pages_free(const tsv_page_pool* pool, int32_t n, const int32_t* slot, const int32_t* first, const int32_t* last, int32_t* status, void* stream) {
  const int r = check_list(pool, n, slot, first, last, status);
  if (r) return r;
  return n ? launch_pages_free(*pool, n, slot, first, last, status, (cudaStream_t)stream) : TSV_OK;
}

int pages_fork(const tsv_page_pool* pool, int32_t n, const int32_t* src, const int32_t* dst, const int32_t* L, void* workspace, size_t workspace_bytes,
               int32_t* status, void* stream) {
  int r;
  if ((r = check_list(pool, n, src, dst, L, status)) || (r = check_ws(workspace, workspace_bytes, pages_workspace(*pool)))) return r;
  return n ? launch_pages_fork(*pool, n, src, dst, L, (char*)workspace, status, (cudaStream_t)stream) : TSV_OK;
}

int pages_compact(const tsv_page_pool* pool, int32_t* n_used, void* workspace, size_t workspace_bytes, void* stream) {
  int r;
  if ((r = check_pool(pool))) return r;
  if (!n_used) return TSV_ERR_NULL;
  if ((r = check_ws(workspace, workspace_bytes, pages_workspace(*pool)))) return r;
  return launch_pages_compact(*pool, n_used, (char*)workspace, (cudaStream_t)stream);
}

}  // extern "C"
