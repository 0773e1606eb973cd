// C ABI of the paged cache: argument checks and launches.
#include <algorithm>
#include <new>
#include <vector>

#include "api_checks.h"
#include "pages.h"

using namespace scalekv;

namespace {

static_assert(kTypeF32 == SCALEKV_F32 && kTypeBf16 == SCALEKV_BF16 && kTypeE4m3 == SCALEKV_E4M3, "element types");

int cache_elem_bytes(const scalekv_pages* c) { return c->dtype == SCALEKV_E4M3 ? 1 : c->dtype == SCALEKV_F32 ? 4 : 2; }

// sizes alone: what the workspace query has
scalekv_status check_page_sizes(const scalekv_shape* s, const scalekv_pages* c) {
  if (!c) return fail(SCALEKV_ERR_INVALID_ARG, "pages is NULL");
  if (c->dtype != SCALEKV_F32 && c->dtype != SCALEKV_BF16 && c->dtype != SCALEKV_E4M3)
    return fail(SCALEKV_ERR_UNSUPPORTED, "pages.dtype %d is not SCALEKV_F32, SCALEKV_BF16 or SCALEKV_E4M3", c->dtype);
  if (c->dtype != SCALEKV_E4M3 && c->dtype != s->dtype)
    return fail(SCALEKV_ERR_UNSUPPORTED, "pages.dtype %d is neither the shape's (%d) nor SCALEKV_E4M3", c->dtype, s->dtype);
  if (c->page_rows < kPageRowsMin || c->page_rows > kPageRowsMax || (c->page_rows & (c->page_rows - 1)))
    return fail(SCALEKV_ERR_UNSUPPORTED, "pages.page_rows %d is not a power of two in %d..%d", c->page_rows, kPageRowsMin,
                kPageRowsMax);
  if (c->n_page < 1) return fail(SCALEKV_ERR_INVALID_ARG, "pages.n_page must be >= 1 (got %d)", c->n_page);
  if (c->n_kv_head < 1 || s->n_head % c->n_kv_head)
    return fail(SCALEKV_ERR_INVALID_ARG, "pages.n_kv_head %d does not divide n_head %d", c->n_kv_head, s->n_head);
  if (c->table_width < 1) return fail(SCALEKV_ERR_INVALID_ARG, "pages.table_width must be >= 1 (got %d)", c->table_width);
  if ((long long)c->table_width * c->page_rows > 1LL << 30)
    return fail(SCALEKV_ERR_UNSUPPORTED, "pages.table_width * page_rows = %lld exceeds 2^30",
                (long long)c->table_width * c->page_rows);
  return SCALEKV_OK;
}

scalekv_status check_stride(long long stride, long long least, long long most, int multiple, const char* name) {
  if (stride < least || stride > most || stride % multiple)
    return fail(SCALEKV_ERR_INVALID_ARG, "%s %lld must be a multiple of %d in %lld..%lld", name, stride, multiple, least, most);
  return SCALEKV_OK;
}

// elements; with kMostReach for a pool or a sequence's rows, offsets stay far from the ends of int64
constexpr long long kMostStride = 1LL << 40, kMostReach = 1LL << 50;

scalekv_status check_reach(long long n, long long stride, const char* name) {
  if (stride > 0 && n > kMostReach / stride)
    return fail(SCALEKV_ERR_UNSUPPORTED, "%s: %lld times a stride of %lld is too far", name, n, stride);
  return SCALEKV_OK;
}

scalekv_status check_pages(const scalekv_shape* s, const scalekv_pages* c) {
  SCALEKV_TRY(check_page_sizes(s, c));
  SCALEKV_TRY(check_dense(c->k, true, "pages.k"));
  SCALEKV_TRY(check_dense(c->v, true, "pages.v"));
  const int per = 16 / cache_elem_bytes(c);
  const long long unit = (long long)c->page_rows * s->head_dim;
  SCALEKV_TRY(check_stride(c->head_stride, unit, kMostStride, per, "pages.head_stride"));
  SCALEKV_TRY(check_stride(c->page_stride, c->n_kv_head * c->head_stride, kMostStride, per, "pages.page_stride"));
  SCALEKV_TRY(check_reach(c->n_page, c->page_stride, "pages"));
  if (c->dtype == SCALEKV_E4M3) {
    if (!c->k_scale || !c->v_scale) return fail(SCALEKV_ERR_INVALID_ARG, "pages.k_scale or v_scale is NULL");
    SCALEKV_TRY(check_stride(c->scale_head_stride, c->page_rows, kMostStride, 1, "pages.scale_head_stride"));
    SCALEKV_TRY(check_stride(c->scale_page_stride, c->n_kv_head * c->scale_head_stride, kMostStride, 1,
                             "pages.scale_page_stride"));
    SCALEKV_TRY(check_reach(c->n_page, c->scale_page_stride, "pages' scales"));
  }
  if (!c->table) return fail(SCALEKV_ERR_INVALID_ARG, "pages.table is NULL");
  if (!c->len) return fail(SCALEKV_ERR_INVALID_ARG, "pages.len is NULL");
  return SCALEKV_OK;
}

scalekv_status check_chunk(const scalekv_shape* s, const scalekv_chunk* chunk) {
  if (!chunk) return fail(SCALEKV_ERR_INVALID_ARG, "chunk is NULL");
  if (chunk->max_new < 1) return fail(SCALEKV_ERR_INVALID_ARG, "chunk.max_new must be >= 1 (got %d)", chunk->max_new);
  SCALEKV_TRY(check_rows(s, chunk->max_new, "chunk.max_new"));
  // rows are numbered over all sequences and heads, in int32, up to the end of a row group (128 at most) behind the last
  if ((long long)s->n_seq * s->n_head * chunk->max_new > 0x7fffffffLL - 255)
    return fail(SCALEKV_ERR_UNSUPPORTED, "n_seq * n_head * max_new = %lld is too large",
                (long long)s->n_seq * s->n_head * chunk->max_new);
  return SCALEKV_OK;
}

scalekv_status check_token_rows(const scalekv_shape* s, const scalekv_rows* r, const scalekv_chunk* chunk, const char* name) {
  if (!r) return fail(SCALEKV_ERR_INVALID_ARG, "%s is NULL", name);
  if (!r->ptr && r->n_row == 0 && chunk->first) return SCALEKV_OK;  // packed, and no sequence has new tokens
  if (!r->ptr) return fail(SCALEKV_ERR_INVALID_ARG, "%s.ptr is NULL", name);
  if (!aligned16(r->ptr)) return fail(SCALEKV_ERR_INVALID_ARG, "%s.ptr is not 16-byte aligned", name);
  const int per = 16 / elem_bytes(s);
  for (const int64_t stride : {r->seq_stride, r->head_stride, r->row_stride})
    if (stride < 0 || stride > kMostStride || stride % per)
      return fail(SCALEKV_ERR_INVALID_ARG, "%s: stride %lld must be a multiple of %d and not negative", name,
                  (long long)stride, per);
  if (r->n_row < 0) return fail(SCALEKV_ERR_INVALID_ARG, "%s.n_row is negative", name);
  SCALEKV_TRY(check_reach(r->n_row, r->row_stride, name));
  if (!chunk->first && r->n_row < chunk->max_new)
    return fail(SCALEKV_ERR_INVALID_ARG, "%s.n_row %d is less than max_new %d", name, r->n_row, chunk->max_new);
  return SCALEKV_OK;
}

// Two tensors of token rows: where `first` places the tokens, row first[s] + t of both belongs to the same token, and what
// lies behind the end of the shorter one would be left out without a word.  (Otherwise max_new rows of each are looked at.)
scalekv_status check_same_rows(const scalekv_rows* a, const char* name_a, const scalekv_rows* b, const char* name_b,
                               const scalekv_chunk* chunk) {
  if (chunk->first && a->n_row != b->n_row)
    return fail(SCALEKV_ERR_INVALID_ARG, "%s has %d rows and %s %d: they must have the same number where first is given",
                name_a, a->n_row, name_b, b->n_row);
  return SCALEKV_OK;
}

struct Span {
  uintptr_t lo, hi;
};
bool meet(Span a, Span b) { return a.lo < b.hi && b.lo < a.hi; }

Span rows_span(const scalekv_shape* s, const scalekv_rows* r, int n_head) {
  const uintptr_t lo = reinterpret_cast<uintptr_t>(r->ptr);
  const long long last = (s->n_seq - 1) * r->seq_stride + (n_head - 1) * r->head_stride +
                         (r->n_row > 0 ? r->n_row - 1 : 0) * r->row_stride + s->head_dim;
  return {lo, lo + (uintptr_t)(last * elem_bytes(s))};
}
Span pool_span(const scalekv_shape* s, const scalekv_pages* c, const void* p) {
  const uintptr_t lo = reinterpret_cast<uintptr_t>(p);
  const long long last =
      (c->n_page - 1) * c->page_stride + (c->n_kv_head - 1) * c->head_stride + (long long)c->page_rows * s->head_dim;
  return {lo, lo + (uintptr_t)(last * cache_elem_bytes(c))};
}
Span scale_span(const scalekv_pages* c, const void* p) {
  const uintptr_t lo = reinterpret_cast<uintptr_t>(p);
  return {lo, lo + (uintptr_t)((c->n_page - 1) * c->scale_page_stride + (c->n_kv_head - 1) * c->scale_head_stride +
                               c->page_rows)};
}
Span kv_bytes(const scalekv_shape* s, const scalekv_kv* kv) {
  Span x;
  kv_span(s, kv, &x.lo, &x.hi);
  return x;
}
bool meets_pool(const scalekv_shape* s, const scalekv_pages* c, Span x) {
  if (meet(x, pool_span(s, c, c->k)) || meet(x, pool_span(s, c, c->v))) return true;
  return c->dtype == SCALEKV_E4M3 && (meet(x, scale_span(c, c->k_scale)) || meet(x, scale_span(c, c->v_scale)));
}

// Do two pools of the same strides share bytes?  (Keys and values may interleave: page by page, or head by head.)
// Blocks of `unit` bytes lie at i * page + h * head, page >= n_head * head, head >= unit.
bool pools_meet(const void* a, const void* b, long long n_page, long long page, int n_head, long long head, long long unit) {
  const uintptr_t ua = reinterpret_cast<uintptr_t>(a), ub = reinterpret_cast<uintptr_t>(b);
  const long long gap = (long long)(ua < ub ? ub - ua : ua - ub);
  if (gap < 0) return false;  // further apart than any pool is long
  const long long pages_apart = gap / page, rest = gap % page;
  // the other block's page: pages_apart or the next, its head: the nearest from below or above
  for (long long i = pages_apart; i <= pages_apart + 1; ++i) {
    if (i >= n_page) continue;
    const long long x = rest - (i - pages_apart) * page;  // in (-page, page)
    const long long h0 = x >= 0 ? x / head : -((-x + head - 1) / head);
    for (long long h = h0; h <= h0 + 1; ++h)
      if (h > -n_head && h < n_head && x - h * head < unit && h * head - x < unit) return true;
  }
  return false;
}

// Does a pool share bytes with scales whose pages lie as far apart as its own (in one record, say)?  Codes lie at i * page +
// h * head, `unit` bytes each, scales `gap` bytes on at i * page + h * scale_head, `rows` bytes each.
bool record_meets(long long gap, long long n_page, long long page, int n_head, long long head, long long unit,
                  long long scale_head, long long rows) {
  auto floor_div = [](long long a, long long b) { return a / b - (a % b < 0); };
  for (int g = 0; g < n_head; ++g) {
    const long long at = gap + g * scale_head, first = floor_div(at, page);
    for (long long i = first; i <= first + 1; ++i) {  // the codes' page, counted from the scales'
      if (i <= -n_page || i >= n_page) continue;
      const long long x = at - i * page, below = floor_div(x, head);
      for (long long h = below; h <= below + 1; ++h)
        if (h >= 0 && h < n_head && h * head < x + rows && x < h * head + unit) return true;
    }
  }
  return false;
}

// Do two of the rows at i * stride[0] + j * stride[1] + k * stride[2], i < n[0] and so on, share bytes?  Rows of d elements,
// which each stride between several rows holds.
bool rows_coincide(const long long (&n)[3], const long long (&stride)[3], int d) {
  int by[3] = {0, 1, 2};
  std::sort(by, by + 3, [&](int a, int b) { return stride[a] < stride[b]; });
  long long reach = d;  // of the dimensions before
  bool nested = true;
  for (const int x : by) {
    if (n[x] == 1) continue;
    nested = nested && stride[x] >= reach;
    reach += (n[x] - 1) * stride[x];
  }
  if (nested) return false;
  // Differences of two rows: of the two dimensions with the fewest rows all (the first not negative: a pair has two signs),
  // and of the third the two that bring them nearest to zero.
  std::sort(by, by + 3, [&](int a, int b) { return n[a] < n[b]; });
  const int x = by[0], y = by[1], z = by[2];
  for (long long i = 0; i < n[x]; ++i)
    for (long long j = 1 - n[y]; j < n[y]; ++j) {
      const long long at = i * stride[x] + j * stride[y];
      const long long k0 = (at < 0 ? -at : at) / stride[z];  // k: less k0, or less k0 + 1, towards zero
      for (long long k = k0; k <= k0 + 1; ++k) {
        if (k >= n[z] || (i == 0 && j == 0 && k == 0)) continue;
        const long long apart = (at < 0 ? -at : at) - k * stride[z];
        if (apart < d && -apart < d) return true;
      }
    }
  return false;
}

PagesView pages_view(const scalekv_shape* s, const scalekv_pages* c) {
  PagesView v;
  const long long e = cache_elem_bytes(c);
  v.k = static_cast<unsigned char*>(c->k);
  v.v = static_cast<unsigned char*>(c->v);
  v.k_scale = c->k_scale;
  v.v_scale = c->v_scale;
  v.table = c->table;
  v.len = c->len;
  v.page = c->page_stride * e;
  v.head = c->head_stride * e;
  v.scale_page = c->scale_page_stride;
  v.scale_head = c->scale_head_stride;
  v.width = c->table_width;
  v.page_shift = __builtin_ctz((unsigned)c->page_rows);
  v.n_page = c->n_page;
  v.n_kv_head = c->n_kv_head;
  v.type = c->dtype;
  return v;
}
RowsView rows_view(const scalekv_shape* s, const scalekv_rows* r) {
  const long long e = elem_bytes(s);
  return RowsView{static_cast<unsigned char*>(r->ptr), r->seq_stride * e, r->head_stride * e, r->row_stride * e, r->n_row};
}

scalekv_status check_mask(const scalekv_mask* m, MaskView* out) {
  *out = MaskView{0, 0, 0};
  if (!m) return SCALEKV_OK;
  if (m->causal != 0 && m->causal != 1) return fail(SCALEKV_ERR_INVALID_ARG, "mask.causal %d is not 0 or 1", m->causal);
  if (m->window < 0) return fail(SCALEKV_ERR_INVALID_ARG, "mask.window is negative (%d)", m->window);
  if (m->n_sink < 0) return fail(SCALEKV_ERR_INVALID_ARG, "mask.n_sink is negative (%d)", m->n_sink);
  // (no position reaches 2^30: larger windows hide nothing, and sums with them stay in int32)
  *out = MaskView{m->causal, std::min(m->window, 1 << 30), std::min(m->n_sink, 1 << 30)};
  return SCALEKV_OK;
}

// the plan of an attention whose arguments have passed the checks
scalekv_status make_plan(const scalekv_shape* s, const scalekv_pages* c, int max_new, const MaskView& mask, PagesPlan* plan) {
  *plan = pages_plan(s->dtype, s->head_dim, s->n_seq, s->n_head, pages_view(s, c), max_new, mask);
  if (plan->n_wg < 0) return fail(SCALEKV_ERR_UNSUPPORTED, "this call needs more than 2^31 - 1 workgroups");
  return SCALEKV_OK;
}

}  // namespace

extern "C" {

scalekv_status scalekv_pages_write(const scalekv_shape* shape, const scalekv_pages* pages, const scalekv_rows* k_new,
                                   const scalekv_rows* v_new, const scalekv_chunk* chunk, void* stream) {
  SCALEKV_TRY(check_shape(shape));
  SCALEKV_TRY(check_pages(shape, pages));
  SCALEKV_TRY(check_chunk(shape, chunk));
  SCALEKV_TRY(check_token_rows(shape, k_new, chunk, "k_new"));
  SCALEKV_TRY(check_token_rows(shape, v_new, chunk, "v_new"));
  SCALEKV_TRY(check_same_rows(k_new, "k_new", v_new, "v_new", chunk));
  if (meets_pool(shape, pages, rows_span(shape, k_new, pages->n_kv_head)) ||
      meets_pool(shape, pages, rows_span(shape, v_new, pages->n_kv_head)))
    return fail(SCALEKV_ERR_INVALID_ARG, "k_new or v_new overlaps the pool");
  const long long e = cache_elem_bytes(pages), unit = (long long)pages->page_rows * shape->head_dim * e;
  if (pools_meet(pages->k, pages->v, pages->n_page, pages->page_stride * e, pages->n_kv_head, pages->head_stride * e, unit))
    return fail(SCALEKV_ERR_INVALID_ARG, "pages.k and pages.v overlap");
  if (pages->dtype == SCALEKV_E4M3) {
    if (pools_meet(pages->k_scale, pages->v_scale, pages->n_page, pages->scale_page_stride, pages->n_kv_head,
                   pages->scale_head_stride, pages->page_rows))
      return fail(SCALEKV_ERR_INVALID_ARG, "pages.k_scale and pages.v_scale overlap");
    for (const void* p : {pages->k, pages->v})
      for (const void* q : {pages->k_scale, pages->v_scale})
        if (meet(pool_span(shape, pages, p), scale_span(pages, q)) &&
            (pages->scale_page_stride != pages->page_stride ||
             record_meets(static_cast<const char*>(q) - static_cast<const char*>(p), pages->n_page, pages->page_stride,
                          pages->n_kv_head, pages->head_stride, unit, pages->scale_head_stride, pages->page_rows)))
          return fail(SCALEKV_ERR_INVALID_ARG, "the scales overlap the pool");
  }
  if (k_new->n_row == 0 && v_new->n_row == 0) return SCALEKV_OK;
  SCALEKV_HIP(launch_pages_write(shape->dtype, shape->head_dim, shape->n_seq, pages_view(shape, pages),
                                 rows_view(shape, k_new), rows_view(shape, v_new),
                                 ChunkView{chunk->max_new, chunk->first, chunk->count}, static_cast<hipStream_t>(stream)),
              "pages write launch");
  return SCALEKV_OK;
}

scalekv_status scalekv_pages_read(const scalekv_shape* shape, const scalekv_pages* pages, const int32_t* idx, int32_t n_row,
                                  const scalekv_kv* k_dst, const scalekv_kv* v_dst, void* stream) {
  SCALEKV_TRY(check_shape(shape));
  SCALEKV_TRY(check_pages(shape, pages));
  SCALEKV_TRY(check_rows(shape, n_row, "n_row"));
  if ((long long)shape->n_seq * shape->n_head * n_row > 0x7fffffffLL)
    return fail(SCALEKV_ERR_UNSUPPORTED, "n_seq * n_head * n_row = %lld is too large",
                (long long)shape->n_seq * shape->n_head * n_row);
  SCALEKV_TRY(check_kv(shape, k_dst, n_row, "k_dst"));
  SCALEKV_TRY(check_kv(shape, v_dst, n_row, "v_dst"));
  const Span k = kv_bytes(shape, k_dst), v = kv_bytes(shape, v_dst);
  if (meet(k, v)) return fail(SCALEKV_ERR_INVALID_ARG, "k_dst and v_dst overlap");
  if (meets_pool(shape, pages, k) || meets_pool(shape, pages, v))
    return fail(SCALEKV_ERR_INVALID_ARG, "k_dst or v_dst overlaps the pool");
  if (n_row == 0) return SCALEKV_OK;
  SCALEKV_HIP(launch_pages_read(shape->dtype, shape->head_dim, shape->n_seq, shape->n_head, pages_view(shape, pages), idx,
                                n_row, KvView{k_dst->ptr, k_dst->seq_stride, k_dst->head_stride},
                                KvView{v_dst->ptr, v_dst->seq_stride, v_dst->head_stride}, static_cast<hipStream_t>(stream)),
              "pages read launch");
  return SCALEKV_OK;
}

scalekv_status scalekv_pages_workspace_bytes(const scalekv_shape* shape, const scalekv_pages* pages, int32_t max_new,
                                             const scalekv_mask* mask, size_t* out) {
  SCALEKV_TRY(check_shape(shape));
  SCALEKV_TRY(check_page_sizes(shape, pages));
  if (!out) return fail(SCALEKV_ERR_INVALID_ARG, "out is NULL");
  const scalekv_chunk chunk{max_new, nullptr, nullptr};
  SCALEKV_TRY(check_chunk(shape, &chunk));
  MaskView m;
  SCALEKV_TRY(check_mask(mask, &m));
  PagesPlan plan;
  SCALEKV_TRY(make_plan(shape, pages, max_new, m, &plan));
  *out = pages_partial_bytes(shape->n_seq, shape->head_dim, shape->n_head / pages->n_kv_head, max_new, plan);
  return SCALEKV_OK;
}

scalekv_status scalekv_pages_attend(const scalekv_shape* shape, const scalekv_pages* pages, const scalekv_rows* q,
                                    const scalekv_chunk* chunk, const scalekv_mask* mask, const scalekv_rows* out, void* ws,
                                    size_t ws_bytes, void* stream) {
  SCALEKV_TRY(check_shape(shape));
  SCALEKV_TRY(check_pages(shape, pages));
  SCALEKV_TRY(check_chunk(shape, chunk));
  SCALEKV_TRY(check_token_rows(shape, q, chunk, "q"));
  SCALEKV_TRY(check_token_rows(shape, out, chunk, "out"));
  SCALEKV_TRY(check_same_rows(q, "q", out, "out", chunk));
  MaskView m;
  SCALEKV_TRY(check_mask(mask, &m));
  if (out->n_row == 0) return SCALEKV_OK;
  // (packed: no stride between sequences, whose rows are those of one tensor)
  const bool packed = chunk->first && out->seq_stride == 0;
  const long long n[3] = {packed ? 1 : shape->n_seq, shape->n_head, chunk->first ? out->n_row : chunk->max_new};
  const long long strides[3] = {out->seq_stride, out->head_stride, out->row_stride};
  for (int x = 0; x < 3; ++x)
    if (n[x] > 1 && strides[x] < shape->head_dim)
      return fail(SCALEKV_ERR_INVALID_ARG, "rows of out coincide: a stride is below head_dim");
  const Span o = rows_span(shape, out, shape->n_head);
  const bool on_q = out->ptr == q->ptr && out->seq_stride == q->seq_stride && out->head_stride == q->head_stride &&
                    out->row_stride == q->row_stride;
  if (!on_q && meet(o, rows_span(shape, q, shape->n_head)))
    return fail(SCALEKV_ERR_INVALID_ARG, "out overlaps q and does not lie exactly on it");
  if (rows_coincide(n, strides, shape->head_dim))
    return fail(SCALEKV_ERR_INVALID_ARG, "rows of out coincide: strides %lld, %lld and %lld for %lld x %lld x %lld rows of %d",
                strides[0], strides[1], strides[2], n[0], n[1], n[2], shape->head_dim);
  if (meets_pool(shape, pages, o)) return fail(SCALEKV_ERR_INVALID_ARG, "out overlaps the pool");
  PagesPlan plan;
  SCALEKV_TRY(make_plan(shape, pages, chunk->max_new, m, &plan));
  const size_t need =
      pages_partial_bytes(shape->n_seq, shape->head_dim, shape->n_head / pages->n_kv_head, chunk->max_new, plan);
  if (need > 0) {
    if (!ws) return fail(SCALEKV_ERR_WORKSPACE, "workspace is NULL (%zu bytes needed)", need);
    if (!aligned16(ws)) return fail(SCALEKV_ERR_INVALID_ARG, "workspace is not 16-byte aligned");
    if (ws_bytes < need) return fail(SCALEKV_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", ws_bytes, need);
    const uintptr_t w = reinterpret_cast<uintptr_t>(ws);
    if (meet(Span{w, w + need}, o) || meet(Span{w, w + need}, rows_span(shape, q, shape->n_head)) ||
        meets_pool(shape, pages, Span{w, w + need}))
      return fail(SCALEKV_ERR_INVALID_ARG, "the workspace overlaps q, out or the pool");
  }
  SCALEKV_HIP(launch_pages_attend(shape->dtype, shape->head_dim, shape->n_seq, shape->n_head, pages_view(shape, pages),
                                  rows_view(shape, q), rows_view(shape, out),
                                  ChunkView{chunk->max_new, chunk->first, chunk->count}, m, resolve_scale(shape), plan, ws,
                                  static_cast<hipStream_t>(stream)),
              "pages attend launch");
  return SCALEKV_OK;
}

scalekv_status scalekv_pages_check(const scalekv_shape* shape, const scalekv_pages* pages, const int32_t* table,
                                   const int32_t* len, const scalekv_chunk* chunk, const int32_t* first,
                                   const int32_t* count, int32_t n_row) {
  SCALEKV_TRY(check_shape(shape));
  SCALEKV_TRY(check_page_sizes(shape, pages));
  if (!table || !len) return fail(SCALEKV_ERR_INVALID_ARG, "table or len is NULL");
  if (chunk) SCALEKV_TRY(check_chunk(shape, chunk));
  const int P = pages->page_rows, width = pages->table_width;
  auto new_of = [&](int s) { return !chunk ? 0 : count ? count[s] : chunk->max_new; };
  for (int s = 0; s < shape->n_seq; ++s) {
    if (len[s] < 0 || (long long)len[s] > (long long)width * P)
      return fail(SCALEKV_ERR_INVALID_ARG, "len[%d] = %d is outside 0..%lld", s, len[s], (long long)width * P);
    for (int i = 0; i < (len[s] + P - 1) / P; ++i) {
      const int page = table[(long long)s * width + i];
      if (page < 0 || page >= pages->n_page)
        return fail(SCALEKV_ERR_INVALID_ARG, "table[%d][%d] = %d is outside 0..%d", s, i, page, pages->n_page - 1);
    }
    const int n = new_of(s);
    if (n < 0 || (chunk && n > chunk->max_new) || n > len[s])
      return fail(SCALEKV_ERR_INVALID_ARG, "count[%d] = %d is outside 0..min(max_new, len[%d] = %d)", s, n, s, len[s]);
    const long long at = first ? first[s] : 0;
    if (n > 0 && (at < 0 || at + n > n_row))
      return fail(SCALEKV_ERR_INVALID_ARG, "rows %lld..%lld of sequence %d are outside 0..%d", at, at + n - 1, s, n_row - 1);
  }
  // pages that receive new tokens belong to one sequence, once
  for (int s = 0; s < shape->n_seq; ++s) {
    const int n = new_of(s);
    if (n == 0) continue;
    for (int i = (len[s] - n) / P; i < (len[s] + P - 1) / P; ++i) {
      const int page = table[(long long)s * width + i];
      for (int o = 0; o < shape->n_seq; ++o)
        for (int j = 0; j < (len[o] + P - 1) / P; ++j)
          if ((o != s || j != i) && table[(long long)o * width + j] == page)
            return fail(SCALEKV_ERR_INVALID_ARG, "page %d receives new tokens of sequence %d and is table[%d][%d] too", page,
                        s, o, j);
    }
  }
  return SCALEKV_OK;
}

scalekv_status scalekv_pages_check_packed(const scalekv_shape* shape, const scalekv_chunk* chunk, const int32_t* first,
                                          const int32_t* count, int32_t n_row) {
  SCALEKV_TRY(check_shape(shape));
  SCALEKV_TRY(check_chunk(shape, chunk));
  if (!first) return fail(SCALEKV_ERR_INVALID_ARG, "first is NULL");
  auto new_of = [&](int s) { return count ? count[s] : chunk->max_new; };
  // the sequence whose tokens begin at each row: where ranges meet, two neighbours among them do
  std::vector<int> by_row;
  try {
    for (int s = 0; s < shape->n_seq; ++s) {
      const int n = new_of(s);
      if (n < 0 || n > chunk->max_new)
        return fail(SCALEKV_ERR_INVALID_ARG, "count[%d] = %d is outside 0..%d", s, n, chunk->max_new);
      if (n == 0) continue;
      const long long at = first[s];
      if (at < 0 || at + n > n_row)
        return fail(SCALEKV_ERR_INVALID_ARG, "rows %lld..%lld of sequence %d are outside 0..%d", at, at + n - 1, s, n_row - 1);
      by_row.push_back(s);
    }
  } catch (const std::bad_alloc&) {
    return fail(SCALEKV_ERR_INVALID_ARG, "no memory for %d sequences", shape->n_seq);
  }
  std::sort(by_row.begin(), by_row.end(),
            [&](int a, int b) { return first[a] != first[b] ? first[a] < first[b] : a < b; });
  for (size_t i = 1; i < by_row.size(); ++i) {
    const int a = by_row[i - 1], b = by_row[i];
    if (first[b] < first[a] + new_of(a))
      return fail(SCALEKV_ERR_INVALID_ARG, "sequences %d and %d share row %d", std::min(a, b), std::max(a, b), first[b]);
  }
  return SCALEKV_OK;
}

}  // extern "C"
