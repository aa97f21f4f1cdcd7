// Host side of the calls that answer with the weights: argument checks and launches.
#include <math.h>
#include <stdarg.h>
#include <stdio.h>

#include "answer.h"

namespace {

int fail(int code, const char *fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof(buf), fmt, ap);
  va_end(ap);
  copes::set_last_error(buf);
  return code;
}

int launch_status(cudaError_t e, const char *who) {
  return e == cudaSuccess ? COPES_OK
                          : fail(COPES_ERR_CUDA, "%s: %s (%s)", who, cudaGetErrorName(e), cudaGetErrorString(e));
}

bool aligned(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

bool overlaps(const void *a, uint64_t na, const void *b, uint64_t nb) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return a && b && na && nb && x < y + nb && y < x + na;
}

// Bytes from the first to past the last element of rows of heads of `count` elements; 0 (never an
// overlap) where a stride is negative.
uint64_t extent(int64_t rows, int64_t row, int64_t heads, int64_t head, int64_t count, int elem) {
  if (rows < 1 || heads < 1 || row < 0 || head < 0) return 0;
  return ((uint64_t)(rows - 1) * row + (uint64_t)(heads - 1) * head + count) * elem;
}

int elem_size(int dtype) { return dtype == COPES_BF16 ? 2 : 4; }

uint64_t pool_bytes(const copes::Cache &c) { return (uint64_t)c.n_pages * c.page_bytes; }

// Checks a cache and fills in what the kernels take.
int check_cache(const copes_kv_cache *p, copes::Cache *c, const char *who) {
  if (!p) return fail(COPES_ERR_INVALID_ARG, "%s: cache is NULL", who);
  if (!p->pool || !p->table || !p->length || !p->refs)
    return fail(COPES_ERR_INVALID_ARG, "%s: pool, table, length or refs is NULL", who);
  if (p->dtype != COPES_BF16 && p->dtype != COPES_FP32)
    return fail(COPES_ERR_INVALID_ARG, "%s: dtype %d is neither COPES_BF16 nor COPES_FP32", who, p->dtype);
  if (p->n_pages < 1 || p->n_layers < 1 || p->n_kv_heads < 1 || p->page_size < 1 || p->n_slots < 1 || p->table_width < 1)
    return fail(COPES_ERR_INVALID_ARG, "%s: every size of the cache must be at least 1", who);
  if (p->head_dim < 8 || p->head_dim > COPES_MAX_HEAD_DIM || p->head_dim % 8)
    return fail(COPES_ERR_SIZE, "%s: head_dim %d is not a multiple of 8 of at most %d", who, p->head_dim,
                COPES_MAX_HEAD_DIM);
  if (p->n_pages > COPES_MAX_PAGES)
    return fail(COPES_ERR_SIZE, "%s: more than %d pages", who, COPES_MAX_PAGES);
  const int64_t most = 0x7FFFFFFF;
  if ((int64_t)p->table_width * p->page_size > most || (int64_t)p->n_slots * p->table_width > most ||
      (int64_t)p->page_size * p->head_dim > most || p->n_layers > 65535 || p->n_kv_heads > 65535)
    return fail(COPES_ERR_SIZE, "%s: a slot, the table, a head's part of a page or an axis of it is too large", who);
  if (!aligned(p->pool, 16) || !aligned(p->table, 4) || !aligned(p->length, 4) || !aligned(p->refs, 4))
    return fail(COPES_ERR_ALIGNMENT, "%s: pool must be 16-byte aligned, table, length and refs 4-byte", who);
  c->pool = static_cast<char *>(p->pool);
  c->table = p->table;
  c->length = p->length;
  c->refs = p->refs;
  c->elem = elem_size(p->dtype);
  c->head_elems = (uint32_t)(p->page_size * p->head_dim);
  c->layer_elems = 2ull * p->n_kv_heads * c->head_elems;
  if (c->layer_elems > (1ull << 44) / p->n_layers)
    return fail(COPES_ERR_SIZE, "%s: a page of more than 2^44 elements", who);
  c->page_bytes = c->layer_elems * p->n_layers * c->elem;
  if (c->page_bytes > (1ull << 48) / p->n_pages) return fail(COPES_ERR_SIZE, "%s: a pool of more than 2^48 bytes", who);
  c->n_pages = p->n_pages;
  c->n_layers = p->n_layers;
  c->n_kv_heads = p->n_kv_heads;
  c->page_size = p->page_size;
  c->head_dim = p->head_dim;
  c->n_slots = p->n_slots;
  c->table_width = p->table_width;
  const void *part[4] = {p->pool, p->table, p->length, p->refs};
  const uint64_t bytes[4] = {pool_bytes(*c), 4ull * p->n_slots * p->table_width, 4ull * p->n_slots, 4ull * p->n_pages};
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < i; ++j)
      if (overlaps(part[i], bytes[i], part[j], bytes[j]))
        return fail(COPES_ERR_INVALID_ARG, "%s: pool, table, length and refs must be disjoint", who);
  return COPES_OK;
}

// A list of n slots, and n <= n_slots where they are distinct.
int check_list(const copes::Cache &c, const void *list, int n, bool distinct, const char *who) {
  if (n < 0) return fail(COPES_ERR_INVALID_ARG, "%s: n is negative", who);
  if (n && !list) return fail(COPES_ERR_INVALID_ARG, "%s: a list of ids is NULL", who);
  if (!aligned(list, 4)) return fail(COPES_ERR_ALIGNMENT, "%s: lists of ids must be 4-byte aligned", who);
  if (distinct && n > c.n_slots) return fail(COPES_ERR_SIZE, "%s: %d distinct slots of %d", who, n, c.n_slots);
  if (n > COPES_MAX_PAGES) return fail(COPES_ERR_SIZE, "%s: a list of more than %d", who, COPES_MAX_PAGES);
  return COPES_OK;
}

int check_workspace(const void *ws, size_t have, size_t need, const char *who) {
  if (!ws || have < need)
    return fail(COPES_ERR_WORKSPACE, "%s: a workspace of %zu bytes is needed, %zu given", who, need, ws ? have : (size_t)0);
  if (!aligned(ws, 16)) return fail(COPES_ERR_ALIGNMENT, "%s: the workspace must be 16-byte aligned", who);
  return COPES_OK;
}

// Arrays that a call reads or writes besides the cache's.
struct Array {
  const void *at;
  uint64_t bytes;
};
bool overlaps(const Array &a, const Array &b) { return overlaps(a.at, a.bytes, b.at, b.bytes); }
Array pool_of(const copes::Cache &c) { return {c.pool, pool_bytes(c)}; }
Array list_of(const int32_t *ids, int n) { return {ids, 4ull * n}; }

// Refuses arrays of which one lies in the cache's books (table, length, refs) or in another; `reading`:
// the last `reading` of them are only read, and may share memory with one another.
template <int N>
int check_disjoint(const copes::Cache &c, const Array (&a)[N], int reading, const char *who) {
  const Array books[3] = {{c.table, 4ull * c.n_slots * c.table_width}, {c.length, 4ull * c.n_slots}, {c.refs, 4ull * c.n_pages}};
  for (int i = 0; i < N; ++i) {
    for (const Array &b : books)
      if (overlaps(a[i], b))
        return fail(COPES_ERR_INVALID_ARG, "%s: an argument lies in the cache's table, length or refs", who);
    for (int j = 0; j < i && j < N - reading; ++j)
      if (overlaps(a[i], a[j])) return fail(COPES_ERR_INVALID_ARG, "%s: an output or the workspace lies in another argument", who);
  }
  return COPES_OK;
}

size_t cache_workspace(const copes::Cache &c) { return 4 * copes::cache_workspace_ints(c.n_pages, c.n_slots); }

}  // namespace

extern "C" {

size_t copes_cache_workspace_bytes(const copes_kv_cache *p) {
  copes::Cache c;
  return check_cache(p, &c, "copes_cache_workspace_bytes") ? 0 : cache_workspace(c);
}

int copes_cache_grow(const copes_kv_cache *p, const int32_t *slots, int n, const int32_t *add, int add_all,
                     void *workspace, size_t workspace_bytes, cudaStream_t stream) {
  const char *who = "copes_cache_grow";
  copes::Cache c;
  int rc = check_cache(p, &c, who);
  if (rc) return rc;
  if ((rc = check_list(c, slots, n, true, who))) return rc;
  if (!aligned(add, 4)) return fail(COPES_ERR_ALIGNMENT, "%s: add must be 4-byte aligned", who);
  if (!add && add_all < 0) return fail(COPES_ERR_INVALID_ARG, "%s: add_all is negative", who);
  if ((rc = check_workspace(workspace, workspace_bytes, cache_workspace(c), who))) return rc;
  const Array arrays[] = {{workspace, cache_workspace(c)}, pool_of(c), list_of(slots, n), list_of(add, n)};
  if ((rc = check_disjoint(c, arrays, 2, who))) return rc;
  return launch_status(copes::launch_cache_grow(c, slots, n, add, add_all, (int32_t *)workspace, stream), who);
}

int copes_cache_append(const copes_kv_cache *p, int layer, const int32_t *slots, const int32_t *position, int n,
                       const void *k, int64_t k_row, int64_t k_head, const void *v, int64_t v_row, int64_t v_head,
                       cudaStream_t stream) {
  const char *who = "copes_cache_append";
  copes::Cache c;
  int rc = check_cache(p, &c, who);
  if (rc) return rc;
  if (layer < 0 || layer >= c.n_layers) return fail(COPES_ERR_INVALID_ARG, "%s: layer %d of %d", who, layer, c.n_layers);
  if ((rc = check_list(c, slots ? slots : p->length, n, false, who))) return rc;
  if (!slots && n > c.n_slots) return fail(COPES_ERR_SIZE, "%s: %d rows without slots, and %d slots", who, n, c.n_slots);
  if (!aligned(position, 4)) return fail(COPES_ERR_ALIGNMENT, "%s: position must be 4-byte aligned", who);
  if (n && (!k || !v)) return fail(COPES_ERR_INVALID_ARG, "%s: k or v is NULL", who);
  if (!aligned(k, c.elem) || !aligned(v, c.elem))
    return fail(COPES_ERR_ALIGNMENT, "%s: k and v must be aligned to their type", who);
  if ((int64_t)n * c.n_kv_heads > 0x7FFFFFFF) return fail(COPES_ERR_SIZE, "%s: more than 2^31-1 rows of heads", who);
  if (overlaps(k, extent(n, k_row, c.n_kv_heads, k_head, c.head_dim, c.elem), c.pool, pool_bytes(c)) ||
      overlaps(v, extent(n, v_row, c.n_kv_heads, v_head, c.head_dim, c.elem), c.pool, pool_bytes(c)))
    return fail(COPES_ERR_INVALID_ARG, "%s: k, v and the pool must be disjoint", who);
  if (overlaps(list_of(slots, n), pool_of(c)) || overlaps(list_of(position, n), pool_of(c)))
    return fail(COPES_ERR_INVALID_ARG, "%s: a list of ids lies in the pool", who);
  return launch_status(copes::launch_cache_append(c, layer, slots, position, n, k, k_row, k_head, v, v_row, v_head,
                                                  stream), who);
}

int copes_cache_fork(const copes_kv_cache *p, const int32_t *parents, const int32_t *children, int n, void *workspace,
                     size_t workspace_bytes, cudaStream_t stream) {
  const char *who = "copes_cache_fork";
  copes::Cache c;
  int rc = check_cache(p, &c, who);
  if (rc) return rc;
  if ((rc = check_list(c, parents, n, true, who)) || (rc = check_list(c, children, n, true, who))) return rc;
  if ((rc = check_workspace(workspace, workspace_bytes, cache_workspace(c), who))) return rc;
  const Array arrays[] = {{workspace, cache_workspace(c)}, pool_of(c), list_of(parents, n), list_of(children, n)};
  if ((rc = check_disjoint(c, arrays, 2, who))) return rc;
  return launch_status(copes::launch_cache_fork(c, parents, children, n, (int32_t *)workspace, stream), who);
}

int copes_cache_free(const copes_kv_cache *p, const int32_t *slots, int n, cudaStream_t stream) {
  const char *who = "copes_cache_free";
  copes::Cache c;
  int rc = check_cache(p, &c, who);
  if (rc) return rc;
  if ((rc = check_list(c, slots, n, false, who))) return rc;
  const Array arrays[] = {list_of(slots, n)};
  if ((rc = check_disjoint(c, arrays, 1, who))) return rc;
  return launch_status(copes::launch_cache_free(c, slots, n, stream), who);
}

int copes_cache_compact(const copes_kv_cache *p, int32_t *counts, void *workspace, size_t workspace_bytes,
                        cudaStream_t stream) {
  const char *who = "copes_cache_compact";
  copes::Cache c;
  int rc = check_cache(p, &c, who);
  if (rc) return rc;
  if (!aligned(counts, 4)) return fail(COPES_ERR_ALIGNMENT, "%s: counts must be 4-byte aligned", who);
  if ((rc = check_workspace(workspace, workspace_bytes, cache_workspace(c), who))) return rc;
  const Array arrays[] = {{workspace, cache_workspace(c)}, pool_of(c), {counts, 8}};
  if ((rc = check_disjoint(c, arrays, 0, who))) return rc;
  return launch_status(copes::launch_cache_compact(c, counts, (int32_t *)workspace, stream), who);
}

int copes_cache_copy_pages(const copes_kv_cache *p, const int32_t *src, const int32_t *dst, int n, cudaStream_t stream) {
  const char *who = "copes_cache_copy_pages";
  copes::Cache c;
  int rc = check_cache(p, &c, who);
  if (rc) return rc;
  if ((rc = check_list(c, src, n, false, who)) || (rc = check_list(c, dst, n, false, who))) return rc;
  if (overlaps(list_of(src, n), pool_of(c)) || overlaps(list_of(dst, n), pool_of(c)))
    return fail(COPES_ERR_INVALID_ARG, "%s: a list of ids lies in the pool", who);
  return launch_status(copes::launch_cache_copy(c, src, dst, n, stream), who);
}

// Query heads come in whole groups of the cache's heads.  The kernel counts tiles of at least 16
// tokens of up to 8 heads, and two more for each row, in 32 bits.
static int check_q_heads(const copes::Cache &c, int n, int q_heads, const char *who) {
  if (q_heads < 1 || q_heads % c.n_kv_heads)
    return fail(COPES_ERR_INVALID_ARG, "%s: %d query heads on %d key-value heads", who, q_heads, c.n_kv_heads);
  const int64_t units = (int64_t)c.n_kv_heads * ((q_heads / c.n_kv_heads + 7) / 8);
  const int64_t tiles = ((int64_t)c.table_width * c.page_size + 15) / 16 + 2;
  if (q_heads > 65535 || (int64_t)n * q_heads > 0x7FFFFFFF || (int64_t)n * units > 0x7FFFFFFF / tiles)
    return fail(COPES_ERR_SIZE, "%s: too many query heads, or tokens that the tables have room for", who);
  return COPES_OK;
}

size_t copes_paged_attention_workspace_bytes(const copes_kv_cache *p, int n, int q_heads) {
  const char *who = "copes_paged_attention_workspace_bytes";
  copes::Cache c;
  if (check_cache(p, &c, who) || check_list(c, p->length, n, false, who) || check_q_heads(c, n, q_heads, who)) return 0;
  return copes::attend_workspace_bytes(c, n, q_heads);
}

int copes_paged_attention(const copes_kv_cache *p, int layer, const int32_t *slots, int n, const void *q, int64_t q_row,
                          int64_t q_head, int q_heads, float scale, void *out, float *lse, void *workspace,
                          size_t workspace_bytes, cudaStream_t stream) {
  const char *who = "copes_paged_attention";
  copes::AttendArgs a{};
  int rc = check_cache(p, &a.c, who);
  if (rc) return rc;
  const copes::Cache &c = a.c;
  if (layer < 0 || layer >= c.n_layers) return fail(COPES_ERR_INVALID_ARG, "%s: layer %d of %d", who, layer, c.n_layers);
  if ((rc = check_list(c, slots ? slots : p->length, n, false, who))) return rc;
  if (!slots && n > c.n_slots) return fail(COPES_ERR_SIZE, "%s: %d rows without slots, and %d slots", who, n, c.n_slots);
  if ((rc = check_q_heads(c, n, q_heads, who))) return rc;
  if (n && (!q || !out)) return fail(COPES_ERR_INVALID_ARG, "%s: q or out is NULL", who);
  if (!isfinite(scale * 1.44269504088896340736f))  // the kernel's, of log2
    return fail(COPES_ERR_INVALID_ARG, "%s: scale log2 e is not finite in fp32", who);
  if (!aligned(q, c.elem) || !aligned(out, 16) || !aligned(lse, 4))
    return fail(COPES_ERR_ALIGNMENT, "%s: out must be 16-byte aligned, q and lse to their type", who);
  const size_t need = copes::attend_workspace_bytes(c, n, q_heads);
  if ((rc = check_workspace(workspace, workspace_bytes, need, who))) return rc;
  const uint64_t rows = (uint64_t)n * q_heads;
  const Array written[] = {{out, rows * c.head_dim * c.elem}, {lse, rows * 4}, {workspace, need}},
              read[] = {pool_of(c), {q, extent(n, q_row, q_heads, q_head, c.head_dim, c.elem)}, list_of(slots, n)};
  if ((rc = check_disjoint(c, written, 0, who))) return rc;
  for (const Array &w : written)
    for (const Array &r : read)
      if (overlaps(w, r))
        return fail(COPES_ERR_INVALID_ARG, "%s: out, lse and the workspace must be disjoint from q, slots and the pool", who);
  a.layer = layer;
  a.n = n;
  a.q_heads = q_heads;
  a.slots = slots;
  a.q = q;
  a.q_row = q_row;
  a.q_head = q_head;
  a.scale = scale;
  a.out = out;
  a.lse = lse;
  return launch_status(copes::launch_paged_attention(p->dtype, a, workspace, stream), who);
}

int copes_token_logprobs(const void *logits, int dtype, int n, int vocab, int64_t row, const int64_t *target,
                         float scale, int top, float *logprob, float *entropy, int64_t *top_ids, float *top_logprobs,
                         cudaStream_t stream) {
  const char *who = "copes_token_logprobs";
  if (dtype != COPES_BF16 && dtype != COPES_FP32)
    return fail(COPES_ERR_INVALID_ARG, "%s: dtype %d is neither COPES_BF16 nor COPES_FP32", who, dtype);
  if (n < 0 || vocab < 1) return fail(COPES_ERR_INVALID_ARG, "%s: n is negative or vocab below 1", who);
  if (vocab > (1 << 30)) return fail(COPES_ERR_SIZE, "%s: a vocabulary of more than 2^30", who);
  if (!(scale > 0.0f) || !(scale <= 1e38f))
    return fail(COPES_ERR_INVALID_ARG, "%s: scale must be positive and at most 1e38", who);
  if (top < 0 || top > COPES_MAX_TOP || top > vocab)
    return fail(COPES_ERR_SIZE, "%s: top %d of a vocabulary of %d, at most %d", who, top, vocab, COPES_MAX_TOP);
  if (n && (!logits || !target || !logprob)) return fail(COPES_ERR_INVALID_ARG, "%s: logits, target or logprob is NULL", who);
  if (n && top && (!top_ids || !top_logprobs))
    return fail(COPES_ERR_INVALID_ARG, "%s: top_ids or top_logprobs is NULL", who);
  if (!aligned(logits, elem_size(dtype)) || !aligned(target, 8) || !aligned(logprob, 4) || !aligned(entropy, 4) ||
      !aligned(top_ids, 8) || !aligned(top_logprobs, 4))
    return fail(COPES_ERR_ALIGNMENT, "%s: an array is not aligned to its type", who);
  const uint64_t rows = n, alternatives = (uint64_t)n * top;
  const Array arrays[] = {{logprob, 4 * rows}, {entropy, 4 * rows}, {top_ids, 8 * alternatives}, {top_logprobs, 4 * alternatives},
                          {logits, extent(n, row, 1, 0, vocab, elem_size(dtype))}, {target, 8 * rows}};
  for (int i = 0; i < 6; ++i)
    for (int j = 0; j < i && j < 4; ++j)
      if (overlaps(arrays[i], arrays[j]))
        return fail(COPES_ERR_INVALID_ARG, "%s: an output overlaps the logits, target or another output", who);
  copes::LogprobArgs a{};
  a.logits = logits;
  a.row = row;
  a.target = target;
  a.n = n;
  a.vocab = vocab;
  a.top = top;
  a.scale = scale;
  a.logprob = logprob;
  a.entropy = entropy;
  a.top_ids = top_ids;
  a.top_logprobs = top_logprobs;
  return launch_status(copes::launch_token_logprobs(dtype, a, stream), who);
}

}  // extern "C"
