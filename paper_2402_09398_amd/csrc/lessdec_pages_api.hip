// C ABI of the paged cache: argument checks and launches.  Nothing here allocates, synchronises or keeps state between calls.
#include "lessdec_pages.h"

namespace {

using namespace lessdec;

inline bool aligned(const void *p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

bool shape_ok(const lessdec_pages_desc *d)
{
  if (!d) return false;
  if (d->slots < 1 || d->slots > LESSDEC_MAX_SLOTS || d->pages < 1 || d->pages >= 1 << 28) return false;
  if (d->page_tokens < kBlock || d->page_tokens > 1024 || d->page_tokens % kBlock) return false;
  if (d->table_len < 1 || (long)d->table_len * d->page_tokens > 1L << 30) return false;
  if (d->heads < 1 || (long)d->pages * d->heads * (d->page_tokens / kBlock) >= 1L << 31) return false;
  if (d->heads > 1024 || (d->head_dim != 64 && d->head_dim != 128)) return false;
  if (d->q_per_kv < 0 || d->q_per_kv > LESSDEC_MAX_Q_PER_KV || d->layers < 1 || d->layers > 1024) return false;
  if (d->dtype != LESSDEC_DTYPE_F16 && d->dtype != LESSDEC_DTYPE_BF16) return false;
  if (d->sinks < 0 || d->window < 0) return false;
  if (d->scale != 0.f && !(d->scale >= 0x1p-40f && d->scale <= 0x1p40f)) return false;
  return true;
}

size_t floats_for(const lessdec_pages_desc *d, int rows)
{
  return pages_attend_floats(d->slots, d->heads, d->q_per_kv > 1 ? d->q_per_kv : 1, d->head_dim, (long)d->table_len * d->page_tokens, rows);
}

// Workspace: counters of lessdec_pages_attend | its shares, or the lists of the other calls
constexpr size_t kCounterBytes = (3 * kPagesWorkers * sizeof(int) + 255) / 256 * 256;
inline void *scratch(const lessdec_pages_desc *d) { return static_cast<char *>(d->workspace) + kCounterBytes; }

size_t workspace_for(const lessdec_pages_desc *d, int rows)
{
  const size_t attend = rows > 0 ? floats_for(d, rows) * sizeof(float) : 0, lists = (size_t)d->pages * sizeof(int32_t);
  const size_t n = attend > lists ? attend : lists;
  return kCounterBytes + (n + 255) / 256 * 256;
}

enum Needs { kTables = 1, kPool = 2, kWork = 4 };

// rows: of lessdec_pages_attend
int check(const lessdec_pages_desc *d, int needs, int rows, int layer, Pages *c)
{
  if (!shape_ok(d) || layer < 0 || layer >= d->layers) return LESSDEC_EINVAL;
  if (!d->table || !d->length || !aligned(d->table, 4) || !aligned(d->length, 4)) return LESSDEC_EINVAL;
  if ((needs & kTables) && (!d->refs || !aligned(d->refs, 4))) return LESSDEC_EINVAL;
  if ((needs & kPool) && (!d->k_codes || !d->v_codes || !d->exps || !aligned(d->k_codes, 16) || !aligned(d->v_codes, 16) || !aligned(d->exps, 2)))
    return LESSDEC_EINVAL;
  if ((needs & kWork) && (!d->workspace || !aligned(d->workspace, 256) || d->workspace_bytes < workspace_for(d, rows))) return LESSDEC_EWORKSPACE;
  c->slots = d->slots; c->pages = d->pages; c->page_tokens = d->page_tokens; c->table_len = d->table_len;
  c->heads = d->heads; c->head_dim = d->head_dim; c->q_per_kv = d->q_per_kv > 1 ? d->q_per_kv : 1;
  const unsigned per = (unsigned)(d->page_tokens / kBlock);
  c->inverse = per == 1 ? 0 : (unsigned)(((1ull << 32) + per - 1) / per);
  // a window that no sequence outgrows is none: positions less the window then stay within an int for any window allowed
  c->sinks = d->sinks; c->window = d->window < d->table_len * d->page_tokens ? d->window : 0;
  const double scale = d->scale > 0.f ? (double)d->scale : d->head_dim == 64 ? 0.125 : 0.08838834764831845;
  c->scale_log2 = (float)(scale * 1.4426950408889634);
  const size_t blocks = (size_t)layer * d->pages * d->heads * (d->page_tokens / kBlock);
  c->k = d->k_codes ? d->k_codes + blocks * kBlock * d->head_dim : nullptr;
  c->v = d->v_codes ? d->v_codes + blocks * kBlock * d->head_dim : nullptr;
  c->exps = d->exps ? d->exps + blocks * 2 : nullptr;
  c->table = d->table; c->length = d->length; c->refs = d->refs;
  return LESSDEC_OK;
}

inline int result(hipError_t e) { return e == hipSuccess ? LESSDEC_OK : LESSDEC_EHIP; }

// elements from a row to the next; -1: not allowed
long row_stride(int64_t stride, long packed)
{
  if (stride == 0) return packed;
  return stride < packed || stride % 8 || stride > (int64_t)1 << 40 ? -1 : (long)stride;
}

}  // namespace

extern "C" {

size_t lessdec_pages_workspace_bytes(const lessdec_pages_desc *desc, int32_t max_rows)
{
  return !shape_ok(desc) || max_rows < 0 ? 0 : workspace_for(desc, max_rows);
}

int lessdec_pages_reset(const lessdec_pages_desc *desc, void *hip_stream)
{
  Pages c;
  const int rc = check(desc, kTables, 0, 0, &c);
  return rc ? rc : result(launch_pages_reset(c, (hipStream_t)hip_stream));
}

int lessdec_pages_reserve(const lessdec_pages_desc *desc, const int32_t *n_new, int32_t *granted, int32_t *plan, void *hip_stream)
{
  Pages c;
  const int rc = check(desc, kTables | kWork, 0, 0, &c);
  if (rc) return rc;
  if (!n_new || !plan || !aligned(n_new, 4) || !aligned(granted, 4) || !aligned(plan, 4)) return LESSDEC_EINVAL;
  if (granted == n_new || plan == n_new || plan == granted) return LESSDEC_EINVAL;
  return result(launch_pages_reserve(c, n_new, granted, plan, static_cast<int *>(scratch(desc)), (hipStream_t)hip_stream));
}

int lessdec_pages_select(const lessdec_pages_desc *desc, const int32_t *from, void *hip_stream)
{
  Pages c;
  const int rc = check(desc, kTables, 0, 0, &c);
  if (rc) return rc;
  if (!from || !aligned(from, 4) || from == desc->length || from == desc->table) return LESSDEC_EINVAL;
  return result(launch_pages_select(c, from, (hipStream_t)hip_stream));
}

int lessdec_pages_compact(const lessdec_pages_desc *desc, int32_t *plan, void *hip_stream)
{
  Pages c;
  const int rc = check(desc, kTables | kWork, 0, 0, &c);
  if (rc) return rc;
  if (!plan || !aligned(plan, 4)) return LESSDEC_EINVAL;
  return result(launch_pages_compact(c, plan, static_cast<int *>(scratch(desc)), (hipStream_t)hip_stream));
}

int lessdec_pages_copy(const lessdec_pages_desc *desc, const int32_t *plan, int32_t max_pairs, void *hip_stream)
{
  Pages c;
  const int rc = check(desc, kPool, 0, 0, &c);
  if (rc) return rc;
  if (!plan || !aligned(plan, 4) || max_pairs < 0) return LESSDEC_EINVAL;
  return max_pairs == 0 ? LESSDEC_OK : result(launch_pages_copy(c, desc->layers, plan, max_pairs, (hipStream_t)hip_stream));
}

int lessdec_pages_append(const lessdec_pages_desc *desc, int32_t layer, const void *k, const void *v, int64_t stride, const int32_t *start,
                         int32_t rows, void *hip_stream)
{
  Pages c;
  const int rc = check(desc, kPool, 0, layer, &c);
  if (rc) return rc;
  const long step = row_stride(stride, (long)desc->heads * desc->head_dim);
  if (step < 0 || rows < 0) return LESSDEC_EINVAL;
  if (rows == 0) return LESSDEC_OK;
  if (!k || !v || !start || !aligned(k, 16) || !aligned(v, 16) || !aligned(start, 4)) return LESSDEC_EINVAL;
  return result(launch_pages_append(c, desc->dtype, AppendArgs{k, v, step, start, rows}, (hipStream_t)hip_stream));
}

int lessdec_pages_attend(const lessdec_pages_desc *desc, int32_t layer, const void *q, int64_t stride, void *out, float *lse, const int32_t *start,
                         int32_t rows, int32_t max_new, void *hip_stream)
{
  Pages c;
  int rc = check(desc, kPool, 0, layer, &c);
  if (rc) return rc;
  const long step = row_stride(stride, (long)desc->heads * c.q_per_kv * desc->head_dim);
  if (step < 0 || rows < 0 || max_new < 0 || (long)rows * c.q_per_kv >= 1L << 31 || ((long)rows * c.q_per_kv / 128 + desc->slots) * desc->heads > 1L << 30) return LESSDEC_EINVAL;
  if (rows == 0 || max_new == 0) return LESSDEC_OK;
  rc = check(desc, kWork, rows, layer, &c);
  if (rc) return rc;
  if (!q || !out || !start || !aligned(q, 16) || !aligned(out, 16) || !aligned(lse, 4) || !aligned(start, 4)) return LESSDEC_EINVAL;
  AttendArgs a{q, step, out, lse, start, rows, max_new < rows ? max_new : rows, static_cast<int *>(desc->workspace),
               static_cast<float *>(scratch(desc))};
  return result(launch_pages_attend(c, desc->dtype, a, (hipStream_t)hip_stream));
}

int lessdec_pages_read(const lessdec_pages_desc *desc, int32_t layer, const int32_t *slots, int32_t n, int32_t first, int32_t count, void *K, void *V,
                       void *hip_stream)
{
  Pages c;
  const int rc = check(desc, kPool, 0, layer, &c);
  if (rc) return rc;
  if (n < 0 || n > 65535 || count < 0) return LESSDEC_EINVAL;
  if (n == 0 || count == 0) return LESSDEC_OK;
  if (!slots || !K || !V || !aligned(slots, 4) || !aligned(K, 16) || !aligned(V, 16)) return LESSDEC_EINVAL;
  return result(launch_pages_read(c, desc->dtype, ReadArgs{slots, n, first, count, K, V}, (hipStream_t)hip_stream));
}

}  // extern "C"
