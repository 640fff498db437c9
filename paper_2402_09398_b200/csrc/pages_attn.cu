// Host side of attention over the paged 8-bit cache: checks of arguments, and which of the two kernels takes which entries
// (pages_step.cuh: few new tokens per sequence; pages_chunk.cu: many).
#include "pages_step.cuh"

namespace less {

int pa_args(const less_pages* d, int32_t layer_begin, int32_t layer_count, int32_t n, const int32_t* seqs, const int32_t* starts,
            int32_t rows, int32_t max_new, const void* q, int64_t q_stride, int32_t window, int32_t sinks, float scale, void* out,
            PgParams* p, PaArgs* a) {
  a->n = 0;
  const int rc = pg_view(d, p);
  if (rc != LESS_OK) return rc;
  if (layer_begin < 0 || layer_count < 1 || layer_begin > d->layers - layer_count) return LESS_ERR_BAD_LAYER_RANGE;
  if (n < 0 || n > (1 << 24) || rows < 0 || (!starts && rows != n) || max_new < 1) return LESS_ERR_INVALID_CONFIG;
  if (window < 0 || sinks < 0 || !(scale > 0.f) || scale > 3e38f) return LESS_ERR_INVALID_CONFIG;
  // rows of a KV head, and items of all (8 rows or 16 each), are counted in 32 bits
  if ((int64_t)rows * d->group > 0x7fffffff) return LESS_ERR_INVALID_CONFIG;
  if (layer_count > 0x7fffffff / ((int64_t)rows * d->group / 8 + n + 1) / d->heads) return LESS_ERR_INVALID_CONFIG;
  if (n == 0 || rows == 0) return LESS_OK;
  if (!seqs || !q || !out) return LESS_ERR_NULL_POINTER;
  if (((uintptr_t)seqs | (uintptr_t)starts) & 3) return LESS_ERR_MISALIGNED;
  if (q_stride < (int64_t)layer_count * d->heads * d->group * d->head_dim) return LESS_ERR_INVALID_CONFIG;
  if ((((uintptr_t)q | (uintptr_t)out) & 15) || (q_stride & 7)) return LESS_ERR_MISALIGNED;
  // no position reaches 2^30
  *a = {q, out, q_stride, seqs, starts, n, rows, layer_begin, layer_count, 0x7fffffff,
        window > (1 << 30) ? 0 : window, sinks > (1 << 30) ? 1 << 30 : sinks, scale};
  return LESS_OK;
}

int launch_pages_attention(const PgParams& p, PaArgs a, int dim, uint32_t flags, int32_t max_new, cudaStream_t s) {
  if (!a.starts) max_new = 1;
  const int64_t most = (int64_t)max_new * p.group;
  int r = most > 0x7fffffff ? 0x7fffffff : (int)most;
  const int step_rows = (int64_t)a.n * a.nl * p.heads * 2 <= pg_sms() ? kStepRowsFew : kStepRows;
  if (r > step_rows) {
    a.max_rows = step_rows;
    const int rc = launch_pages_chunk(p, a, dim, flags, s);
    if (rc != LESS_OK || !a.starts || p.group > step_rows) return rc;   // without starts all entries are alike
    r = step_rows;
  }
  return launch_pages_step<kAll>(p, a, dim, flags, r, LESS_PAGES_PARTIAL_BYTES, kPgCounters, s);
}

}  // namespace less

using namespace less;

extern "C" int less_pages_attention(const less_pages* d, int32_t layer_begin, int32_t layer_count, int32_t n,
                                    const int32_t* seqs, const int32_t* starts, int32_t rows, int32_t max_new,
                                    const void* q, int64_t q_stride, int32_t window, int32_t sinks, float scale,
                                    void* out, void* stream) {
  PgParams p;
  PaArgs a;
  const int rc = pa_args(d, layer_begin, layer_count, n, seqs, starts, rows, max_new, q, q_stride, window, sinks, scale, out, &p, &a);
  if (rc != LESS_OK || a.n == 0) return rc;
  return launch_pages_attention(p, a, d->head_dim, d->flags, max_new, (cudaStream_t)stream);
}
