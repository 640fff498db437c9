// Host side of the many-token kernel (pages_chunk.cuh): how far keys are split, and the launches.
#include "pages_chunk.cuh"

namespace less {

template <typename T, int D, bool E4M3>
static int launch_chunk(const PgParams& p, const PaArgs& a, cudaStream_t s) {
  constexpr size_t smem = (size_t)(2 * PC_ROWS + 2 * PC_STAGES * PC_KEYS) * D * 2 + sizeof(PcShared);
  static std::atomic<unsigned long long> done{0};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return fail_cuda("cudaGetDevice");
  if (dev >= 64 || !(done.load(std::memory_order_relaxed) >> dev & 1)) {
    if (cudaFuncSetAttribute(pages_chunk_kernel<T, D, E4M3, kAll>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) !=
        cudaSuccess)
      return fail_cuda("shared memory opt-in of pages_chunk_kernel");
    if (dev < 64) done.fetch_or(1ull << dev, std::memory_order_relaxed);
  }
  const int64_t slots = (int64_t)a.rows * p.group / (2 * PC_ROWS) + a.n, heads = (int64_t)p.heads * a.nl;
  if (slots * heads >= 0x7fffffff) return LESS_ERR_INVALID_CONFIG;
  // Items that are sure to exist; with fewer of them than multiprocessors their keys are split (measured: two sequences of
  // 30 000 tokens, eight KV heads, 48 rows each: 489 us unsplit, 82 us in nine parts)
  int64_t items = (int64_t)a.rows * p.group / (2 * PC_ROWS);
  if (items < a.n) items = a.n;
  int64_t splits = pg_sms() / (items * heads);
  const int64_t room = (int64_t)(LESS_PAGES_PARTIAL_BYTES / ((size_t)2 * PC_ROWS * (D + 2) * 4)) / (slots * heads);
  splits = splits > 32 ? 32 : splits;
  splits = splits > room ? room : splits;
  splits = splits < 1 ? 1 : splits;
  const int rc = pg_launch("pages_chunk_kernel", pages_chunk_kernel<T, D, E4M3, kAll>, dim3((unsigned)(slots * heads + 1), (unsigned)splits),
                           pc_threads(kAll), smem, s, p, a, (int)splits);
  if (rc != LESS_OK || splits == 1) return rc;
  const int64_t warps = (int64_t)a.rows * heads * p.group;
  return pg_launch("pages_chunk_join_kernel", pages_chunk_join_kernel<T, D>, dim3((unsigned)((warps + 7) / 8)), 256, 0, s, p, a,
                   (int)splits);
}

int launch_pages_chunk(const PgParams& p, const PaArgs& a, int dim, uint32_t flags, cudaStream_t s) {
  const bool e4m3 = flags & LESS_PAGES_E4M3;
  if (flags & LESS_PAGES_BF16) {
    if (dim == 128) return e4m3 ? launch_chunk<__nv_bfloat16, 128, true>(p, a, s) : launch_chunk<__nv_bfloat16, 128, false>(p, a, s);
    return e4m3 ? launch_chunk<__nv_bfloat16, 64, true>(p, a, s) : launch_chunk<__nv_bfloat16, 64, false>(p, a, s);
  }
  if (dim == 128) return e4m3 ? launch_chunk<__half, 128, true>(p, a, s) : launch_chunk<__half, 128, false>(p, a, s);
  return e4m3 ? launch_chunk<__half, 64, true>(p, a, s) : launch_chunk<__half, 64, false>(p, a, s);
}

}  // namespace less
