// The first half of attention over shared pages (pages_shared.cu): the tokens of a group over the blocks that all of them
// see, with the many-token kernel, for which the group is one entry.
#include "pages_chunk.cuh"

namespace less {

template <typename T, int D, bool E4M3>
static int launch_prefix_chunk(const PgParams& p, const PaSharedArgs& a, cudaStream_t s) {
  constexpr size_t smem = (size_t)(2 * PC_ROWS + 2 * PC_STAGES * PC_KEYS) * D * 2 + sizeof(PcShared);
  static std::atomic<unsigned long long> done{0};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return fail_cuda("cudaGetDevice");
  if (dev >= 64 || !(done.load(std::memory_order_relaxed) >> dev & 1)) {
    if (cudaFuncSetAttribute(pages_chunk_kernel<T, D, E4M3, kShared>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) !=
        cudaSuccess)
      return fail_cuda("shared memory opt-in of pages_chunk_kernel");
    if (dev < 64) done.fetch_or(1ull << dev, std::memory_order_relaxed);
  }
  const int64_t slots = (int64_t)a.rows * p.group / (2 * PC_ROWS) + a.n, heads = (int64_t)p.heads * a.nl;
  if (slots * heads >= 0x7fffffff) return LESS_ERR_INVALID_CONFIG;
  return pg_launch("pages_chunk_kernel", pages_chunk_kernel<T, D, E4M3, kShared>, dim3((unsigned)(slots * heads + 1), (unsigned)a.splits),
                   pc_threads(kShared), smem, s, p, a, a.splits);
}

int launch_pages_prefix(const PgParams& p, const PaSharedArgs& a, int dim, uint32_t flags, cudaStream_t s) {
  const bool e4m3 = flags & LESS_PAGES_E4M3;
  if (flags & LESS_PAGES_BF16) {
    if (dim == 128) return e4m3 ? launch_prefix_chunk<__nv_bfloat16, 128, true>(p, a, s) : launch_prefix_chunk<__nv_bfloat16, 128, false>(p, a, s);
    return e4m3 ? launch_prefix_chunk<__nv_bfloat16, 64, true>(p, a, s) : launch_prefix_chunk<__nv_bfloat16, 64, false>(p, a, s);
  }
  if (dim == 128) return e4m3 ? launch_prefix_chunk<__half, 128, true>(p, a, s) : launch_prefix_chunk<__half, 128, false>(p, a, s);
  return e4m3 ? launch_prefix_chunk<__half, 64, true>(p, a, s) : launch_prefix_chunk<__half, 64, false>(p, a, s);
}

}  // namespace less
