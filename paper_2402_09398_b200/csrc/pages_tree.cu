// Groups of few rows whose sequences share their first pages (pages_shared.cu): the step kernel with a group as one entry.
#include "pages_step.cuh"

namespace less {

int launch_pages_tree(const PgParams& p, const PaSharedArgs& a, int dim, uint32_t flags, cudaStream_t s) {
  return launch_pages_step<kTree>(p, a, dim, flags, a.tile, LESS_PAGES_PARTIAL_BYTES, kPgCounters, s);
}

}  // namespace less
