// Reordering of a context's batch rows in place (a step of beam search): row b becomes what row parents[b] was, in all
// arrays of the state.
//
// Bound by memory: the rows that somebody else becomes are read once, the rows that change are written once.  The arrays are
// batch-major, so a group's rows are `beams` byte strings, and what a CTA takes of them (a piece of the same bytes of every
// row) can be permuted without regard to any other CTA: it brings the pieces of all sources into shared memory, waits, and
// writes.  Two such tiles per CTA, so that one is on its way while the other is written; two CTAs per multiprocessor.
// A warp takes a row's piece: 8 groups of 8 rows, 2.69 GB read and written: 482 us, 5.6 TB/s (a thread per unit of any row,
// with a division each: 509 us).  A state of 2 MB: 5.3 - 8 us, which is the launch and the two looks at the parents.
#include <atomic>

#include "less_internal.cuh"
#include "pipeline.cuh"

namespace less {

constexpr int RO_THREADS = 256, RO_CTAS = 2;
constexpr int RO_UNITS = 48 * 1024 / 16;                  // 16-byte units of a tile
constexpr int RO_BEAMS = 2048;                            // rows of a group at most: a unit of each in a tile
constexpr int RO_ARRAYS = 7;

struct RoArgs {
  unsigned char* base[RO_ARRAYS];
  int64_t units[RO_ARRAYS];                               // 16-byte units of a row
  int64_t tiles[RO_ARRAYS + 1];                           // tiles of a group before the array's
  int32_t* count;                                         // [batch][count_row]
  int count_row;
  const int32_t* parents;
  int32_t* status;
  int batch, beams, width;                                // width: units of a row in a tile
};

__device__ __forceinline__ void ro_copy16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}

__global__ void __launch_bounds__(RO_THREADS, RO_CTAS) state_reorder_kernel(RoArgs a) {
  extern __shared__ __align__(16) unsigned char ro_smem[];  // two tiles, then the lists
  int16_t* slot = reinterpret_cast<int16_t*>(ro_smem + 2 * RO_UNITS * 16);   // [beams] of a row: its place among the sources, -1
  int16_t* source = slot + a.beams;                         // [sources] rows
  int16_t* moved = source + a.beams;                        // [moved] rows that change
  int16_t* from = moved + a.beams;                          // [moved] place of their parents
  __shared__ int sources, moves;
  const int tid = threadIdx.x;
  pdl_wait_primary();
  // (no early launch of dependents: a decode kernel may read the state as soon as the kernel before its step's first is done)
  bool bad = false;
  for (int b = tid; b < a.batch; b += RO_THREADS) {
    const int p = __ldcg(a.parents + b), g = b / a.beams * a.beams;
    bad |= p < g || p >= g + a.beams;
  }
  if (__syncthreads_or(bad)) {                              // nothing changes
    if (tid == 0) set_status(a.status, kStatusBounds, 95);
    return;
  }
  const int64_t per_group = a.tiles[RO_ARRAYS], total = per_group * (a.batch / a.beams);
  const int64_t begin = total * blockIdx.x / gridDim.x, end = total * (blockIdx.x + 1) / gridDim.x;
  int group = -1;
  const uint32_t smem = smem_u32(ro_smem);

  struct Tile {
    const unsigned char* row0;                              // first unit of the tile in the group's first row
    int64_t pitch;
    int n;                                                  // units per row
  };
  auto tile = [&](int64_t t) {
    Tile x;
    const int g = (int)(t / per_group);
    const int64_t u = t - g * per_group;
    int k = 0;
    while (u >= a.tiles[k + 1]) ++k;
    const int64_t first = (u - a.tiles[k]) * a.width;
    x.pitch = a.units[k] * 16;
    x.row0 = a.base[k] + (int64_t)g * a.beams * x.pitch + first * 16;
    x.n = (int)min((int64_t)a.width, a.units[k] - first);
    return x;
  };
  // the lists of a group; the block has read those of the one before
  auto enter = [&](int g) {
    __syncthreads();
    for (int b = tid; b < a.beams; b += RO_THREADS) slot[b] = -1;
    if (tid == 0) sources = moves = 0;
    __syncthreads();
    for (int b = tid; b < a.beams; b += RO_THREADS) {
      const int p = __ldcg(a.parents + g * a.beams + b) - g * a.beams;
      if (p != b) {
        moved[atomicAdd(&moves, 1)] = (int16_t)b;
        slot[p] = 0;
      }
    }
    __syncthreads();
    for (int b = tid; b < a.beams; b += RO_THREADS)
      if (slot[b] == 0) {
        const int s = atomicAdd(&sources, 1);
        source[s] = (int16_t)b;
        slot[b] = (int16_t)s;
      }
    __syncthreads();
    for (int i = tid; i < moves; i += RO_THREADS) from[i] = slot[__ldcg(a.parents + g * a.beams + moved[i]) - g * a.beams];
    __syncthreads();
  };
  auto fetch = [&](const Tile& x, int buf) {
    for (int s = tid >> 5; s < sources; s += RO_THREADS / 32) {
      const unsigned char* from_row = x.row0 + source[s] * x.pitch;
      const uint32_t to = smem + (uint32_t)(buf * RO_UNITS + s * x.n) * 16;
      for (int u = tid & 31; u < x.n; u += 32) ro_copy16(to + u * 16, from_row + (int64_t)u * 16);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };

  Tile cur = {};
  for (int64_t t = begin; t < end; ++t) {
    const int buf = (int)(t - begin) & 1;
    const int g = (int)(t / per_group);
    if (g != group) {                                       // a new group: nothing is on its way
      enter(g);
      group = g;
      if (moves == 0) {                                     // a group in which all beams live on
        t = min(end, (g + 1) * per_group) - 1;
        continue;
      }
      cur = tile(t);
      fetch(cur, buf);
      if (t == g * per_group) {                             // live slots: 4 bytes per instance, rows need not be 16-byte aligned
        int32_t* row = a.count + (int64_t)g * a.beams * a.count_row;
        const int columns = min(RO_THREADS, RO_UNITS * 4 / a.beams);   // a thread owns a column
        int32_t* tmp = reinterpret_cast<int32_t*>(ro_smem + (buf ^ 1) * RO_UNITS * 16) + tid;
        for (int i = tid; i < a.count_row && tid < columns; i += columns) {
          for (int s = 0; s < sources; ++s) tmp[s * columns] = __ldcg(row + (int64_t)source[s] * a.count_row + i);
          for (int m = 0; m < moves; ++m) row[(int64_t)moved[m] * a.count_row + i] = tmp[from[m] * columns];
        }
        __syncthreads();
      }
    }
    Tile nxt = {};
    const bool more = t + 1 < end && (t + 1) / per_group == g;
    if (more) {
      nxt = tile(t + 1);
      fetch(nxt, buf ^ 1);
      asm volatile("cp.async.wait_group 1;" ::: "memory");
    } else {
      asm volatile("cp.async.wait_group 0;" ::: "memory");
    }
    __syncthreads();
    const uint4* in = reinterpret_cast<const uint4*>(ro_smem) + buf * RO_UNITS;
    for (int m = tid >> 5; m < moves; m += RO_THREADS / 32) {
      uint4* dst = reinterpret_cast<uint4*>(const_cast<unsigned char*>(cur.row0) + moved[m] * cur.pitch);
      const uint4* src = in + from[m] * cur.n;
#pragma unroll 4
      for (int u = tid & 31; u < cur.n; u += 32) dst[u] = src[u];
    }
    __syncthreads();
    cur = nxt;
  }
}

}  // namespace less

using namespace less;

extern "C" int less_reorder(less_ctx* c, int32_t beams, const int32_t* parents, void* stream) {
  if (!c || !parents) return LESS_ERR_NULL_POINTER;
  if (beams < 1 || beams > RO_BEAMS || c->d.B % beams) return LESS_ERR_INVALID_CONFIG;
  if ((uintptr_t)parents & 3) return LESS_ERR_MISALIGNED;
  const Dims& d = c->d;
  const int64_t n = (int64_t)d.L * d.Hd;                    // instances of a batch row
  const int64_t bytes[RO_ARRAYS] = {n * d.N * d.D * 2, n * d.N * d.D * 2, n * d.Np * 4, n * d.Np * 4,
                                    n * d.N * d.R * 4, n * d.R * d.D * 4, n * d.R * 4};
  void* base[RO_ARRAYS] = {c->a.kslots, c->a.vslots, c->a.pos, c->a.acc, c->a.psic, c->a.H, c->a.z};
  RoArgs a = {};
  a.width = RO_UNITS / beams;
  for (int k = 0; k < RO_ARRAYS; ++k) {
    a.base[k] = (unsigned char*)base[k];
    a.units[k] = bytes[k] / 16;
    a.tiles[k + 1] = a.tiles[k] + (a.units[k] + a.width - 1) / a.width;
  }
  a.count = c->a.count;
  a.count_row = (int)n;
  a.parents = parents;
  a.status = c->a.status;
  a.batch = d.B;
  a.beams = beams;
  const size_t smem = (size_t)2 * RO_UNITS * 16 + (size_t)4 * beams * 2;
  static std::atomic<unsigned long long> done{0};
  if (c->device >= 64 || !(done.load(std::memory_order_relaxed) >> c->device & 1)) {
    if (cudaFuncSetAttribute(state_reorder_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 2 * RO_UNITS * 16 + 8 * RO_BEAMS) !=
        cudaSuccess)
      return fail_cuda("shared memory opt-in of state_reorder_kernel");
    if (c->device < 64) done.fetch_or(1ull << c->device, std::memory_order_relaxed);
  }
  const int64_t tiles = a.tiles[RO_ARRAYS] * (d.B / beams);
  const int grid = (int)(tiles < (int64_t)RO_CTAS * c->sms ? tiles : (int64_t)RO_CTAS * c->sms);
  cudaStream_t s = (cudaStream_t)stream;
  c->launches += 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(RO_THREADS);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = c->pdl && !c->profile ? 1 : 0;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, state_reorder_kernel, a);
  return e == cudaSuccess ? check_launch("state_reorder_kernel") : fail_cuda("state_reorder_kernel", e);
}

extern "C" int less_state_view(less_ctx* c, less_state* out) {
  if (!c || !out) return LESS_ERR_NULL_POINTER;
  *out = {c->a.kslots, c->a.vslots, c->a.pos, c->a.acc, c->a.psic, c->a.H, c->a.z, c->a.count, c->d.N, c->d.Np};
  return LESS_OK;
}
