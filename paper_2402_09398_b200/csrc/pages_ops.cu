// Maps of the paged 8-bit cache: sequences grow, shrink, fork, lose what their window has left behind, and the pool
// closes up.  All of it runs on the device in stream order - lengths, tables and counts are device arrays that the
// host need not know - so that a captured step can allocate.
//
// Pages are handed out deterministically (the lowest free ones, in the order of the call's list).  The plan of a call
// is one block's work: the maps are small (4 bytes per page and per table entry), and the order is a prefix sum.
// Moving page contents is bound by memory (2 x bytes) and takes the whole GPU in a second launch, except in resize,
// where a page is copied only if a sequence grows inside a page that another one holds: there the plan's cluster of
// eight blocks copies, and the usual step pays one launch (4 such sequences in one layer 23 us; 96 in eight layers, 201 MB,
// 612 us, much more than a fork of as many).
//
// Measured, launches included: four children of one sequence freed and forked again (two calls, three launches) 14 us;
// 96 children of 32 sequences in eight layers, 8 heads (203 MB of pages copied): 37 us; a pool of 64
// sequences, a quarter of it ended, trimmed and closed up (196 MB): 51 us.  A plan is a chain of loads and scans in one
// block, some microseconds in which the rest of the GPU waits.
#include <atomic>
#include <string.h>

#include "less_internal.cuh"
#include "pages.cuh"

namespace less {

constexpr int PO_THREADS = 1024;
constexpr int PO_CLUSTER = 8;

// inclusive scan over the block's 1024 values, one per thread; *total = their sum.  Two barriers.
__device__ __forceinline__ int block_scan(int v, int* warp_sums, int* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int x = v;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, d);
    if (lane >= d) x += y;
  }
  __syncthreads();                                   // the sums of an earlier scan have been read
  if (lane == 31) warp_sums[warp] = x;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll 8
  for (int w = 0; w < PO_THREADS / 32; ++w) {
    const int y = warp_sums[w];
    before += w < warp ? y : 0;
    all += y;
  }
  *total = all;
  return x + before;
}

// The lowest `want` free pages (refs == 0) go to list[0 .. want) in ascending order; returns how many are free.
// A thread looks over a stretch of its own, so the order needs one scan.  Whole block.
// `first`: free_group of the thread's first four pages, which a caller that changes no counts before may ask for early.
__device__ __forceinline__ uint32_t free_group(const PgParams& p, int i, int end) {   // bit k: page i + k is free
  uint32_t f = 0;
  if (i + 4 <= end) {
    const int4 r = __ldcg(reinterpret_cast<const int4*>(p.refs + i));
    f = (r.x == 0) | (r.y == 0) << 1 | (r.z == 0) << 2 | (r.w == 0) << 3;
  } else {
    for (int j = i; j < end; ++j) f |= (uint32_t)(__ldcg(p.refs + j) == 0) << (j - i);
  }
  return f;
}
__device__ __forceinline__ int pages_per_thread(const PgParams& p) { return pg_ceil(pg_ceil(p.pages, PO_THREADS), 4) * 4; }
__device__ __forceinline__ uint32_t first_group(const PgParams& p) {
  const int begin = min(p.pages, (int)threadIdx.x * pages_per_thread(p));
  return free_group(p, begin, min(p.pages, begin + pages_per_thread(p)));
}
__device__ __forceinline__ int take_free(const PgParams& p, uint32_t first, int want, int* list, int* warp_sums) {
  const int per = pages_per_thread(p), begin = min(p.pages, (int)threadIdx.x * per), end = min(p.pages, begin + per);
  int mine = __popc(first);
  for (int i = begin + 4; i < end; i += 4) mine += __popc(free_group(p, i, end));
  int total;
  int at = block_scan(mine, warp_sums, &total) - mine;
  if (mine)
    for (int i = begin; i < end && at < want; i += 4)
      for (uint32_t f = i == begin ? first : free_group(p, i, end); f && at < want; f &= f - 1) list[at++] = i + __ffs(f) - 1;
  __syncthreads();
  return total;
}

__device__ __forceinline__ void copy_mags(const PgParams& p, int layer, int src, int dst, int tid, int threads) {
  const int m = p.heads * 2 * (p.pt / kPageBlock);
  const float* a = p.amax + pg_mag(p, layer, src, 0);
  float* b = p.amax + pg_mag(p, layer, dst, 0);
  for (int i = tid; i < m; i += threads) b[i] = __ldcg(a + i);
}

__device__ __forceinline__ void cluster_sync_all() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// A listed sequence found twice: the first entry counts.  A bitmap in shared memory tells whether there is any such;
// only then the first entries are worked out, in p.mark.
constexpr int PO_BITS = 65536;
struct Listed {
  uint32_t seen[PO_BITS / 32];
};
// whether thread-owned entry i (of the block's strided loop) sets a bit that is set already; caller synchronises before
__device__ __forceinline__ bool listed_again(Listed& l, const PgParams& p, int s) {
  if (p.seqs > PO_BITS) return true;                     // too many to tell: work it out
  return atomicOr(&l.seen[s >> 5], 1u << (s & 31)) >> (s & 31) & 1;
}

enum { kAnyBad = 1, kAnyAgain = 2, kAnyShrink = 4, kAnyGrow = 8 };

__global__ void __cluster_dims__(PO_CLUSTER, 1, 1) __launch_bounds__(PO_THREADS)
    pages_resize_kernel(PgParams p, int D, int n, const int32_t* seqs, const int32_t* want) {
  __shared__ int sums[PO_THREADS / 32];
  __shared__ Listed listed;
  __shared__ int nmoves;
  __shared__ uint32_t any;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  pg_wait();
  if (blockIdx.x == 0) {
    if (tid == 0) {
      nmoves = 0;
      any = 0;
    }
    for (int i = tid; i < min(PO_BITS, p.seqs + 31) / 32; i += PO_THREADS) listed.seen[i] = 0;
    uint32_t mine = pg_stopped(p) ? kAnyBad : 0;
    __syncthreads();
    // a list that holds a bad entry changes nothing
    for (int i = tid; i < n; i += PO_THREADS) {
      const int s = __ldg(seqs + i), w = __ldg(want + i);
      const int old = s >= 0 && s < p.seqs ? __ldcg(p.lens + s) : -1;
      if (w < 0 || w > p.seq_pages * p.pt || !pg_len_ok(p, old)) {
        pg_status(p.status, kPagesBounds, 10);
        mine |= kAnyBad;
      } else {
        if (listed_again(listed, p, s)) mine |= kAnyAgain;
        mine |= w < old ? kAnyShrink : w > old ? kAnyGrow : 0;
      }
    }
    mine = __reduce_or_sync(0xffffffffu, mine);
    if (lane == 0 && mine) atomicOr(&any, mine);
    __syncthreads();
    const uint32_t flags = any;
    if (!(flags & kAnyBad)) {
      const bool twice = flags & kAnyAgain;
      if (twice) {
        for (int i = tid; i < n; i += PO_THREADS) p.mark[seqs[i]] = n;
        __syncthreads();
        for (int i = tid; i < n; i += PO_THREADS) atomicMin(p.mark + seqs[i], i);
        __syncthreads();
      }
      auto counts = [&](int i, int s) { return !twice || __ldcg(p.mark + s) == i; };
      if (flags & kAnyShrink) {
        // pages behind the new ends
        for (int i = warp; i < n; i += PO_THREADS / 32) {
          const int s = __ldg(seqs + i), w = __ldg(want + i), old = __ldcg(p.lens + s);
          __syncwarp();
          if (w >= old || !counts(i, s)) continue;
          int32_t* row = p.table + (size_t)s * p.seq_pages;
          for (int o = pg_ceil(w, p.pt) + lane; o < min(p.seq_pages, pg_ceil(old, p.pt)); o += 32) {
            const int page = __ldcg(row + o);
            if (page >= 0 && page < p.pages) atomicSub(p.refs + page, 1);
            row[o] = -1;
          }
          if (lane == 0) p.lens[s] = w;
        }
        __syncthreads();
      }
      if (flags & kAnyGrow) {
        // how many pages every entry lacks, and from where in the list of free pages it takes them
        int total = 0;
        bool lost = false;
        for (int base = 0; base < n; base += PO_THREADS) {
          const int i = base + tid;
          int need = 0, split = 0;
          if (i < n) {
            const int s = __ldg(seqs + i), w = __ldg(want + i), old = __ldcg(p.lens + s);
            if (w > old && counts(i, s)) {
              if (old & (p.pt - 1)) {
                const int held = __ldcg(p.table + (size_t)s * p.seq_pages + (old >> p.pt_shift));
                lost |= held < 0 || held >= p.pages;       // cut back into pages that were trimmed
                split = held >= 0 && held < p.pages && __ldcg(p.refs + held) > 1;
              }
              need = pg_ceil(w, p.pt) - pg_ceil(old, p.pt) + split;
            }
          }
          int sum;
          const int upto = block_scan(need, sums, &sum);
          if (i < n) p.off[i] = (total + upto - need) * 2 + split;
          total += sum;
        }
        lost = __syncthreads_or(lost);
        const int free_pages = total ? take_free(p, first_group(p), total, p.fresh, sums) : 0;
        if (lost || total > free_pages) {                  // then no sequence grows
          if (tid == 0) pg_status(p.status, lost ? kPagesState : kPagesExhausted, 11);
        } else if (total == 0) {
          for (int i = tid; i < n; i += PO_THREADS) {
            const int s = __ldg(seqs + i);
            if (counts(i, s)) p.lens[s] = __ldg(want + i);   // those that shrink have their lengths already
          }
        } else {
          for (int i = warp; i < n; i += PO_THREADS / 32) {
            const int s = __ldg(seqs + i), w = __ldg(want + i), old = __ldcg(p.lens + s);
            __syncwarp();
            if (w <= old || !counts(i, s)) continue;
            const int at = __ldcg(p.off + i), split = at & 1;
            const int first = pg_ceil(old, p.pt) - split, need = pg_ceil(w, p.pt) - first;
            int32_t* row = p.table + (size_t)s * p.seq_pages + first;
            for (int k = lane; k < need; k += 32) {
              const int page = __ldcg(p.fresh + (at >> 1) + k);
              if (split && k == 0) {
                const int held = __ldcg(row), m = atomicAdd(&nmoves, 1);
                p.moves[1 + 2 * m] = held;
                p.moves[2 + 2 * m] = page;
                atomicSub(p.refs + held, 1);
              }
              row[k] = page;
              p.refs[page] = 1;
            }
            if (lane == 0) p.lens[s] = w;
          }
        }
      }
    }
    __syncthreads();
    if (tid == 0) p.moves[0] = nmoves;
  }
  cluster_sync_all();
  const int moves = __ldcg(p.moves);
  for (int m = 0; m < moves; ++m)
    for (int layer = 0; layer < p.layers; ++layer) {
      const int src = __ldcg(p.moves + 1 + 2 * m), dst = __ldcg(p.moves + 2 + 2 * m), units = p.heads * 2 * p.pt * D / 16;
      const uint4* from = reinterpret_cast<const uint4*>(p.codes + pg_slab(p, D, layer, src, 0));
      uint4* to = reinterpret_cast<uint4*>(p.codes + pg_slab(p, D, layer, dst, 0));
      for (int u = blockIdx.x * PO_THREADS + tid; u < units; u += PO_CLUSTER * PO_THREADS) to[u] = __ldcg(from + u);
      if ((int)blockIdx.x == layer % PO_CLUSTER) copy_mags(p, layer, src, dst, tid, PO_THREADS);
    }
}

// Fork, the plan: which pairs need a copy of the page that is still being filled, and which free page each gets.
// moves[0] = -1 tells the second kernel that the call was refused.
__global__ void __launch_bounds__(PO_THREADS) pages_fork_plan_kernel(PgParams p, int n, const int32_t* src,
                                                                     const int32_t* dst) {
  __shared__ int sums[PO_THREADS / 32];
  __shared__ Listed listed;
  const int tid = threadIdx.x;
  pg_wait();
  for (int i = tid; i < min(PO_BITS, p.seqs + 31) / 32; i += PO_THREADS) listed.seen[i] = 0;
  // asked for before they are needed: what is free, and (of the first entries) what is copied
  const uint32_t free4 = first_group(p);
  int held0 = -1, len0 = 0;
  bool bad = pg_stopped(p), again = false;
  __syncthreads();
  for (int i = tid; i < n; i += PO_THREADS) {
    const int a = __ldg(src + i), b = __ldg(dst + i);
    if (a < 0 || a >= p.seqs || b < 0 || b >= p.seqs || !pg_len_ok(p, __ldcg(p.lens + a))) {
      pg_status(p.status, kPagesBounds, 20);
      bad = true;
    } else {
      if (i == tid) {
        len0 = __ldcg(p.lens + a);
        if (len0 & (p.pt - 1)) held0 = __ldcg(p.table + (size_t)a * p.seq_pages + (len0 >> p.pt_shift));
      }
      if (__ldcg(p.lens + b) != 0) {                       // a destination is empty, listed once, and no source
        pg_status(p.status, kPagesState, 21);
        bad = true;
      }
      again |= listed_again(listed, p, b);
    }
  }
  const bool small = p.seqs <= PO_BITS;
  bad = __syncthreads_or(bad || (small && again));         // (twice among the destinations)
  if (small && again) pg_status(p.status, kPagesState, 21);
  if (!bad && !small) {
    for (int i = tid; i < n; i += PO_THREADS) {
      p.mark[src[i]] = n;
      p.mark[dst[i]] = n;
    }
    __syncthreads();
    for (int i = tid; i < n; i += PO_THREADS) atomicMin(p.mark + dst[i], i);
    __syncthreads();
  }
  if (!bad) {
    for (int i = tid; i < n; i += PO_THREADS) {
      const int a = __ldg(src + i), b = __ldg(dst + i);
      bad |= small ? listed.seen[a >> 5] >> (a & 31) & 1 : __ldcg(p.mark + b) != i || __ldcg(p.mark + a) != n;
    }
    if (bad) pg_status(p.status, kPagesState, 21);
    bad = __syncthreads_or(bad);
  }
  int total = 0;
  if (!bad) {
    for (int base = 0; base < n; base += PO_THREADS) {
      const int i = base + tid;
      int held = held0, len = len0;
      if (base && i < n) {
        held = -1;
        const int a = __ldg(src + i);
        len = __ldcg(p.lens + a);
        if (len & (p.pt - 1)) held = __ldcg(p.table + (size_t)a * p.seq_pages + (len >> p.pt_shift));
      }
      if (i >= n || held >= p.pages) held = -1;
      int sum;
      const int at = total + block_scan(held >= 0, sums, &sum) - 1;
      if (i < n) p.off[i] = held >= 0 ? at : -1;
      if (held >= 0) p.moves[1 + 2 * at] = held;
      total += sum;
    }
    const int free_pages = total ? take_free(p, free4, total, p.fresh, sums) : 0;
    if (total > free_pages) {
      if (tid == 0) pg_status(p.status, kPagesExhausted, 22);
      bad = true;
    } else {
      for (int k = tid; k < total; k += PO_THREADS) {
        const int page = __ldcg(p.fresh + k);
        p.moves[2 + 2 * k] = page;
        p.refs[page] = 1;
      }
    }
  }
  if (tid == 0) p.moves[0] = bad ? -1 : total;
}

// Compact, the plan: with `live` pages in use, the i-th page in use at or behind index `live` moves to the i-th free
// one before it.  fresh[page] = where a page in use is afterwards.
__global__ void __launch_bounds__(PO_THREADS) pages_compact_plan_kernel(PgParams p) {
  __shared__ int sums[PO_THREADS / 32];
  const int tid = threadIdx.x;
  pg_wait();
  if (pg_stopped(p)) {
    if (tid == 0) p.moves[0] = -1;
    return;
  }
  const int per = pg_ceil(pg_ceil(p.pages, PO_THREADS), 4) * 4;
  const int begin = min(p.pages, tid * per), end = min(p.pages, begin + per);
  int mine = 0;
  for (int i = begin; i < end; ++i) mine += __ldcg(p.refs + i) > 0;
  int live;
  block_scan(mine, sums, &live);
  // pages of this thread's stretch that move: holes before `live`, pages in use from there on
  int holes = 0, movers = 0;
  for (int i = begin; i < end; ++i) {
    const bool used = __ldcg(p.refs + i) > 0;
    holes += !used && i < live;
    movers += used && i >= live;
  }
  int all, h = block_scan(holes, sums, &all) - holes, m = block_scan(movers, sums, &all) - movers;
  for (int i = begin; i < end; ++i) {
    const bool used = __ldcg(p.refs + i) > 0;
    if (!used && i < live) p.moves[2 + 2 * h++] = i;
    if (used && i >= live) p.moves[1 + 2 * m++] = i;
    p.fresh[i] = i;
  }
  __syncthreads();
  for (int k = tid; k < all; k += PO_THREADS) {
    const int a = __ldcg(p.moves + 1 + 2 * k), b = __ldcg(p.moves + 2 + 2 * k);
    p.fresh[a] = b;
    p.refs[b] = __ldcg(p.refs + a);
    p.refs[a] = 0;
  }
  if (tid == 0) p.moves[0] = all;
}

// Carries out a plan: the table rows (fork: n rows; compact: every row), then the page copies, over the whole GPU.
// Sources and destinations are disjoint (destinations were free).
// A warp per run, 4 KB of it on their way, measured on the pool of 64 sequences: blocks instead of warps 66 us against 55,
// 8 KB on their way 56 against 50 (replayed), 4 CTAs per SM with fewer registers instead of 3 with 80: 52 against 50.
constexpr int PM_THREADS = 256, PM_UNITS = 8;          // 16-byte units of a lane on their way at once

template <bool FORK>
__global__ void __launch_bounds__(PM_THREADS) pages_move_kernel(PgParams p, int D, int n, const int32_t* src,
                                                                const int32_t* dst) {
  const int tid = threadIdx.x;
  pg_wait();
  const int moves = __ldcg(p.moves);
  if (moves < 0) return;
  const int rows = FORK ? n : p.seqs;
  for (int i = blockIdx.x; i < rows; i += gridDim.x) {
    if (FORK) {
      const int a = src[i], b = dst[i], len = __ldcg(p.lens + a), at = __ldcg(p.off + i);
      const int32_t* from = p.table + (size_t)a * p.seq_pages;
      int32_t* to = p.table + (size_t)b * p.seq_pages;
      const int whole = len >> p.pt_shift;
      for (int o = tid; o < p.seq_pages; o += PM_THREADS) {
        int page = -1;
        if (o < whole) {
          page = __ldcg(from + o);
          if (page >= 0 && page < p.pages) atomicAdd(p.refs + page, 1);
        } else if (o == whole && at >= 0) {
          page = __ldcg(p.moves + 2 + 2 * at);
        }
        to[o] = page;
      }
      if (tid == 0) p.lens[b] = len;
    } else {
      int32_t* row = p.table + (size_t)i * p.seq_pages;
      for (int o = tid; o < p.seq_pages; o += PM_THREADS) {
        const int page = __ldcg(row + o);
        if (page >= 0 && page < p.pages) row[o] = __ldcg(p.fresh + page);
      }
    }
  }
  // a warp per run (one head's keys or values of a page in one layer, 1 to 32 KB)
  const int lane = tid & 31, runs = p.heads * 2, per_move = p.layers * runs, run = p.pt * D / 16;
  const int64_t work = (int64_t)moves * per_move;
  for (int64_t w = (int64_t)blockIdx.x * (PM_THREADS / 32) + (tid >> 5); w < work; w += (int64_t)gridDim.x * (PM_THREADS / 32)) {
    // 64-bit divisions only where the numbers need them
    const int m = work <= 0x7fffffff ? (int)w / per_move : (int)(w / per_move);
    const int rest = (int)(w - (int64_t)m * per_move), layer = rest / runs, hw = rest - layer * runs;
    const int src_page = __ldcg(p.moves + 1 + 2 * m), dst_page = __ldcg(p.moves + 2 + 2 * m);
    const uint4* from = reinterpret_cast<const uint4*>(p.codes + pg_slab(p, D, layer, src_page, 0)) + (size_t)hw * run;
    uint4* to = reinterpret_cast<uint4*>(p.codes + pg_slab(p, D, layer, dst_page, 0)) + (size_t)hw * run;
    if (hw == 0) copy_mags(p, layer, src_page, dst_page, lane, 32);
    for (int u0 = 0; u0 < run; u0 += 32 * PM_UNITS) {
      uint4 x[PM_UNITS];
#pragma unroll
      for (int k = 0; k < PM_UNITS; ++k)
        if (u0 + 32 * k + lane < run) x[k] = __ldcg(from + u0 + 32 * k + lane);
#pragma unroll
      for (int k = 0; k < PM_UNITS; ++k)
        if (u0 + 32 * k + lane < run) __stcs(to + u0 + 32 * k + lane, x[k]);
    }
  }
}

// Reorder, the plan: entry i becomes what entry parents[i] was.  Whole pages are shared: their counts change by the number
// of an entry's children less one.  Of its children one inherits the page that is still being filled (the entry itself if
// it is its own child, else the first of the list), the others get copies in the lowest free pages, among them those that
// this call releases.  p.off[i] = number of the copy that entry i gets, p.mark[i] = its new length, both for the second
// kernel; a copy's source carries the number of its 16-token blocks in use, less one, in its top four bits.
// Bound by latency: a chain of some dependent loads and scans in one CTA, which all need all entries.  These lie in shared
// memory and four entries' pages are counted at a time (512 entries of up to 16 pages: 25 us with the entries in global
// memory, 18 us now).
constexpr int PO_REORDER = 8192;                       // entries of a call
constexpr int PO_ENTRY = 20;                           // bytes of each: sequence, length, parent, children, the first of them
__global__ void __launch_bounds__(PO_THREADS) pages_reorder_plan_kernel(PgParams p, int n, const int32_t* seqs,
                                                                        const int32_t* parents) {
  extern __shared__ int32_t po_entries[];
  __shared__ int sums[PO_THREADS / 32];
  __shared__ Listed listed;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  int32_t *seq = po_entries, *length = seq + n, *parent = length + n, *children = parent + n, *heir = children + n;
  pg_wait();
  for (int i = tid; i < min(PO_BITS, p.seqs + 31) / 32; i += PO_THREADS) listed.seen[i] = 0;
  bool bad = pg_stopped(p), again = false;
  __syncthreads();
  for (int i = tid; i < n; i += PO_THREADS) {
    const int s = __ldg(seqs + i), a = __ldcg(parents + i);   // (a selection has written the latter: past L1)
    const int len = s >= 0 && s < p.seqs ? __ldcg(p.lens + s) : -1;
    if (a < 0 || a >= n || !pg_len_ok(p, len)) {
      pg_status(p.status, kPagesBounds, 40);
      bad = true;
    } else {
      again |= listed_again(listed, p, s);
    }
    seq[i] = s;
    length[i] = len;
    parent[i] = a;
    children[i] = 0;
    heir[i] = 0x7fffffff;                              // -1: the entry itself
  }
  bad = __syncthreads_or(bad);
  if (!bad && p.seqs > PO_BITS) {                      // too many sequences for the bitmap
    for (int i = tid; i < n; i += PO_THREADS) p.mark[seq[i]] = n;
    __syncthreads();
    for (int i = tid; i < n; i += PO_THREADS) atomicMin(p.mark + seq[i], i);
    __syncthreads();
    again = false;
    for (int i = tid; i < n; i += PO_THREADS) again |= __ldcg(p.mark + seq[i]) != i;
  }
  if (!bad && again) pg_status(p.status, kPagesState, 41);
  if (__syncthreads_or(bad || again)) {
    if (tid == 0) p.moves[0] = -1;
    return;
  }
  for (int i = tid; i < n; i += PO_THREADS) {
    const int a = parent[i];
    atomicAdd(children + a, 1);
    atomicMin(heir + a, a == i ? -1 : i);
  }
  __syncthreads();
  // counts of the pages that lose or gain holders, four entries of a warp at a time; `sign` -1 takes it back
  auto count = [&](int sign) {
    constexpr int N = 4;
    for (int i0 = warp * N; i0 < n; i0 += PO_THREADS / 32 * N) {
      int most = 0;
#pragma unroll
      for (int k = 0; k < N; ++k)
        if (i0 + k < n && children[i0 + k] != 1) most = max(most, pg_ceil(length[i0 + k], p.pt));
      for (int o = lane; o < most; o += 32) {
        int page[N];
#pragma unroll
        for (int k = 0; k < N; ++k) {
          const int i = i0 + k;
          page[k] = -1;
          if (i < n && children[i] != 1 && o < pg_ceil(length[i], p.pt)) page[k] = __ldcg(p.table + (size_t)seq[i] * p.seq_pages + o);
        }
#pragma unroll
        for (int k = 0; k < N; ++k) {
          if (page[k] < 0 || page[k] >= p.pages) continue;
          const int more = children[i0 + k] - 1, d = o < length[i0 + k] >> p.pt_shift ? more : min(more, 0);
          if (d) atomicAdd(p.refs + page[k], sign * d);
        }
      }
    }
    __syncthreads();
  };
  count(1);
  // the copies: behind the counts, so that their pages are asked for while those are on their way
  int total = 0;
  for (int base = 0; base < n; base += PO_THREADS) {
    const int i = base + tid;
    int held = -1, used = 0;
    if (i < n) {
      const int a = parent[i], len = length[a], h = heir[a];
      if ((len & (p.pt - 1)) && (h < 0 ? a : h) != i) {
        held = __ldcg(p.table + (size_t)seq[a] * p.seq_pages + (len >> p.pt_shift));
        used = pg_ceil(len & (p.pt - 1), kPageBlock);
      }
      if (held >= p.pages) held = -1;
    }
    int sum;
    const int at = total + block_scan(held >= 0, sums, &sum) - 1;
    if (i < n) {
      p.off[i] = held >= 0 ? at : -1;
      p.mark[i] = length[parent[i]];
    }
    if (held >= 0) p.moves[1 + 2 * at] = (int)((uint32_t)held | (uint32_t)(used - 1) << 28);
    total += sum;
  }
  bad = total && take_free(p, first_group(p), total, p.fresh, sums) < total;
  if (bad) {
    count(-1);
    if (tid == 0) pg_status(p.status, kPagesExhausted, 42);
  } else {
    for (int k = tid; k < total; k += PO_THREADS) {
      const int page = __ldcg(p.fresh + k);
      p.moves[2 + 2 * k] = page;
      p.refs[page] = 1;
    }
  }
  if (tid == 0) p.moves[0] = bad ? -1 : total;
}

// Carries it out: the entries' rows of the table, a CTA per stretch of columns (in place, through shared memory), and the
// blocks in use of the pages that are copied, a warp per head's keys or values of one in one layer.  Bound by memory: a
// copied page's blocks in use are read and written once (512 sequences in eight layers, 176 MB: 36 us; both kernels 56 us.
// With the tables' rows in global memory and all columns in one CTA: 76 us).
__global__ void __launch_bounds__(PM_THREADS) pages_reorder_move_kernel(PgParams p, int D, int n, const int32_t* seqs,
                                                                        const int32_t* parents, int columns) {
  extern __shared__ int32_t po_rows[];                 // [n][columns]
  const int tid = threadIdx.x;
  pg_wait();
  const int moves = __ldcg(p.moves);
  if (moves < 0) return;
  for (int c0 = blockIdx.x * columns; c0 < p.seq_pages; c0 += gridDim.x * columns) {
    __syncthreads();
#pragma unroll 4
    for (int u = tid; u < n * columns; u += PM_THREADS) {
      const int i = u / columns, o = c0 + u - i * columns;
      if (o < p.seq_pages) po_rows[u] = __ldcg(p.table + (size_t)__ldg(seqs + i) * p.seq_pages + o);
    }
    __syncthreads();
#pragma unroll 4
    for (int u = tid; u < n * columns; u += PM_THREADS) {
      const int i = u / columns, o = c0 + u - i * columns, a = __ldcg(parents + i), copy = __ldcg(p.off + i), len = __ldcg(p.mark + i);
      if (a == i || o >= p.seq_pages) continue;
      int page = po_rows[a * columns + o - c0];
      if (copy >= 0 && o == len >> p.pt_shift) page = __ldcg(p.moves + 2 + 2 * copy);
      p.table[(size_t)__ldg(seqs + i) * p.seq_pages + o] = page;
    }
  }
  for (int i = blockIdx.x * PM_THREADS + tid; i < n; i += gridDim.x * PM_THREADS) p.lens[__ldg(seqs + i)] = __ldcg(p.mark + i);
  const int lane = tid & 31, runs = p.heads * 2, per_move = p.layers * runs, blocks = p.pt / kPageBlock;
  const int64_t work = (int64_t)moves * per_move;
  for (int64_t w = (int64_t)blockIdx.x * (PM_THREADS / 32) + (tid >> 5); w < work; w += (int64_t)gridDim.x * (PM_THREADS / 32)) {
    const int m = work <= 0x7fffffff ? (int)w / per_move : (int)(w / per_move);
    const int rest = (int)(w - (int64_t)m * per_move), layer = rest / runs, hw = rest - layer * runs;
    const uint32_t src = (uint32_t)__ldcg(p.moves + 1 + 2 * m);
    const int src_page = (int)(src & 0x0fffffffu), used = (int)(src >> 28) + 1, dst_page = __ldcg(p.moves + 2 + 2 * m);
    const int run = used * D;                          // 16-byte units
    const uint4* from = reinterpret_cast<const uint4*>(p.codes + pg_slab(p, D, layer, src_page, 0)) + (size_t)hw * p.pt * D / 16;
    uint4* to = reinterpret_cast<uint4*>(p.codes + pg_slab(p, D, layer, dst_page, 0)) + (size_t)hw * p.pt * D / 16;
    if (lane < used)
      p.amax[pg_mag(p, layer, dst_page, 0) + hw * blocks + lane] = __ldcg(p.amax + pg_mag(p, layer, src_page, 0) + hw * blocks + lane);
    for (int u0 = 0; u0 < run; u0 += 32 * PM_UNITS) {
      uint4 x[PM_UNITS];
#pragma unroll
      for (int k = 0; k < PM_UNITS; ++k)
        if (u0 + 32 * k + lane < run) x[k] = __ldcg(from + u0 + 32 * k + lane);
#pragma unroll
      for (int k = 0; k < PM_UNITS; ++k)
        if (u0 + 32 * k + lane < run) __stcs(to + u0 + 32 * k + lane, x[k]);
    }
  }
}

// Trim: a block per entry; an entry listed twice finds the pages gone (the exchange hands each out once)
__global__ void __launch_bounds__(128) pages_trim_kernel(PgParams p, int n, const int32_t* seqs, int sinks, int window) {
  pg_wait();
  const int s = seqs[blockIdx.x];
  if (__ldcg(p.status) != 0) return;
  if (s < 0 || s >= p.seqs) {
    if (threadIdx.x == 0) pg_status(p.status + kLateStatus, kPagesBounds, 30);
    return;
  }
  const int keep = __ldcg(p.lens + s) - window;          // first token that a window still covers
  int32_t* row = p.table + (size_t)s * p.seq_pages;
  for (int o = pg_ceil(sinks, p.pt) + threadIdx.x; o < p.seq_pages && (int64_t)(o + 1) * p.pt <= keep; o += 128) {
    if (__ldcg(row + o) < 0) continue;
    const int page = atomicExch(row + o, -1);
    if (page >= 0 && page < p.pages) atomicSub(p.refs + page, 1);
  }
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------
struct PgLayout {
  size_t moves, mark, off, fresh, counters, partial, shared, total;
};

// the workspace: status | counters | plan | partial results of attention | what its entries share
static PgLayout pg_layout(const less_pages* d) {
  PgLayout l;
  size_t at = 256;
  auto take = [&](size_t bytes) {
    const size_t r = at;
    at = (at + bytes + 255) / 256 * 256;
    return r;
  };
  const size_t most = (size_t)(d->pages > d->seqs ? d->pages : d->seqs);
  l.counters = take(kPgCounters * 4);
  l.moves = take((1 + 2 * most) * 4);
  l.mark = take((size_t)d->seqs * 4);
  l.off = take((size_t)d->seqs * 4);
  l.fresh = take(most * 4);
  l.partial = take(LESS_PAGES_PARTIAL_BYTES);
  l.shared = take((size_t)d->seqs * 48);
  l.total = at;
  return l;
}

static bool valid_pages(const less_pages* d) {
  if (d->layers < 1 || d->heads < 1 || d->pages < 1 || d->seqs < 1 || d->seq_pages < 1) return false;
  if (d->group < 1 || d->group > 128) return false;
  if (d->head_dim != 64 && d->head_dim != 128) return false;
  if (d->page_tokens < LESS_PAGE_BLOCK || d->page_tokens > 256 || (d->page_tokens & (d->page_tokens - 1))) return false;
  if (d->flags & ~(uint32_t)(LESS_PAGES_E4M3 | LESS_PAGES_BF16)) return false;
  if (d->layers > 65535 || d->pages > (1 << 28) || d->seqs > (1 << 24)) return false;
  if ((int64_t)d->seq_pages * d->page_tokens > (1 << 30)) return false;               // positions are 32-bit
  if ((int64_t)d->seqs * d->seq_pages > (1 << 29)) return false;                       // so are sums of table entries
  if ((int64_t)d->heads * d->group > 65535) return false;
  if ((int64_t)d->heads * 2 * d->page_tokens * d->head_dim > (1 << 30)) return false;  // a page of one layer
  return true;
}

int pg_view(const less_pages* d, PgParams* p) {
  if (!d) return LESS_ERR_NULL_POINTER;
  if (!valid_pages(d)) return LESS_ERR_INVALID_CONFIG;
  if (!d->codes || !d->amax || !d->table || !d->lens || !d->refs || !d->workspace) return LESS_ERR_NULL_POINTER;
  if (((uintptr_t)d->codes | (uintptr_t)d->amax | (uintptr_t)d->table | (uintptr_t)d->lens | (uintptr_t)d->refs) & 15)
    return LESS_ERR_MISALIGNED;
  if ((uintptr_t)d->workspace & 255) return LESS_ERR_MISALIGNED;
  const PgLayout l = pg_layout(d);
  if (d->workspace_bytes < l.total) return LESS_ERR_ARENA_TOO_SMALL;
  char* w = (char*)d->workspace;
  p->layers = d->layers;
  p->heads = d->heads;
  p->group = d->group;
  p->pt = d->page_tokens;
  p->pt_shift = 0;
  while ((1 << p->pt_shift) < d->page_tokens) ++p->pt_shift;
  p->pages = d->pages;
  p->seqs = d->seqs;
  p->seq_pages = d->seq_pages;
  p->codes = (uint8_t*)d->codes;
  p->amax = d->amax;
  p->table = d->table;
  p->lens = d->lens;
  p->refs = d->refs;
  p->status = (int32_t*)w;
  p->counters = (int32_t*)(w + l.counters);
  p->moves = (int32_t*)(w + l.moves);
  p->mark = (int32_t*)(w + l.mark);
  p->off = (int32_t*)(w + l.off);
  p->fresh = (int32_t*)(w + l.fresh);
  p->partial = (float*)(w + l.partial);
  return LESS_OK;
}

void* pg_shared(const less_pages* d) { return (char*)d->workspace + pg_layout(d).shared; }

int pg_sms() {
  static std::atomic<int> sms[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 148;
  int v = sms[dev].load(std::memory_order_relaxed);
  if (v == 0) {
    if (cudaDeviceGetAttribute(&v, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || v < 1) v = 148;
    sms[dev].store(v, std::memory_order_relaxed);
  }
  return v;
}

}  // namespace less

using namespace less;

extern "C" {

size_t less_pages_workspace_bytes(const less_pages* d) { return d && valid_pages(d) ? pg_layout(d).total : 0; }

int less_pages_reset(const less_pages* d, void* stream) {
  PgParams p;
  const int rc = pg_view(d, &p);
  if (rc != LESS_OK) return rc;
  cudaStream_t s = (cudaStream_t)stream;
  if (cudaMemsetAsync(d->table, 0xff, (size_t)d->seqs * d->seq_pages * 4, s) != cudaSuccess ||
      cudaMemsetAsync(d->lens, 0, (size_t)d->seqs * 4, s) != cudaSuccess ||
      cudaMemsetAsync(d->refs, 0, (size_t)d->pages * 4, s) != cudaSuccess ||
      cudaMemsetAsync(d->workspace, 0, pg_layout(d).moves, s) != cudaSuccess)
    return fail_cuda("less_pages_reset");
  return LESS_OK;
}

int less_pages_resize(const less_pages* d, int32_t n, const int32_t* seqs, const int32_t* lens, void* stream) {
  PgParams p;
  const int rc = pg_view(d, &p);
  if (rc != LESS_OK) return rc;
  if (n < 0 || n > d->seqs) return LESS_ERR_INVALID_CONFIG;
  if (n == 0) return LESS_OK;
  if (!seqs || !lens) return LESS_ERR_NULL_POINTER;
  if (((uintptr_t)seqs | (uintptr_t)lens) & 3) return LESS_ERR_MISALIGNED;
  return pg_launch("pages_resize_kernel", pages_resize_kernel, dim3(PO_CLUSTER), PO_THREADS, 0, (cudaStream_t)stream, p, d->head_dim, n, seqs,
                   lens);
}

int less_pages_fork(const less_pages* d, int32_t n, const int32_t* src, const int32_t* dst, void* stream) {
  PgParams p;
  int rc = pg_view(d, &p);
  if (rc != LESS_OK) return rc;
  if (n < 0 || n > d->seqs) return LESS_ERR_INVALID_CONFIG;
  if (n == 0) return LESS_OK;
  if (!src || !dst) return LESS_ERR_NULL_POINTER;
  if (((uintptr_t)src | (uintptr_t)dst) & 3) return LESS_ERR_MISALIGNED;
  rc = pg_launch("pages_fork_plan_kernel", pages_fork_plan_kernel, dim3(1), PO_THREADS, 0, (cudaStream_t)stream, p, n, src, dst);
  if (rc != LESS_OK) return rc;
  const int64_t ctas = n + (int64_t)n * d->layers * pg_ceil(d->heads * 2, PM_THREADS / 32);
  const int grid = (int)(ctas < 8 * pg_sms() ? ctas : 8 * pg_sms());
  return pg_launch("pages_move_kernel", pages_move_kernel<true>, dim3(grid), PM_THREADS, 0, (cudaStream_t)stream, p, d->head_dim, n, src, dst);
}

int less_pages_reorder(const less_pages* d, int32_t n, const int32_t* seqs, const int32_t* parents, void* stream) {
  PgParams p;
  int rc = pg_view(d, &p);
  if (rc != LESS_OK) return rc;
  if (n < 0 || n > d->seqs || n > PO_REORDER) return LESS_ERR_INVALID_CONFIG;
  if (n == 0) return LESS_OK;
  if (!seqs || !parents) return LESS_ERR_NULL_POINTER;
  if (((uintptr_t)seqs | (uintptr_t)parents) & 3) return LESS_ERR_MISALIGNED;
  cudaStream_t s = (cudaStream_t)stream;
  static std::atomic<unsigned long long> done{0};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return fail_cuda("cudaGetDevice");
  if (dev >= 64 || !(done.load(std::memory_order_relaxed) >> dev & 1)) {
    if (cudaFuncSetAttribute(pages_reorder_plan_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, PO_REORDER * PO_ENTRY) != cudaSuccess)
      return fail_cuda("shared memory opt-in of pages_reorder_plan_kernel");
    if (dev < 64) done.fetch_or(1ull << dev, std::memory_order_relaxed);
  }
  rc = pg_launch("pages_reorder_plan_kernel", pages_reorder_plan_kernel, dim3(1), PO_THREADS, (size_t)n * PO_ENTRY, s, p, n, seqs, parents);
  if (rc != LESS_OK) return rc;
  // columns of the table that a CTA takes at a time: about a thousand cells
  int columns = 1024 / n;
  if (columns > d->seq_pages) columns = d->seq_pages;
  if (columns < 1) columns = 1;
  // at most every entry but one of a family has a page copied
  const int64_t ctas = (int64_t)n * d->layers * pg_ceil(d->heads * 2, PM_THREADS / 32), cuts = pg_ceil(d->seq_pages, columns);
  const int64_t most = ctas > cuts ? ctas : cuts;
  const int grid = (int)(most < 8 * pg_sms() ? most : 8 * pg_sms());
  return pg_launch("pages_reorder_move_kernel", pages_reorder_move_kernel, dim3(grid), PM_THREADS, (size_t)n * columns * 4, s, p, d->head_dim,
                   n, seqs, parents, columns);
}

int less_pages_trim(const less_pages* d, int32_t n, const int32_t* seqs, int32_t sinks, int32_t window, void* stream) {
  PgParams p;
  const int rc = pg_view(d, &p);
  if (rc != LESS_OK) return rc;
  if (n < 0 || n > d->seqs || sinks < 0 || window < 1) return LESS_ERR_INVALID_CONFIG;
  if (sinks > (1 << 30)) sinks = 1 << 30;                // no sequence is longer
  if (n == 0) return LESS_OK;
  if (!seqs) return LESS_ERR_NULL_POINTER;
  if ((uintptr_t)seqs & 3) return LESS_ERR_MISALIGNED;
  return pg_launch("pages_trim_kernel", pages_trim_kernel, dim3(n), 128, 0, (cudaStream_t)stream, p, n, seqs, sinks, window);
}

int less_pages_compact(const less_pages* d, void* stream) {
  PgParams p;
  int rc = pg_view(d, &p);
  if (rc != LESS_OK) return rc;
  rc = pg_launch("pages_compact_plan_kernel", pages_compact_plan_kernel, dim3(1), PO_THREADS, 0, (cudaStream_t)stream, p);
  if (rc != LESS_OK) return rc;
  return pg_launch("pages_move_kernel", pages_move_kernel<false>, dim3(8 * pg_sms()), PM_THREADS, 0, (cudaStream_t)stream, p, d->head_dim, 0,
                   (const int32_t*)nullptr, (const int32_t*)nullptr);
}

int less_pages_poll_status(const less_pages* d, void* stream) {
  PgParams p;
  const int rc = pg_view(d, &p);
  if (rc != LESS_OK) return rc;
  cudaStream_t s = (cudaStream_t)stream;
  int32_t st[4] = {0, 0, 0, 0};
  if (cudaMemcpyAsync(st, p.status, 16, cudaMemcpyDeviceToHost, s) != cudaSuccess ||
      cudaStreamSynchronize(s) != cudaSuccess)
    return fail_cuda("less_pages_poll_status");
  if (st[0] == 0) st[0] = st[kLateStatus];
  if (st[0] == 0) return LESS_OK;
  if (cudaMemsetAsync(p.status, 0, 16, s) != cudaSuccess) return fail_cuda("less_pages_poll_status");
  if (st[0] == kPagesExhausted) return LESS_ERR_PAGES_EXHAUSTED;
  if (st[0] == kPagesState) return LESS_ERR_BAD_STATE;
  return st[0] == kStatusTimeout ? LESS_ERR_DEVICE_TIMEOUT : LESS_ERR_DEVICE_BOUNDS;
}

}  // extern "C"
