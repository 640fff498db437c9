// Attention of a few new tokens per sequence over the paged 8-bit cache (the step kernel):
//
//   o = sum_j p_j v_j / sum_j p_j,   p_j = exp(scale q . k_j),   j <= i, and (j > i - window or j < sinks)
//
// Bound by memory: every visible code is read once (2 D bytes per token and KV head; 4 D flops per byte pair and
// query head).  So the whole kernel is built around the stream of code tiles:
//   - The work - (sequence, layer, head, group of rows) items of as many 16-token blocks as the item sees - is one
//     long list of blocks that is cut into equal stretches, one per warp of a grid that just fills the GPU: a batch
//     of one long sequence and a ragged batch load it alike.  Lengths are read on the device.  What of an item a
//     warp did not do alone is merged afterwards: in the block of warps first, then, by the block that arrives last,
//     over blocks (a counter that the last one resets; the order of the sum is fixed).  Short items are padded to whole
//     stretches instead, so that there is nothing to merge (one token of 250, 8 heads: 9.7 us, cut evenly 13.5).
//   - A tile lies in memory in the order of the mma operand fragments (pages.cuh), so a lane copies (cp.async) and
//     reads back the very bytes it needs: no barrier, no transposition, no bank conflicts.
//   - Scores are computed transposed (m16n8k16: 16 tokens x 16 dimensions of K times 8 query rows): eight rows fill an
//     instruction, and the codes, converted to fp16 exactly, are never scaled - the magnitude of a key block is part of
//     the factor that turns a score into an exponent, that of a value block, as log2 a_v, part of the exponent.
//   - A row's sums are relative to 2^m, m a reference near the largest exponent of late (pages_attn.cuh): it is moved, and
//     the sums rescaled, when exponents leave a range around it, which one vote per pair of blocks finds; a pair costs no
//     shuffles otherwise.
// Roundings: bf16 queries become fp16 after division by a power of two of their row (11 bits are enough for 8; what
// lies 2^-14 below the row's largest loses bits, 2^-25 of the largest at most).  P = p a_v / 2^m goes into the second
// product as fp16 high part plus fp16 rest (22 bits); next to a bf16 output, which is rounded to 2^-8, the rest is left
// out: 2^-11 of each.  Either way P below 2^-14 is off by up to 2^-25, at most 2^-18 of the largest P of the pair.  The
// output is rounded once.
//
// Measured: 64 sequences of up to 4000 tokens, 8 KV heads x 4 queries of D 128 (264 MB): 68 us, 3.9 TB/s; two of 100 000
// and more, 8 x 8 (474 MB): 96 us, 4.9 TB/s; 16 sequences, 40 heads, window 1024 (169 MB): 44 us, 3.8 TB/s.  Some 6 us
// are the beginning (entries, cut, first pages: a chain of four loads), a few the merges; in between SMs differ (the same
// number of bytes takes some of them a quarter longer).  Stretches handed out at run time instead cost 8 to 30 us
// more at two long sequences: more parts to merge.
#pragma once

#include <atomic>
#include <type_traits>

#include "less_internal.cuh"
#include "pages_attn.cuh"
#include "tc_common.cuh"

namespace less {

constexpr int PS_WARPS = 6, PS_THREADS = PS_WARPS * 32;
// CTAs per SM: two (168 registers a thread, 96 KB of tiles per CTA) unless the rows' sums need more registers
__host__ __device__ constexpr int ps_ctas(int NT, int D) { return NT * D <= 128 ? 2 : 1; }
// Blocks that an item is counted as more than it has: its beginning and end take a warp as long as some blocks, and with
// sequences that end a few tokens behind what they share, an even cut of the blocks alone hands one warp dozens of items (64
// sequences of 1 to 1000 tokens of their own, 32 heads: 234 us, of which SMs are busy for 66 on average; with 6 blocks more
// each 68 us, with 3, 10 or 16 longer).
__host__ __device__ constexpr int ps_more(PaMode mode) { return mode == kAll ? 0 : 6; }
constexpr int PS_RING = 4;                     // tiles of a warp: two being worked on, two on their way
constexpr int PS_MIN_BLOCKS = 4;               // blocks a warp takes at least (one token of 250: 2 the same, 8: 9.7 -> 13.3 us)

__device__ __forceinline__ int64_t div64(int64_t a, int64_t b) {       // not negative; 32-bit where the numbers allow
  return (a | b) >> 32 ? a / b : (int64_t)((uint32_t)a / (uint32_t)b);
}

// codes are read once per call: they leave L2 first (2 to 5 % on batches larger than L2, nothing on smaller ones)
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, uint64_t policy) {
  asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "l"(policy) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t movmatrix(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

// One item: rows [row0, row0 + valid) of a (sequence, layer, head)'s tokens x group rows.
struct Item {
  int64_t begin;                // first block in the list of all blocks
  int blocks;
  int valid;                    // rows of this item
  int h, row0, tok_row, lj;
  int extra;                    // kRest: there are parts of its rows over shared blocks; kTree: rows that nobody writes, a bit each
};

struct PsShared {
  int64_t units[PS_THREADS + 1];  // blocks of the entries before a thread's
  int items[PS_THREADS + 1];      // items of the entries before a thread's
  int most[PS_WARPS];             // blocks of the longest item
  int64_t sum_u[PS_WARPS];
  int sum_i[PS_WARPS];
  PgEntry entry[PS_THREADS];      // with no more entries than threads: the entries
  Item part[PS_WARPS][2];         // the item that a warp holds a part of: begun before its stretch (0), or going on behind it
  float* where[PS_WARPS][2];      // the part: rows x D values, then (maximum, sum) of the rows; null = none
  int last[2];                    // whether this CTA merges the part-0 / part-1 item over all CTAs
};

// kTree: the rows of a warp's item, each of an entry of its own perhaps
struct PsTreeRow {
  int first;                    // the first row of the same entry
  int pos;                      // position of its token, -1 = sees nothing
  int start, count;             // the entry's blocks beside the shared ones, where they begin behind these (first rows; else none)
  int seq, len;
  RestBlocks rest;
};

// a part lies in shared or in global memory; there it may come from another CTA of this launch: past L1
__device__ __forceinline__ float2 load_part2(const float* s) {
  float2 v;
  asm volatile("ld.relaxed.gpu.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "l"(s) : "memory");
  return v;
}
__device__ __forceinline__ float4 load_part4(const float* s) {
  float4 v;
  asm volatile("ld.relaxed.gpu.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "l"(s) : "memory");
  return v;
}

// address of an item's row: rows are (token, query head of the group); `layers` of them lie between tokens
__device__ __forceinline__ int64_t row_offset(const PgParams& p, int layers, int D, const Item& it, int r) {
  const int rr = it.row0 + r, tok = rr / p.group, hd = rr - tok * p.group;
  return ((int64_t)(it.tok_row + tok) * layers + it.lj) * ((int64_t)p.heads * p.group * D) +
         ((int64_t)it.h * p.group + hd) * D;
}

// kRest: a row's N values from f (relative to 2^m, sum l) and the one or two parts over shared blocks; row: its number among
// the parts
template <int D, int N>
__device__ __forceinline__ void join_shared(const PgParams& p, const PaSharedArgs& a, int64_t row, int d0, float* f, float m, float l) {
  const int64_t rows = (int64_t)a.rows * a.nl * p.heads * p.group;
  const float2 w0 = __ldcg(a.weights + row), w1 = a.splits > 1 ? __ldcg(a.weights + rows + row) : make_float2(-INFINITY, 0.f);
  const float top = fmaxf(m, fmaxf(w0.x, w1.x));
  float x = l == 0.f ? 0.f : l * pa_ex2(m - top), x0 = w0.y == 0.f ? 0.f : w0.y * pa_ex2(w0.x - top),
        x1 = w1.y == 0.f ? 0.f : w1.y * pa_ex2(w1.x - top);
  const float sum = x + x0 + x1, inv = sum == 0.f ? 0.f : 1.f / sum;
  x *= inv;
  x0 *= inv;
  x1 *= inv;
  const float* v = a.parts + row * D + d0;
#pragma unroll
  for (int i = 0; i < N; i += 4) {
    float4 y = make_float4(f[i] * x, f[i + 1] * x, f[i + 2] * x, f[i + 3] * x);
    if (x0 != 0.f) {                                       // else its values may not have been written
      const float4 z = __ldcg(reinterpret_cast<const float4*>(v + i));
      y = make_float4(fmaf(x0, z.x, y.x), fmaf(x0, z.y, y.y), fmaf(x0, z.z, y.z), fmaf(x0, z.w, y.w));
    }
    if (x1 != 0.f) {
      const float4 z = __ldcg(reinterpret_cast<const float4*>(v + rows * D + i));
      y = make_float4(fmaf(x1, z.x, y.x), fmaf(x1, z.y, y.y), fmaf(x1, z.z, y.z), fmaf(x1, z.w, y.w));
    }
    f[i] = y.x;
    f[i + 1] = y.y;
    f[i + 2] = y.z;
    f[i + 3] = y.w;
  }
}

template <typename T, int D, int NT, bool E4M3, PaMode MODE>
__global__ void __launch_bounds__(PS_THREADS, ps_ctas(NT, D)) pages_step_kernel(PgParams p, typename PaWork<MODE>::Args a) {
  typedef PaWork<MODE> Work;
  constexpr int R = 8 * NT, MT = D / 16;
  constexpr int TILE = 16 * D, CH = TILE / 512;           // bytes of a tile; 16-byte pieces per lane
  constexpr int SLOT = R * (D + 2);
  // the rest of the probabilities matters next to an fp16 output (2^-11), not next to a bf16 one (2^-8)
  constexpr bool LO = std::is_same<T, __half>::value;
  extern __shared__ __align__(16) unsigned char ps_ring[];
  __shared__ PsShared sh;
  __shared__ PsTreeRow tree[MODE == kTree ? PS_WARPS : 1][MODE == kTree ? R : 1];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  // kRest: the kernel before it in the stream gives the parts that are joined, nothing else that is read here; what that one
  // has waited for is complete.  So it is waited for only where parts are read, and before any CTA ends.
  auto wait_parts = [] { if (MODE == kRest) pdl_wait_primary(); };
  if (MODE == kRest) pdl_launch_dependents(); else pg_wait();

  // ---- the list of blocks: a thread counts the entries of a stretch of its own, one scan orders them ----
  const int per_thread = pg_ceil(a.n, PS_THREADS);
  auto entry_items = [&](int i, const PgEntry& e, typename Work::B& b, int& tiles) -> int {
    const int64_t nr = (int64_t)e.count * p.group;
    if (nr == 0 || nr > a.max_rows || (MODE == kTree && nr < 0)) return 0;
    b = Work::blocks(a, i, e);
    tiles = (int)((nr + R - 1) / R);
    return tiles * a.nl * p.heads;
  };
  auto tree_rest = [&](int i, const PgEntry& e) -> int {  // the most blocks beside the shared ones that an item of it has
    if constexpr (MODE == kTree) return e.count > 0 ? __ldcg(a.entries + __ldcg(a.groups + 2 * i).w).w : 0;
    return 0;
  };
  int per_warp;
  int64_t pad = 0;
  {
    int64_t mu = 0;
    int mi = 0, most = 0;
    for (int i = tid * per_thread; i < min(a.n, (tid + 1) * per_thread); ++i) {
      typename Work::B b;
      int tiles;
      const PgEntry e = Work::entry(p, a, i);
      if (per_thread == 1) sh.entry[tid] = e;
      // entries overlap then, and the items of all might not be counted in 32 bits (else the host has made sure of that)
      if (MODE == kTree ? e.count < 0 : pg_descends(a.starts, i)) most = 0x7fffffff;
      const int items = entry_items(i, e, b, tiles);
      if (items) {
        const int blocks = max(1, b.count() + tree_rest(i, e));
        mu += (int64_t)items * (blocks + ps_more(MODE));
        mi += items;
        most = max(most, blocks);
      }
    }
    int64_t xu = mu;
    int xi = mi;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int64_t yu = __shfl_up_sync(0xffffffffu, xu, d);
      const int yi = __shfl_up_sync(0xffffffffu, xi, d);
      if (lane >= d) {
        xu += yu;
        xi += yi;
      }
    }
    most = __reduce_max_sync(0xffffffffu, most);
    if (lane == 31) {
      sh.sum_u[warp] = xu;
      sh.sum_i[warp] = xi;
      sh.most[warp] = most;
    }
    __syncthreads();
    for (int w = 0; w < PS_WARPS; ++w) {
      most = max(most, sh.most[w]);
      if (w < warp) {
        xu += sh.sum_u[w];
        xi += sh.sum_i[w];
      }
    }
    if (most == 0x7fffffff) {                              // pg_entry has reported it
      wait_parts();
      return;
    }
    sh.units[tid + 1] = xu;
    sh.items[tid + 1] = xi;
    if (tid == 0) {
      sh.units[0] = 0;
      sh.items[0] = 0;
    }
    __syncthreads();
    // How the list is cut: every warp gets a stretch of the same length.  Where items are short they are padded to whole
    // stretches of k warps each: then none is split, or only inside a CTA.  Times in blocks at full load, merging inside
    // a CTA costs about 2 of them, over CTAs 8.
    const int64_t workers = (int64_t)gridDim.x * PS_WARPS, items = sh.items[PS_THREADS], sum = sh.units[PS_THREADS];
    per_warp = max(PS_MIN_BLOCKS, ((int)min((int64_t)1 << 30, div64(sum + workers - 1, workers)) + 1) & ~1);
    int cost = per_warp + 8;
#pragma unroll
    for (int k = 1; k <= PS_WARPS; ++k) {
      if (PS_WARPS % k) continue;
      const int w = max(PS_MIN_BLOCKS, (pg_ceil(most, k) + 1) & ~1);
      const int64_t rounds = div64(items * k + workers - 1, workers);
      if (rounds > (k == 1 ? 64 : 1) || most > (1 << 20)) continue;
      const int c = (int)rounds * w + (k > 1 ? 2 : 0);
      if (c < cost) {
        cost = c;
        per_warp = (int)rounds * w;
        pad = (int64_t)k * w;
      }
    }
  }
  // blocks before the entries of thread j, in the list that is cut up
  auto before = [&](int j) -> int64_t { return pad ? (int64_t)sh.items[j] * pad : sh.units[j]; };
  const int64_t total = before(PS_THREADS), per_cta = (int64_t)PS_WARPS * per_warp;
  const int64_t cta_begin = (int64_t)blockIdx.x * per_cta, cta_end = min(total, cta_begin + per_cta);
  if (cta_begin >= total) {
    wait_parts();
    return;
  }
  int64_t u = min(total, cta_begin + (int64_t)warp * per_warp);
  const int64_t ue = min(total, u + per_warp);
  if (lane < 2) sh.where[warp][lane] = nullptr;
  if (tid < 2) sh.last[tid] = 0;

  const uint32_t ring = (uint32_t)__cvta_generic_to_shared(ps_ring) + warp * (PS_RING * 2 * TILE) + lane * 16;
  const uint64_t policy = l2_evict_first_policy();
  const unsigned char* ring_g = ps_ring + warp * (PS_RING * 2 * TILE) + lane * 16;
  float* slots = p.partial + (size_t)(blockIdx.x * PS_WARPS) * SLOT;            // a warp's part 0
  float* cta_slots = p.partial + (size_t)gridDim.x * PS_WARPS * SLOT;           // a CTA's two parts

  // ---- where this warp starts ----
  int ei = 0, index = 0, bo = 0;            // entry, item of the entry, block of the item
  int64_t entry_begin = 0;
  PgEntry e = {};
  typename Work::B vb = {};
  int tiles = 1, items = 0, real = 1, blocks = 1;   // blocks of an item, and with its padding
  auto next_entry = [&]() {                 // the first entry at or behind ei that has items; false = none
    for (; ei < a.n; ++ei) {
      e = per_thread == 1 ? sh.entry[ei] : Work::entry(p, a, ei);
      items = entry_items(ei, e, vb, tiles);
      if (items == 0) continue;
      real = max(1, vb.count() + tree_rest(ei, e));
      blocks = pad ? (int)pad : real + ps_more(MODE);
      return true;
    }
    return false;
  };
  if (u < ue) {
    int lo = 0, hi = PS_THREADS - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (before(mid) <= u) lo = mid; else hi = mid - 1;
    }
    ei = lo * per_thread;
    entry_begin = before(lo);
    while (next_entry() && u >= entry_begin + (int64_t)items * blocks) {
      entry_begin += (int64_t)items * blocks;
      ++ei;
    }
    if (ei >= a.n) u = ue;                  // cannot be, unless the lengths changed under the call
    index = (int)div64(u - entry_begin, blocks);
    bo = (int)((u - entry_begin) - (int64_t)index * blocks);
  }

  while (u < ue) {
    // ---- the item ----
    Item it;
    it.begin = entry_begin + (int64_t)index * blocks;
    it.blocks = blocks;
    it.row0 = (index % tiles) * R;
    it.h = (index / tiles) % p.heads;
    it.lj = index / tiles / p.heads;
    it.tok_row = e.row0;
    it.valid = min(R, e.count * p.group - it.row0);
    if constexpr (MODE == kRest) {
      const int4 of = __ldcg(a.entries + ei);
      it.extra = of.x + of.z - of.y > 0;
    }
    const int first = bo, end = (int)min((int64_t)blocks, bo + (ue - u));
    int last = vb.count() > 0 ? min(end, real) : first;             // what of it has tokens
    if constexpr (MODE == kTree) {
      // whose the rows are; the blocks that their entries see beside the shared ones follow those
      const int4 ge = __ldcg(a.groups + 2 * ei), gb = __ldcg(a.groups + 2 * ei + 1);
      const int trow = e.row0 + (it.row0 + min(lane, it.valid - 1)) / p.group;
      int who = ge.w + trow - e.row0;
      if (a.starts) {
        who = ge.w;
        for (int c = ge.w; c < gb.w; c += 32) {
          const int stop = c + lane < gb.w ? __ldg(a.starts + c + lane + 1) : 0x7fffffff;
#pragma unroll
          for (int k = 0; k < R; ++k) {
            const int n = __popc(__ballot_sync(0xffffffffu, stop <= __shfl_sync(0xffffffffu, trow, k)));
            if (lane == k) who += n;
          }
        }
      }
      const bool mine = lane < it.valid && who < gb.w;
      PgEntry en = {0, 0, 0, 0};
      if (mine) en = pg_entry(p, a.seqs, a.starts, a.rows, who);
      const int before = __shfl_up_sync(0xffffffffu, who, 1);
      const bool head = mine && (lane == 0 || before != who);
      const uint32_t heads = __ballot_sync(0xffffffffu, head);
      it.extra = (int)__ballot_sync(0xffffffffu, lane < it.valid && en.count == 0);
      const RestBlocks rest = rest_blocks(visible_blocks(a, en.len, en.count), gb);
      const int n = head && en.count ? rest.count() : 0;
      int upto = n;
#pragma unroll
      for (int d = 1; d < R; d <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, upto, d);
        if (lane >= d) upto += y;
      }
      __syncwarp();                                        // the item before has been read
      if (lane < R)
        tree[warp][lane] = {31 - __clz((int)(heads & (2u << lane) - 1u)), mine && en.count ? en.len - en.count + trow - en.row0 : -1,
                            upto - n, n, en.seq, en.len, rest};
      last = min(end, vb.count() + __shfl_sync(0xffffffffu, upto, R - 1));
      __syncwarp();
    }
    const int layer = a.layer0 + it.lj;

    // ---- pages and magnitudes: lane i knows the tile of block `batch + i` and, one batch ahead, `batch + 32 + i` ----
    const uint8_t* head_codes = p.codes + (((size_t)layer * p.pages) * p.heads + it.h) * ((size_t)2 * p.pt * D);
    const float* head_mags = p.amax + (((size_t)layer * p.pages) * p.heads + it.h) * ((size_t)2 * (p.pt / kPageBlock));
    struct Tile {
      const uint8_t* codes;       // null = none
      float ak, lav;              // magnitude of the keys, log2 of the values'
      // kTree: position of the first token, the entry's length, the first row that sees it (-1: all do)
      int j0, len, who;
    };
    auto lookup = [&](int b) {
      Tile tl = {nullptr, 0.f, kNoValues, 0, 0, -1};
      if (b + lane < last) {
        int seq = e.seq, block;
        if (MODE == kTree) {
          const int u = b + lane, behind = u - vb.count();
          if (behind < 0) {
            block = vb.at(u);
            tl.len = 0x7fffffff;
          } else {
            for (int k = 0; k < it.valid; ++k)
              if (tree[warp][k].count && behind >= tree[warp][k].start) tl.who = k;
            const PsTreeRow& row = tree[warp][tl.who];
            block = row.rest.at(behind - row.start);
            seq = row.seq;
            tl.len = row.len;
          }
          tl.j0 = block * kPageBlock;
        } else {
          block = vb.at(b + lane);
        }
        const int tok = block * kPageBlock, inner = (tok & (p.pt - 1)) / kPageBlock;
        const int page = pg_page(p, seq, tok >> p.pt_shift);
        if (page >= 0) {
          const size_t slab = (size_t)page * p.heads * 2;
          tl.codes = head_codes + slab * ((size_t)p.pt * D) + (size_t)inner * TILE;
          const float* mg = head_mags + slab * (p.pt / kPageBlock) + inner;
          tl.ak = __ldcg(mg);
          const float av = __ldcg(mg + p.pt / kPageBlock);
          if (av >= kLeastValue) tl.lav = log2f(av);
        }
      }
      return tl;
    };
    Tile cur = lookup(first), nxt = {nullptr, 0.f, kNoValues, 0, 0, -1};
    const size_t to_values = (size_t)p.pt * D;
    // the tiles of blocks b and b + 1 on their way to ring slots `slot` and `slot + 1`
    auto fetch = [&](const Tile& tl, int at, int slot) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const uint8_t* codes = reinterpret_cast<const uint8_t*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(tl.codes), at + k));
        if (codes) {
          codes += lane * 16;
          const uint32_t dst = ring + (slot + k) * (2 * TILE);
#pragma unroll
          for (int i = 0; i < CH; ++i) cp_async16(dst + i * 512, codes + i * 512, policy);
          codes += to_values;
#pragma unroll
          for (int i = 0; i < CH; ++i) cp_async16(dst + TILE + i * 512, codes + i * 512, policy);
        }
      }
      cp_async_commit();
    };
    fetch(cur, 0, 0);

    // ---- its queries: operand fragments, the score factor and the position of the rows of this lane ----
    uint32_t qf[NT][D / 8];
    float crow[NT][2];
    int pos[NT][2], owner[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int r = nt * 8 + g;
      uint4 w[D / 32];
#pragma unroll
      for (int i = 0; i < D / 32; ++i) w[i] = make_uint4(0, 0, 0, 0);
      if (r < it.valid) {
        const int rr = it.row0 + r, tok = rr / p.group, hd = rr - tok * p.group;
        const T* src = reinterpret_cast<const T*>(a.q) + (int64_t)(e.row0 + tok) * a.q_stride +
                       ((int64_t)it.lj * p.heads + it.h) * p.group * D + hd * D + t * (D / 4);
#pragma unroll
        for (int i = 0; i < D / 32; ++i) w[i] = __ldcg(reinterpret_cast<const uint4*>(src) + i);
      }
      float up = 1.f;
      if (!std::is_same<T, __half>::value) {
        const __nv_bfloat162* y = reinterpret_cast<const __nv_bfloat162*>(w);
        float most = 0.f;
#pragma unroll
        for (int i = 0; i < D / 8; ++i) {
          const float2 f = __bfloat1622float2(y[i]);
          most = fmaxf(most, fmaxf(fabsf(f.x), fabsf(f.y)));
        }
        most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
        most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
        // 2^e <= most < 2^(e + 1): the row divided by 2^e
        const int ex = min(max((int)(__float_as_uint(most) >> 23), 1), 253);
        up = __uint_as_float((uint32_t)ex << 23);
        const float down = __uint_as_float((uint32_t)(254 - ex) << 23);
#pragma unroll
        for (int i = 0; i < D / 8; ++i) {
          const float2 f = __bfloat1622float2(y[i]);
          qf[nt][i] = pack2(f.x * down, f.y * down);
        }
      } else {
#pragma unroll
        for (int i = 0; i < D / 8; ++i) qf[nt][i] = reinterpret_cast<const uint32_t*>(w)[i];
      }
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int rc = nt * 8 + 2 * t + c;
        crow[nt][c] = a.scale * 1.4426950408889634f / pg_top<E4M3>() * __shfl_sync(0xffffffffu, up, (2 * t + c) * 4);
        pos[nt][c] = MODE == kTree ? tree[warp][rc].pos : rc < it.valid ? e.len - e.count + (it.row0 + rc) / p.group : -1;
        if (MODE == kTree) owner[nt][c] = tree[warp][rc].first;
      }
    }
    const int first_pos = e.len - e.count + it.row0 / p.group, last_pos = e.len - e.count + (it.row0 + it.valid - 1) / p.group;
    const bool all_rows = it.valid == R && (MODE != kTree || it.extra == 0);

    float o[NT][MT][4], m[NT][2], l[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[nt][mt][i] = 0.f;
      m[nt][0] = m[nt][1] = 0.f;
      l[nt][0] = l[nt][1] = 0.f;
    }

    int low = 0;                                           // how far the references are below their highest: a byte per row of the lane
    int slot = 0;
    for (int b = first; b < last; b += 2) {
      const int at = (b - first) & 31;                     // lane of block b
      if (at == 0) {
        if (b != first) cur = nxt;
        nxt = b + 32 < last ? lookup(b + 32) : Tile{nullptr, 0.f, kNoValues, 0, 0, -1};
      }
      fetch(at + 2 < 32 ? cur : nxt, (at + 2) & 31, slot ^ 2);
      cp_async_wait<1>();
      float ak[2], lav[2];
      bool here[2];
      int j0[2], len[2], who[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        ak[k] = __shfl_sync(0xffffffffu, cur.ak, at + k);
        lav[k] = __shfl_sync(0xffffffffu, cur.lav, at + k);
        here[k] = __shfl_sync(0xffffffffu, (int)(cur.codes != nullptr), at + k);
        if (MODE == kTree) {
          j0[k] = __shfl_sync(0xffffffffu, cur.j0, at + k);
          len[k] = __shfl_sync(0xffffffffu, cur.len, at + k);
          who[k] = __shfl_sync(0xffffffffu, cur.who, at + k);
        } else {
          j0[k] = vb.at(b + k) * kPageBlock;
          len[k] = e.len;
          who[k] = -1;
        }
      }
      const unsigned char* tile = ring_g + slot * (2 * TILE);
      slot ^= 2;

      // ---- scores: 2 x 16 tokens x 8 NT rows ----
      float s[2][NT][4];
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) s[k][nt][0] = s[k][nt][1] = s[k][nt][2] = s[k][nt][3] = 0.f;
#pragma unroll
      for (int half = 0; half < D / 64; ++half) {
        uint4 kk[2][2];
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int j = 0; j < 2; ++j)
            kk[k][j] = *reinterpret_cast<const uint4*>(tile + k * (2 * TILE) + (j * (D / 64) + half) * 512);
#pragma unroll
        for (int w = 0; w < 4; ++w)
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const uint32_t w0 = w == 0 ? kk[k][0].x : w == 1 ? kk[k][0].y : w == 2 ? kk[k][0].z : kk[k][0].w;
            const uint32_t w1 = w == 0 ? kk[k][1].x : w == 1 ? kk[k][1].y : w == 2 ? kk[k][1].z : kk[k][1].w;
            uint32_t a0, a1, a2, a3;
            pg_unpack4<E4M3>(w0, a0, a2);
            pg_unpack4<E4M3>(w1, a1, a3);
            const int ks = half * 4 + w;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) mma16816(s[k][nt], a0, a1, a2, a3, qf[nt][2 * ks], qf[nt][2 * ks + 1]);
          }
      }
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const bool whole = MODE == kTree ? all_rows && here[k] && who[k] < 0 :
                           all_rows && here[k] && j0[k] + kPageBlock - 1 <= first_pos &&
                           (!a.window || j0[k] > last_pos - a.window || j0[k] + kPageBlock <= a.sinks);
        // this lane's tokens: accumulator rows g and g + 8
        const int ja = j0[k] + 4 * (g >> 1) + (g & 1), jb = ja + 2;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const uint64_t factor = f32x2_mul(f32x2_pack(ak[k], ak[k]), f32x2_pack(crow[nt][0], crow[nt][1]));
          const uint64_t offset = f32x2_pack(lav[k] - m[nt][0], lav[k] - m[nt][1]);
#pragma unroll
          for (int i = 0; i < 4; i += 2)
            f32x2_unpack(f32x2_fma(f32x2_pack(s[k][nt][i], s[k][nt][i + 1]), factor, offset), s[k][nt][i], s[k][nt][i + 1]);
          if (!whole) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int j = i < 2 ? ja : jb, at_row = pos[nt][i & 1];
              if (!here[k] || j > at_row || (a.window && j <= at_row - a.window && j >= a.sinks)) s[k][nt][i] = -INFINITY;
              if (MODE == kTree && who[k] >= 0 && who[k] != owner[nt][i & 1]) s[k][nt][i] = -INFINITY;
            }
          }
        }
      }
      // the reference is set by the first pair, and follows: a row that it has left has a lane whose own keys lie outside
      bool away = b == first;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const float x = fmaxf(fmaxf(s[0][nt][c], s[0][nt][2 + c]), fmaxf(s[1][nt][c], s[1][nt][2 + c]));
          away |= x > kRefMost || (x < kRefLeast && x > -INFINITY);
        }
      if (__any_sync(0xffffffffu, away)) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            float x = fmaxf(fmaxf(s[0][nt][c], s[0][nt][2 + c]), fmaxf(s[1][nt][c], s[1][nt][2 + c]));
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, d));
            float d = 0.f;                                   // what the reference moves by
            if (x > kRefMost || (x > -INFINITY && (x < kRefBack || b == first)))
              d = x - (x > kRefMost && b != first ? kRefUp : kRefNew);
            if (b != first && __any_sync(0xffffffffu, d != 0.f)) {
              float big = fmaxf(l[nt][c], fabsf(o[nt][0][c]));
#pragma unroll
              for (int i = 4; i < 32; i <<= 1) big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, i));
              if (big > 0.f) {                               // down by so much that no sum passes 2^104
                const int sh = 16 * nt + 8 * c, is = low >> sh & 255;
                d = fmaxf(d, (float)max(is - 60, min(0, (int)(__float_as_uint(big) >> 23) - 127 - 90)));
                low = (low & ~(255 << sh)) | max(0, is - __float2int_rd(d)) << sh;
              }
              d = (m[nt][c] + d) - m[nt][c];                 // as the reference is rounded
              const float f = big > 0.f ? pa_ex2(-d) : 1.f;
              l[nt][c] = pa_scaled(l[nt][c], -d);
#pragma unroll
              for (int mt = 0; mt < MT; ++mt) {
                o[nt][mt][c] *= f;
                o[nt][mt][2 + c] *= f;
              }
            }
            m[nt][c] += d;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              s[k][nt][c] -= d;
              s[k][nt][2 + c] -= d;
            }
          }
      }
      // ---- probabilities times the value magnitude: second operand of the product with the values ----
      uint32_t ph[2][NT][2], pl[2][NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const float back = -kSumBits - lav[k];
          const uint32_t some = lav[k] == kNoValues ? 0u : 0xffffffffu;
          float x[4];
#pragma unroll
          for (int i = 0; i < 4; i += 2) {
            float p0, p1;
            f32x2_unpack(f32x2_add(f32x2_pack(s[k][nt][i], s[k][nt][i + 1]), f32x2_pack(back, back)), p0, p1);
            x[i] = pa_ex2(s[k][nt][i]);
            x[i + 1] = pa_ex2(s[k][nt][i + 1]);
            f32x2_unpack(f32x2_add(f32x2_pack(l[nt][0], l[nt][1]), f32x2_pack(pa_ex2(p0), pa_ex2(p1))), l[nt][0], l[nt][1]);
          }
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const __half2 hi = __floats2half2_rn(x[2 * i], x[2 * i + 1]);
            ph[k][nt][i] = movmatrix(*reinterpret_cast<const uint32_t*>(&hi) & some);
            if (LO) {
              const float2 high = __half22float2(hi);
              pl[k][nt][i] = movmatrix(pack2(x[2 * i] - high.x, x[2 * i + 1] - high.y) & some);
            }
          }
        }
      }
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        // tokens behind the end may hold any byte, a slot without a tile or values of magnitude 0 too; a NaN code would
        // survive its zero probability
        uint32_t keep = 0xffffffffu;
        if (E4M3 && (!here[k] || lav[k] == kNoValues || j0[k] > len[k] - kPageBlock)) {
          const int left = here[k] && lav[k] != kNoValues ? len[k] - (j0[k] + 4 * t) : 0;
          keep = left <= 0 ? 0u : (left >= 4 ? keep : keep >> (8 * (4 - left)));
        }
#pragma unroll
        for (int i = 0; i < CH; ++i) {
          const uint4 v4 = *reinterpret_cast<const uint4*>(tile + k * (2 * TILE) + TILE + i * 512);
          uint32_t w[4] = {v4.x, v4.y, v4.z, v4.w};
          if (E4M3) {
#pragma unroll
            for (int dd = 0; dd < 4; ++dd) w[dd] &= keep;
          }
#pragma unroll
          for (int dd = 0; dd < 4; dd += 2) {
            uint32_t a0, a1, a2, a3;
            pg_unpack4<E4M3>(w[dd], a0, a2);
            pg_unpack4<E4M3>(w[dd + 1], a1, a3);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              mma16816(o[nt][2 * i + dd / 2], a0, a1, a2, a3, ph[k][nt][0], ph[k][nt][1]);
              if (LO) mma16816(o[nt][2 * i + dd / 2], a0, a1, a2, a3, pl[k][nt][0], pl[k][nt][1]);
            }
          }
        }
      }
    }
    cp_async_wait<0>();

    // ---- the item's rows, or a part of them ----
    const bool complete = first == 0 && end == blocks;
    const int which = first == 0 ? 1 : 0;
    // the ring is free again with the last item of a warp's stretch
    const bool done = u + (end - first) == ue;
    float* slot_out = SLOT * 4 <= PS_RING * 2 * TILE && done ? reinterpret_cast<float*>(ps_ring + warp * (PS_RING * 2 * TILE))
                                                             : slots + (size_t)warp * SLOT;
    __syncwarp();
    if (complete) wait_parts();
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        float sum = l[nt][c];
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        const int rc = nt * 8 + 2 * t + c;
        if (rc >= it.valid || (MODE == kTree && it.extra >> rc & 1)) continue;
        const float unit = (sum > 0.f ? 1.f / sum : 0.f) * (0x1p-8f / pg_top<E4M3>());
        float f[D / 8];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          f[2 * mt] = o[nt][mt][c] * unit;
          f[2 * mt + 1] = o[nt][mt][2 + c] * unit;
        }
        if (sum != sum) {                                    // a query that is not finite
#pragma unroll
          for (int i = 0; i < D / 8; ++i) f[i] = sum;
        }
        if (complete) {
          int layers = a.nl;
          if constexpr (MODE == kRest) {
            layers = a.out_layers;
            if (it.extra) {
              const float2 ml = pa_share(m[nt][c], sum);
              join_shared<D, D / 8>(p, a, row_offset(p, a.nl, D, it, rc) / D, g * (D / 8), f, ml.x, ml.y);
            }
          }
          T* dst = reinterpret_cast<T*>(a.out) + row_offset(p, layers, D, it, rc) + g * (D / 8);
#pragma unroll
          for (int i = 0; i < D / 8; i += 8) store8<T>(dst + i, f + i);
        } else {
          float* dst = slot_out + rc * D + g * (D / 8);
#pragma unroll
          for (int i = 0; i < D / 8; i += 4) *reinterpret_cast<float4*>(dst + i) = make_float4(f[i], f[i + 1], f[i + 2], f[i + 3]);
          if (g == 0) {
            *reinterpret_cast<float2*>(slot_out + R * D + 2 * rc) = pa_share(m[nt][c], sum);
          }
        }
      }
    if (!complete && lane == 0) {
      sh.part[warp][which] = it;
      sh.where[warp][which] = slot_out;
    }

    // ---- next ----
    u += end - first;
    bo = 0;
    if (++index == items && u < ue) {
      index = 0;
      entry_begin += (int64_t)items * blocks;
      ++ei;
      if (!next_entry()) break;             // as above
    }
  }
  wait_parts();
  __syncthreads();

  // ---- merge: a warp takes a row, lanes own four dimensions each (with D 64 the upper half repeats the lower) ----
  auto merge_row = [&](auto part_of, int parts, int r, float4& f, float& mm, float& ll) {
    auto load2 = [&](const float* s) { return load_part2(s + R * D + 2 * r); };
    auto load4 = [&](const float* s) { return load_part4(s + r * D + (lane % (D / 4)) * 4); };

    constexpr int N = 16;                               // parts on their way at once
    float4 v[N];
    auto ask = [&](int base) {
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (base + i < parts) v[i] = load4(part_of(base + i));
    };
    // the weights of N parts at a time are lanes'; the values are asked for before the maximum is known
    float2 ml = make_float2(-INFINITY, 0.f);
    if (lane < parts) ml = load2(part_of(lane));
    ask(0);
    mm = ml.x;
    for (int i = lane + 32; i < parts; i += 32) mm = fmaxf(mm, load2(part_of(i)).x);
#pragma unroll
    for (int d = 16; d; d >>= 1) mm = fmaxf(mm, __shfl_xor_sync(0xffffffffu, mm, d));
    f = make_float4(0.f, 0.f, 0.f, 0.f);
    ll = 0.f;
    for (int base = 0; base < parts; base += N) {
      if (base) {
        ml = make_float2(-INFINITY, 0.f);
        if (lane < N && base + lane < parts) ml = load2(part_of(base + lane));
        ask(base);
      }
      const float w = ml.y == 0.f ? 0.f : ml.y * pa_ex2(ml.x - mm);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        if (base + i >= parts) break;
        const float wi = __shfl_sync(0xffffffffu, w, i);
        ll += wi;
        f.x = fmaf(wi, v[i].x, f.x);
        f.y = fmaf(wi, v[i].y, f.y);
        f.z = fmaf(wi, v[i].z, f.z);
        f.w = fmaf(wi, v[i].w, f.w);
      }
    }
    const float inv = ll == 0.f ? 0.f : 1.f / ll;
    f = make_float4(f.x * inv, f.y * inv, f.z * inv, f.w * inv);
  };
  auto row_done = [&](const Item& it, int r, float4 f, float mm, float ll) {
    int layers = a.nl;
    if constexpr (MODE == kRest) {
      layers = a.out_layers;
      if (it.extra) {
        float v[4] = {f.x, f.y, f.z, f.w};
        join_shared<D, 4>(p, a, row_offset(p, a.nl, D, it, r) / D, lane * 4, v, mm, ll);
        f = make_float4(v[0], v[1], v[2], v[3]);
      }
    }
    store4(reinterpret_cast<T*>(a.out) + row_offset(p, layers, D, it, r) + lane * 4, f);
  };
  // Inside the CTA: the items that go on behind one of its warps (part 1), or begin before the first (part 0 of warp 0),
  // all rows dealt out to the warps in turn
  bool outside = false;
  int turn = 0;
  for (int k = -1; k < PS_WARPS; ++k) {
    const int w0 = max(k, 0), wh = k < 0 ? 0 : 1;
    if (!sh.where[w0][wh]) continue;
    const Item it = sh.part[w0][wh];
    const int64_t end = it.begin + it.blocks;
    const int wl = (int)div64(min(end, cta_end) - 1 - cta_begin, per_warp);
    const bool inside = it.begin >= cta_begin && end <= cta_end;
    outside |= !inside;
    float* mine = cta_slots + (size_t)(2 * blockIdx.x + wh) * SLOT;
    auto part_of = [&](int i) { return (const float*)sh.where[w0 + i][i == 0 ? wh : 0]; };
    for (int r = 0; r < it.valid; ++r, ++turn) {
      if (turn % PS_WARPS != warp || (MODE == kTree && it.extra >> r & 1)) continue;
      float4 f;
      float mm, ll;
      merge_row(part_of, wl - w0 + 1, r, f, mm, ll);
      if (lane < D / 4) {
        if (inside) {
          row_done(it, r, f, mm, ll);
        } else {
          *reinterpret_cast<float4*>(mine + r * D + lane * 4) = f;
          if (lane == 0) *reinterpret_cast<float2*>(mine + R * D + 2 * r) = make_float2(mm, ll);
        }
      }
    }
  }
  if (!outside) return;                                      // the same for all threads
  __threadfence();
  __syncthreads();
  // Over the CTAs: the last one to arrive does it
  if (tid < 2) {
    // the item that began before this CTA, and the one that goes on behind it
    int w0 = tid == 0 ? 0 : PS_WARPS - 1;
    if (tid == 1)
      while (w0 >= 0 && !sh.where[w0][1]) --w0;
    if (w0 >= 0 && sh.where[w0][tid]) {
      const Item it = sh.part[w0][tid];
      const int64_t end = it.begin + it.blocks;
      if (it.begin < cta_begin || end > cta_end) {
        const int c0 = (int)div64(it.begin, per_cta), c1 = (int)div64(end - 1, per_cta);
        if (atomicAdd(p.counters + c0, 1) == c1 - c0) {
          p.counters[c0] = 0;
          __threadfence();
          sh.last[tid] = w0 + 1;
        }
      }
    }
  }
  __syncthreads();
  for (int which = 0; which < 2; ++which) {
    if (!sh.last[which]) continue;
    const Item it = sh.part[sh.last[which] - 1][which];
    const int c0 = (int)div64(it.begin, per_cta), c1 = (int)div64(it.begin + it.blocks - 1, per_cta);
    auto part_of = [&](int i) { return cta_slots + (size_t)(2 * (c0 + i) + (i == 0 ? 1 : 0)) * SLOT; };
    for (int r = warp; r < it.valid; r += PS_WARPS) {
      if (MODE == kTree && it.extra >> r & 1) continue;
      float4 f;
      float mm, ll;
      merge_row(part_of, c1 - c0 + 1, r, f, mm, ll);
      if (lane < D / 4) row_done(it, r, f, mm, ll);
    }
  }
}

// room: bytes at p.partial
template <typename T, int D, int NT, bool E4M3, PaMode MODE>
inline int launch_step(const PgParams& p, const typename PaWork<MODE>::Args& a, size_t room, int counters, cudaStream_t s) {
  constexpr size_t smem = (size_t)PS_WARPS * PS_RING * 2 * 16 * D;
  static std::atomic<unsigned long long> done{0};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return fail_cuda("cudaGetDevice");
  if (dev >= 64 || !(done.load(std::memory_order_relaxed) >> dev & 1)) {
    if (cudaFuncSetAttribute(pages_step_kernel<T, D, NT, E4M3, MODE>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             (int)smem) != cudaSuccess)
      return fail_cuda("shared memory opt-in of pages_step_kernel");
    if (dev < 64) done.fetch_or(1ull << dev, std::memory_order_relaxed);
  }
  // a part of each warp, and two of the CTA; a counter per CTA
  constexpr size_t cta_bytes = (size_t)(PS_WARPS + 2) * 8 * NT * (D + 2) * 4;
  int grid = ps_ctas(NT, D) * pg_sms();
  const int most = (int)(room / cta_bytes);
  if (grid > most) grid = most;
  if (grid > counters) grid = counters;
  return pg_launch("pages_step_kernel", pages_step_kernel<T, D, NT, E4M3, MODE>, dim3(grid), PS_THREADS, smem, s, p, a);
}

template <typename T, bool E4M3, PaMode MODE>
inline int launch_step_dim(const PgParams& p, const typename PaWork<MODE>::Args& a, int dim, int rows, size_t room, int counters, cudaStream_t s) {
  if (dim == 128)
    return rows > 8 ? launch_step<T, 128, 2, E4M3, MODE>(p, a, room, counters, s) : launch_step<T, 128, 1, E4M3, MODE>(p, a, room, counters, s);
  return rows > 8 ? launch_step<T, 64, 2, E4M3, MODE>(p, a, room, counters, s) : launch_step<T, 64, 1, E4M3, MODE>(p, a, room, counters, s);
}

// rows: the most of an entry, as far as the host knows
template <PaMode MODE>
inline int launch_pages_step(const PgParams& p, const typename PaWork<MODE>::Args& a, int dim, uint32_t flags, int rows, size_t room, int counters, cudaStream_t s) {
  const bool e4m3 = flags & LESS_PAGES_E4M3;
  if (flags & LESS_PAGES_BF16)
    return e4m3 ? launch_step_dim<__nv_bfloat16, true, MODE>(p, a, dim, rows, room, counters, s)
                : launch_step_dim<__nv_bfloat16, false, MODE>(p, a, dim, rows, room, counters, s);
  return e4m3 ? launch_step_dim<__half, true, MODE>(p, a, dim, rows, room, counters, s)
              : launch_step_dim<__half, false, MODE>(p, a, dim, rows, room, counters, s);
}

}  // namespace less
