// Attention over the paged 8-bit cache for groups of sequences that share their first pages (beams of one text, samples,
// conversations behind one instruction): what ordinary attention gives, with the shared pages read once for a group.
//
//   o = (l_s o_s 2^(m_s - m) + l_r o_r 2^(m_r - m)) / (l_s 2^(m_s - m) + l_r 2^(m_r - m))
//
// with (m, l, o) reference, sum and quotient of a softmax over the shared blocks (s) and over the rest (r): the two halves
// are the kernels of ordinary attention, once with a group as one entry, whose rows are the tokens of all its sequences, once
// with the sequences as entries and the other blocks.  The second joins them where it would have written its result.
// Groups of few rows (tokens x query heads of a KV head) take one pass instead: a tile of 8 or 16 rows goes over the shared blocks
// and then over the rest of the entries that its rows are of, each masked for the other rows (pages_tree.cu).
// The second half waits for the first only where it joins: it runs beside the kernel that joins parts (the 16 sequences below: 124 ->
// 114 us).
// Bound: the halves are ordinary attention's kernels, see there.  16 sequences over one text of 100 003 tokens (8 KV heads x 8,
// 212 MB): 114 us; one after the other the look at the tables takes 12, the first half 96, the joining of its parts 10, the
// second half 20.  Ordinary attention: 385 to 457.  64 sequences behind 4096 tokens in common, 32 heads: 97 us (ordinary 344 to
// 364).
// Of more than 32 rows a group, probabilities over the shared blocks are rounded to fp16 once (11 bits), as the many-token kernel
// does; the rests, and groups in one pass, keep 22 bits next to an fp16 output, as ordinary attention of few tokens does.  (The
// 64 sequences below: the mean error against 64 bits is 2.15e-4 instead of 2.07e-4.)
// What a group shares is found on the device: the leading pages that the tables of all its sequences have in common, of
// these the blocks that all its tokens see (a window moves with a sequence's end).  So a group is only a hint.
#include "pages_step.cuh"

namespace less {

constexpr int PX_THREADS = 1024, PX_PER = 8;              // table entries of a lane on their way

// One CTA per group.  A list of groups that is not [0 .. n] ascending is reported; then all entries are one group that shares
// nothing.
constexpr int PX_TILES = 1024;                            // tiles whose blocks are counted one by one
__global__ void __launch_bounds__(PX_THREADS) pages_common_kernel(PgParams p, PaSharedArgs a, const int32_t* groups, int ngroups) {
  __shared__ int common, least_seen, most_len, least_wb, some, lead, refused, descends, most_rest;
  __shared__ unsigned long long sum_rest;
  __shared__ int tile_rest[PX_TILES];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = blockIdx.x;
  int4* entries = const_cast<int4*>(a.entries);
  int4* of = const_cast<int4*>(a.groups);
  pg_wait();
  tile_rest[tid] = 0;
  if (tid == 0) {
    common = least_seen = least_wb = 0x7fffffff;
    most_len = some = refused = descends = most_rest = 0;
    sum_rest = 0;
    lead = -1;
  }
  const int g0 = __ldg(groups + g), g1 = __ldg(groups + g + 1);
  bool bad = false;
  for (int i = tid; i < ngroups; i += PX_THREADS) {
    const int b = __ldg(groups + i), e = __ldg(groups + i + 1);
    bad |= b < 0 || e < b || e > a.n || (i == 0 && b != 0) || (i == ngroups - 1 && e != a.n);
  }
  bad = __syncthreads_or(bad);
  if (bad && tid == 0) pg_status(p.status, kPagesBounds, 50);
  const int e0 = !bad ? g0 : g ? a.n : 0, e1 = bad ? a.n : g1;
  PgEntry mine = {0, 0, 0, 0};                            // the first of the thread's entries: looked up once
  for (int i = e0 + tid; i < e1; i += PX_THREADS) {
    const PgEntry e = pg_entry(p, a.seqs, a.starts, a.rows, i);
    if (i == e0 + tid) mine = e;
    const int rows = a.starts ? __ldg(a.starts + i + 1) - __ldg(a.starts + i) : 1;
    if (rows < 0) descends = 1;
    if (rows != e.count || e.len < e.count) refused = 1;   // not to be trusted: nobody of the group shares
    if (e.count == 0) continue;
    atomicAdd(&some, 1);
    atomicMax(&lead, i);
    atomicMin(&least_seen, e.len - e.count + 1);
    atomicMax(&most_len, e.len);
    if (a.window) atomicMin(&least_wb, max(0, e.len - e.count - a.window + 1) / kPageBlock);
  }
  __syncthreads();
  int4 blocks = make_int4(0, 0, 0, 0);
  int seq = 0;
  if (!bad && !refused && some > 1) {
    const int seen = least_seen / kPageBlock;             // blocks that the first token of every entry sees
    seq = __ldg(a.seqs + lead);
    const int pages = pg_ceil(seen * kPageBlock, p.pt);
    const int32_t* first = p.table + (size_t)seq * p.seq_pages;
    // a warp per stretch of an entry's table
    const int cuts = pg_ceil(pages, 32 * PX_PER);
    for (int64_t u = warp; u < (int64_t)(e1 - e0) * cuts; u += PX_THREADS / 32) {
      const int i = e0 + (int)(u / cuts), o = (int)(u % cuts) * 32 * PX_PER;
      if (a.starts && __ldg(a.starts + i + 1) == __ldg(a.starts + i)) continue;
      const int32_t* row = p.table + (size_t)__ldg(a.seqs + i) * p.seq_pages;
      if (row == first) continue;
      int x[PX_PER], y[PX_PER];
#pragma unroll
      for (int k = 0; k < PX_PER; ++k) {
        const int at = o + 32 * k + lane;
        x[k] = at < pages ? __ldcg(row + at) : 0;
        y[k] = at < pages ? __ldcg(first + at) : 0;
      }
      int at = 0x7fffffff;
#pragma unroll
      for (int k = PX_PER - 1; k >= 0; --k)
        if (x[k] != y[k]) at = o + 32 * k + lane;
      at = __reduce_min_sync(0xffffffffu, at);
      if (at != 0x7fffffff && lane == 0) atomicMin(&common, at);
    }
    __syncthreads();
    blocks.z = min(seen, (int)min((int64_t)common * (p.pt / kPageBlock), (int64_t)1 << 28));
    if (a.window) {
      blocks.y = min(blocks.z, pg_ceil(max(0, most_len - a.window), kPageBlock));
      blocks.x = min(min(a.sinks / kPageBlock, least_wb), blocks.y);
    }
    if (blocks.x + blocks.z - blocks.y <= 0) blocks = make_int4(0, 0, 0, 0);
  }
  const int row0 = e0 < a.n ? (a.starts ? min(max(__ldg(a.starts + e0), 0), a.rows) : e0) : a.rows;
  const int end = a.starts ? min(max(__ldg(a.starts + e1), row0), a.rows) : max(e1, row0);
  if (a.tile) {                                            // the most blocks beside the shared ones that the rows of a tile have
    const int64_t tiles = ((int64_t)(end - row0) * p.group + a.tile - 1) / a.tile;
    for (int i = e0 + tid; i < e1; i += PX_THREADS) {
      const PgEntry e = i == e0 + tid ? mine : pg_entry(p, a.seqs, a.starts, a.rows, i);
      if (e.count == 0) continue;
      const int rest = rest_blocks(visible_blocks(a, e.len, e.count), blocks).count();
      atomicMax(&most_rest, rest);
      atomicAdd(&sum_rest, (unsigned long long)rest);
      if (tiles <= PX_TILES && !descends) {
        const int from = (e.row0 - row0) * p.group;          // below PX_TILES * a.tile
        for (int k = from / a.tile; k <= (from + e.count * p.group - 1) / a.tile; ++k) atomicAdd(&tile_rest[k], rest);
      }
    }
    __syncthreads();
    int most = tid < tiles ? tile_rest[tid] : 0;
    if (tiles > PX_TILES || descends) most = (int)min((unsigned long long)a.tile * most_rest, sum_rest);
    most = __reduce_max_sync(0xffffffffu, most);
    __syncthreads();                                         // most_rest has been read
    if (tid == 0) most_rest = 0;
    __syncthreads();
    if (lane == 0) atomicMax(&most_rest, most);
    __syncthreads();
    blocks.w = most_rest;
  }
  for (int i = e0 + tid; i < e1; i += PX_THREADS) entries[i] = blocks;
  if (tid == 0) {
    of[2 * g] = make_int4(seq, row0, descends ? -1 : end - row0, e0);
    of[2 * g + 1] = make_int4(blocks.x, blocks.y, blocks.z, e1);
  }
}

// Joins the parts of a row into the first: a warp per row, all loads of eight parts on their way at once.  (Rows that share
// nothing have no parts; what becomes of what lies there nobody reads.)
template <int D>
__global__ void __launch_bounds__(256) pages_parts_kernel(PgParams p, PaSharedArgs a, int parts) {
  constexpr int LANES = D / 4, N = 8;
  pg_wait();
  const int lane = threadIdx.x % LANES;
  const int64_t rows = (int64_t)a.rows * a.nl * p.heads * p.group, row = ((int64_t)blockIdx.x * 256 + threadIdx.x) / LANES;
  if (row >= rows) return;
  float m = -INFINITY, sum = 0.f;
  float4 f = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int s0 = 0; s0 < parts; s0 += N) {
    float2 w[N];
    float4 v[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
      w[k] = make_float2(-INFINITY, 0.f);
      if (s0 + k >= parts) continue;
      w[k] = __ldcg(a.weights + (s0 + k) * rows + row);
      v[k] = __ldcg(reinterpret_cast<const float4*>(a.parts + ((s0 + k) * rows + row) * D) + lane);
    }
    float top = m;
#pragma unroll
    for (int k = 0; k < N; ++k) top = fmaxf(top, w[k].x);
    const float back = sum == 0.f ? 0.f : pa_ex2(m - top);
    f = make_float4(f.x * back, f.y * back, f.z * back, f.w * back);
    sum *= back;
    m = top;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      if (w[k].y == 0.f) continue;                         // its values were not written
      const float x = w[k].y * pa_ex2(w[k].x - m);
      sum += x;
      f = make_float4(fmaf(x, v[k].x, f.x), fmaf(x, v[k].y, f.y), fmaf(x, v[k].z, f.z), fmaf(x, v[k].w, f.w));
    }
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  reinterpret_cast<float4*>(a.parts + row * D)[lane] = make_float4(f.x * inv, f.y * inv, f.z * inv, f.w * inv);
  // the first part's weight, which all lanes of the row have read (with D 64 two rows of a warp go ways of their own)
  __syncwarp(D == 128 ? 0xffffffffu : 0xffffu << (threadIdx.x & 16));
  if (lane == 0) a.weights[row] = make_float2(m, sum);
}

// Rows of an entry (tokens x query heads of a group) up to which sharing is worth it: an entry with more fills a tile of the
// many-token kernel on its own, which reads codes once per 256 rows (more than 128: half a tile at least).
constexpr int kSharedRows = 128;
// Rows of a group up to which it takes one pass, reading the shared blocks once per tile of rows: two launches instead of
// three or four (a group of 16 rows, 8 heads, 4000 shared: 31 us, in two halves 41; of 64 rows over 16 000: 62 and 52).
constexpr int kTreeRows = 32;
// Tiles of 8 rows let two CTAs run on a multiprocessor, tiles of 16 read the shared blocks half as often.  They are taken
// where the former could read that many bytes again (16 groups of 16 rows, 8 heads, 4000 shared, 131 MB: 56 us with 8 rows, 64
// with 16; of 32 rows, 262 MB: 114 and 99; of 16 rows over 16 000, 524 MB: 185 and 151).  The host knows what tables can hold,
// not lengths: the figures are of tables as wide as the longest sequence.  With wider ones 16 x 4 beams of 100 - 3000 tokens
// take tiles of 16 rows as well (512 pages of 64 tokens: 53 us instead of 47).
constexpr double kTreeAgain = 192 << 20;
// Bytes that sharing could save at most, as far as the host knows, below which it is not tried: finding out what is shared
// takes 4 to 8 us, which is what ordinary attention takes to read that often (10 us for four short sequences).  Again by what
// tables can hold: four sequences of 266 tokens take 11 us with a table as wide as they are, 15.5 with one of 512 pages.
constexpr double kSharedLeast = 16 << 20;
// Parts of a row that the second half joins itself (join_shared); more are joined by a kernel of their own first (36 parts:
// 8 us of its own).
constexpr int kJoinParts = 2;
constexpr size_t kStepBytes = (size_t)10 << 20;           // of the partial results: those of the second half's step kernel

}  // namespace less

using namespace less;

extern "C" int less_pages_shared_attention(const less_pages* d, int32_t layer_begin, int32_t layer_count, int32_t n,
                                           const int32_t* seqs, const int32_t* starts, int32_t rows, int32_t max_new,
                                           int32_t ngroups, const int32_t* groups, int32_t max_group, const void* q,
                                           int64_t q_stride, int32_t window, int32_t sinks, float scale, void* out,
                                           void* stream) {
  PgParams p;
  PaSharedArgs a = {};
  int rc = pa_args(d, layer_begin, layer_count, n, seqs, starts, rows, max_new, q, q_stride, window, sinks, scale, out, &p, &a);
  if (rc != LESS_OK) return rc;
  if (n > d->seqs || ngroups < (n ? 1 : 0) || ngroups > n || max_group < 1) return LESS_ERR_INVALID_CONFIG;
  if (a.n == 0) return LESS_OK;
  if (!groups) return LESS_ERR_NULL_POINTER;
  if ((uintptr_t)groups & 3) return LESS_ERR_MISALIGNED;
  cudaStream_t s = (cudaStream_t)stream;
  const int64_t own = (int64_t)(starts ? max_new : 1) * d->group, all = (int64_t)max_group * d->group;
  const double most = (double)layer_count * d->heads * d->seq_pages * d->page_tokens * 2 * d->head_dim;   // bytes of a sequence
  const double save = (n - ngroups) * most;
  const size_t row_bytes = (size_t)d->head_dim * 4 + 8, room = LESS_PAGES_PARTIAL_BYTES - kStepBytes;
  const int64_t layer_rows = (int64_t)rows * d->heads * d->group, fit = (int64_t)(room / row_bytes) / layer_rows;
  if (own > kSharedRows || save < kSharedLeast || (fit == 0 && all > kTreeRows))
    return launch_pages_attention(p, a, d->head_dim, d->flags, max_new, s);
  int4* found = (int4*)pg_shared(d);
  a.entries = found;
  a.groups = found + d->seqs;
  if (all <= kTreeRows) a.tile = (double)((all + 7) / 8 - (all + 15) / 16) * ngroups * most >= kTreeAgain ? 16 : 8;
  rc = pg_launch("pages_common_kernel", pages_common_kernel, dim3(ngroups), PX_THREADS, 0, s, p, a, groups, ngroups);
  if (rc != LESS_OK) return rc;
  if (all <= kTreeRows) {
    a.n = ngroups;
    return launch_pages_tree(p, a, d->head_dim, d->flags, s);
  }
  // as many layers at a time as there is room for the parts of
  a.out_layers = layer_count;
  a.parts = p.partial + kStepBytes / 4;
  const size_t layer = (size_t)d->heads * d->group * d->head_dim * 2;
  for (int l0 = 0; l0 < layer_count && rc == LESS_OK; l0 += a.nl) {
    a.nl = (int)(fit < layer_count - l0 ? fit : layer_count - l0);
    a.layer0 = layer_begin + l0;
    a.q = (const char*)q + l0 * layer;
    a.out = (char*)out + l0 * layer;
    PaSharedArgs b = a;
    b.n = ngroups;
    b.window = b.sinks = 0;
    b.max_rows = 0;
    // how far the keys are split: as in ordinary attention
    const int64_t lists = (int64_t)a.nl * d->heads;
    b.twins = all <= 128 && fit / a.nl >= 2;
    int64_t items = (int64_t)rows * d->group / 256;
    if (items < ngroups) items = ngroups;
    int64_t splits = pg_sms() / (items * lists);
    if (splits > 32) splits = 32;
    if (splits > fit / a.nl / (b.twins ? 2 : 1)) splits = fit / a.nl / (b.twins ? 2 : 1);
    if (splits < 1) splits = 1;
    const int parts = (int)splits * (b.twins ? 2 : 1);
    b.splits = (int)splits;
    a.weights = b.weights = (float2*)(a.parts + parts * layer_rows * a.nl * d->head_dim);
    rc = launch_pages_prefix(p, b, d->head_dim, d->flags, s);
    a.splits = parts;
    if (rc == LESS_OK && parts > kJoinParts) {
      const int64_t threads = layer_rows * a.nl * (d->head_dim / 4);
      const dim3 grid((unsigned)((threads + 255) / 256));
      rc = d->head_dim == 128 ? pg_launch("pages_parts_kernel", pages_parts_kernel<128>, grid, 256, 0, s, p, a, parts)
                              : pg_launch("pages_parts_kernel", pages_parts_kernel<64>, grid, 256, 0, s, p, a, parts);
      a.splits = 1;
    }
    if (rc == LESS_OK) rc = launch_pages_step<kRest>(p, a, d->head_dim, d->flags, own > 8 ? 16 : 8, kStepBytes, kPgCounters, s);
  }
  return rc;
}
