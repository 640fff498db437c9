// Attention over the paged 8-bit cache for groups of sequences that share their first pages (beams of one text, samples,
// conversations behind one instruction): what ordinary attention gives, with the shared pages read once for a group.
//
//   o = (l_s o_s 2^(m_s - m) + l_r o_r 2^(m_r - m)) / (l_s 2^(m_s - m) + l_r 2^(m_r - m))
//
// with (m, l, o) reference, sum and quotient of a softmax over the shared blocks (s) and over the rest (r): the two halves
// are the kernels of ordinary attention, once with a group as one entry, whose rows are the tokens of all its sequences, once
// with the sequences as entries and the other blocks.  The second joins them where it would have written its result.
// What a group shares is found on the device: the leading pages that the tables of all its sequences have in common, of
// these the blocks that all its tokens see (a window moves with a sequence's end).  So a group is only a hint.
#include "pages_step.cuh"

namespace less {

constexpr int PX_THREADS = 512;

// One CTA per group.  A list of groups that is not [0 .. n] ascending is reported, and then nobody shares.
__global__ void __launch_bounds__(PX_THREADS) pages_common_kernel(PgParams p, PaArgs a, const int32_t* groups, int ngroups) {
  __shared__ int common, least_seen, most_len, least_wb, some, lead;
  __shared__ int refused;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = blockIdx.x;
  int4* entries = const_cast<int4*>(a.entries);
  int4* of = const_cast<int4*>(a.groups);
  pg_wait();
  if (tid == 0) {
    common = least_seen = least_wb = 0x7fffffff;
    most_len = some = refused = 0;
    lead = -1;
  }
  bool bad = false;
  for (int i = tid; i < ngroups; i += PX_THREADS) {
    const int b = __ldg(groups + i), e = __ldg(groups + i + 1);
    bad |= b < 0 || e < b || e > a.n || (i == 0 && b != 0) || (i == ngroups - 1 && e != a.n);
  }
  if (__syncthreads_or(bad)) {
    if (tid == 0) pg_status(p.status, kPagesBounds, 50);
    for (int i = g * PX_THREADS + tid; i < a.n; i += gridDim.x * PX_THREADS) entries[i] = make_int4(0, 0, 0, 0);
    if (tid < 2) of[2 * g + tid] = make_int4(0, 0, 0, 0);
    return;
  }
  const int e0 = __ldg(groups + g), e1 = __ldg(groups + g + 1);
  for (int i = e0 + tid; i < e1; i += PX_THREADS) {
    const PgEntry e = pg_entry(p, a.seqs, a.starts, a.rows, i);
    const int rows = a.starts ? __ldg(a.starts + i + 1) - __ldg(a.starts + i) : 1;
    if (rows != e.count || e.len < e.count) atomicOr(&refused, 1);   // not to be trusted: nobody of the group shares
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
  if (!refused && some > 1) {
    const int seen = least_seen / kPageBlock;             // blocks that the first token of every entry sees
    seq = __ldg(a.seqs + lead);
    const int pages = pg_ceil(seen * kPageBlock, p.pt);
    const int32_t* first = p.table + (size_t)seq * p.seq_pages;
    for (int i = e0 + warp; i < e1; i += PX_THREADS / 32) {
      if (a.starts && __ldg(a.starts + i + 1) == __ldg(a.starts + i)) continue;
      const int32_t* row = p.table + (size_t)__ldg(a.seqs + i) * p.seq_pages;
      if (row == first) continue;
      for (int o = 0; o < pages; o += 128) {
        bool differs[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int at = o + 32 * k + lane;
          differs[k] = at < pages && __ldcg(row + at) != __ldcg(first + at);
        }
        int at = -1;
#pragma unroll
        for (int k = 3; k >= 0; --k) {
          const uint32_t m = __ballot_sync(0xffffffffu, differs[k]);
          if (m) at = o + 32 * k + __ffs(m) - 1;
        }
        if (at >= 0 && lane == 0) atomicMin(&common, at);
        if (at >= 0 || __any_sync(0xffffffffu, *(volatile int*)&common <= o)) break;   // or another entry has parted before
      }
    }
    __syncthreads();
    blocks.z = min(seen, (int)min((int64_t)common * (p.pt / kPageBlock), (int64_t)1 << 28));
    if (a.window) {
      blocks.y = min(blocks.z, pg_ceil(max(0, most_len - a.window), kPageBlock));
      blocks.x = min(min(a.sinks / kPageBlock, least_wb), blocks.y);
    }
    if (blocks.x + blocks.z - blocks.y <= 0) blocks = make_int4(0, 0, 0, 0);
  }
  for (int i = e0 + tid; i < e1; i += PX_THREADS) entries[i] = blocks;
  if (tid == 0) {
    const int row0 = e0 < a.n ? (a.starts ? min(max(__ldg(a.starts + e0), 0), a.rows) : e0) : a.rows;
    const int end = a.starts ? min(max(__ldg(a.starts + e1), row0), a.rows) : e1;
    of[2 * g] = make_int4(seq, row0, blocks.z ? end - row0 : 0, 0);
    of[2 * g + 1] = blocks;
  }
}

// Rows of an entry (tokens x query heads of a group) up to which sharing is worth it: an entry with more fills a tile of the
// many-token kernel on its own, which reads codes once per 256 rows.
constexpr int kSharedRows = 128;
constexpr size_t kStepBytes = (size_t)10 << 20;           // of the partial results: those of either half's step kernel

}  // namespace less

using namespace less;

extern "C" int less_pages_shared_attention(const less_pages* d, int32_t layer_begin, int32_t layer_count, int32_t n,
                                           const int32_t* seqs, const int32_t* starts, int32_t rows, int32_t max_new,
                                           int32_t ngroups, const int32_t* groups, int32_t max_group, const void* q,
                                           int64_t q_stride, int32_t window, int32_t sinks, float scale, void* out,
                                           void* stream) {
  PgParams p;
  PaArgs a;
  int rc = pa_args(d, layer_begin, layer_count, n, seqs, starts, rows, max_new, q, q_stride, window, sinks, scale, out, &p, &a);
  if (rc != LESS_OK) return rc;
  if (n > d->seqs || ngroups < (n ? 1 : 0) || ngroups > n || max_group < 1) return LESS_ERR_INVALID_CONFIG;
  if (a.n == 0) return LESS_OK;
  if (!groups) return LESS_ERR_NULL_POINTER;
  if ((uintptr_t)groups & 3) return LESS_ERR_MISALIGNED;
  cudaStream_t s = (cudaStream_t)stream;
  const int64_t own = (int64_t)(starts ? max_new : 1) * d->group, all = (int64_t)max_group * d->group;
  const size_t row_bytes = (size_t)d->head_dim * 4 + 8, room = LESS_PAGES_PARTIAL_BYTES - 2 * kStepBytes;
  const int64_t layer_rows = (int64_t)rows * d->heads * d->group, fit = (int64_t)(room / row_bytes) / layer_rows;
  if (own > kSharedRows || fit == 0) return launch_pages_attention(p, a, d->head_dim, d->flags, max_new, s);
  a.entries = p.shared;
  a.groups = p.shared + d->seqs;
  rc = pg_launch("pages_common_kernel", pages_common_kernel, dim3(ngroups), PX_THREADS, 0, s, p, a, groups, ngroups);
  // as many layers at a time as there is room for the parts of
  a.out_layers = layer_count;
  a.parts = p.partial + 2 * kStepBytes / 4;
  const size_t layer = (size_t)d->heads * d->group * d->head_dim * 2;
  for (int l0 = 0; l0 < layer_count && rc == LESS_OK; l0 += a.nl) {
    a.nl = (int)(fit < layer_count - l0 ? fit : layer_count - l0);
    a.layer0 = layer_begin + l0;
    a.q = (const char*)q + l0 * layer;
    a.out = (char*)out + l0 * layer;
    PaArgs b = a;
    PgParams pb = p;
    b.n = ngroups;
    b.window = b.sinks = 0;
    b.max_rows = 0;
    pb.partial = p.partial + kStepBytes / 4;
    pb.counters = p.counters + kPgCounters / 2;
    const int64_t lists = (int64_t)a.nl * d->heads;
    const bool many = all > (ngroups * lists * 2 <= pg_sms() ? kStepRowsFew : kStepRows);
    int64_t splits = 1;
    if (many) {                                           // as in ordinary attention
      int64_t items = (int64_t)rows * d->group / 256;
      if (items < ngroups) items = ngroups;
      splits = pg_sms() / (items * lists);
      if (splits > 32) splits = 32;
      if (splits > fit / a.nl) splits = fit / a.nl;
      if (splits < 1) splits = 1;
    } else {
      b.max_rows = 0x7fffffff;
    }
    a.splits = b.splits = (int)splits;
    a.weights = b.weights = (float2*)(a.parts + splits * layer_rows * a.nl * d->head_dim);
    rc = launch_pages_prefix(pb, b, d->head_dim, d->flags, all > 0x7fffffff ? 0x7fffffff : (int)all, many, kStepBytes, kPgCounters / 2, s);
    if (rc == LESS_OK)
      rc = launch_pages_step<kRest>(p, a, d->head_dim, d->flags, own > 8 ? 16 : 8, kStepBytes, kPgCounters / 2, s);
  }
  return rc;
}
