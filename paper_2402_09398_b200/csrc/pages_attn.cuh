// What the two attention kernels over the paged 8-bit cache share (pages_step.cuh, pages_chunk.cuh).
#pragma once

#include "pages.cuh"

namespace less {

struct PaArgs {
  const void* q;
  void* out;
  int64_t q_stride;              // elements from token to token
  const int32_t* seqs;
  const int32_t* starts;
  int n, rows, layer0, nl;
  int max_rows;                  // entries with more rows (tokens x query heads of a group) are not this kernel's
  int window, sinks;             // window 0 = all
  float scale;
};

// attention of sequences that share their first pages (pages_shared.cu)
struct PaSharedArgs : PaArgs {
  const int4* groups;            // two of each group: {sequence, first row, tokens, first entry}, {sb, wb, eb, end of its entries}
                                 // with the blocks that it shares; tokens -1: starts that descend
  const int4* entries;           // of each entry: {sb, wb, eb, the most blocks that rows of a tile of its group have beside
                                 // the shared ones}
  float* parts;                  // [splits][rows * nl * heads * group][D]: results over the shared blocks
  float2* weights;               // [splits][rows * nl * heads * group]: (reference, sum); not written for entries that share nothing
  int splits;
  int tile;                      // rows of a tile of groups in one pass; 0: they are not
  int twins;                     // the many-token kernel leaves two parts for each of its splits
  int out_layers;                // layers between the rows of `out`
};

// What a launch is for: all that an entry sees; all that the entries of a group see (the group is then the entry; of a tile's
// rows all see the shared blocks, and those of an entry the rest of its blocks); the shared blocks alone (again the group is
// the entry, and results are parts); the rest of an entry's blocks (the parts are joined).
enum PaMode { kAll, kTree, kShared, kRest };

// the 16-token blocks that the tokens of an entry see: [0, sb) and [wb, eb)
struct Blocks {
  int sb, wb, eb;
  __device__ __forceinline__ int count() const { return sb + eb - wb; }
  __device__ __forceinline__ int at(int u) const { return u < sb ? u : wb + (u - sb); }
};
__device__ __forceinline__ Blocks visible_blocks(const PaArgs& a, int len, int count) {
  Blocks b;
  b.eb = pg_ceil(len, kPageBlock);
  b.sb = b.wb = 0;
  if (a.window) {
    b.wb = max(0, len - count - a.window + 1) / kPageBlock;
    b.sb = min(b.wb, pg_ceil(a.sinks, kPageBlock));
  }
  return b;
}

// Shared blocks, all of them visible to every token of a group: [0, sb) and [wb, eb).  An entry's rest is what remains of
// its own [0, sb) and [wb, eb): three stretches (sb and wb of a group are at most, at least those of its entries).
struct RestBlocks {
  int a, na, b, nb, c, nc;
  __device__ __forceinline__ int count() const { return na + nb + nc; }
  __device__ __forceinline__ int at(int u) const { return u < na ? a + u : u < na + nb ? b + u - na : c + u - na - nb; }
};
__device__ __forceinline__ RestBlocks rest_blocks(const Blocks& all, const int4& shared) {
  RestBlocks r;
  r.a = shared.x;
  r.na = max(0, all.sb - shared.x);
  r.b = all.wb;
  r.nb = max(0, shared.y - all.wb);
  r.c = max(shared.z, all.wb);
  r.nc = max(0, all.eb - r.c);
  return r;
}

// entry i and the blocks that it is about
template <PaMode MODE>
struct PaWork;
template <>
struct PaWork<kAll> {
  typedef PaArgs Args;
  typedef Blocks B;
  static __device__ __forceinline__ PgEntry entry(const PgParams& p, const PaArgs& a, int i) { return pg_entry(p, a.seqs, a.starts, a.rows, i); }
  static __device__ __forceinline__ B blocks(const PaArgs& a, int, const PgEntry& e) { return visible_blocks(a, e.len, e.count); }
};
template <>
struct PaWork<kTree> {
  typedef PaSharedArgs Args;
  typedef Blocks B;
  static __device__ __forceinline__ PgEntry entry(const PgParams&, const PaSharedArgs& a, int i) {
    const int4 g = __ldcg(a.groups + 2 * i);
    return {g.x, g.y, g.z, 0};
  }
  static __device__ __forceinline__ B blocks(const PaSharedArgs& a, int i, const PgEntry&) {
    const int4 b = __ldcg(a.groups + 2 * i + 1);
    return {b.x, b.y, b.z};
  }
};
template <>
struct PaWork<kShared> {
  typedef PaSharedArgs Args;
  typedef Blocks B;
  static __device__ __forceinline__ PgEntry entry(const PgParams&, const PaSharedArgs& a, int i) {
    const int4 g = __ldcg(a.groups + 2 * i), b = __ldcg(a.groups + 2 * i + 1);
    const int tokens = b.x + b.z - b.y > 0 ? g.z : 0;
    return {g.x, g.y, tokens, b.z * kPageBlock + tokens};  // every token lies behind the shared ones
  }
  static __device__ __forceinline__ B blocks(const PaSharedArgs& a, int i, const PgEntry&) {
    const int4 b = __ldcg(a.groups + 2 * i + 1);
    return {b.x, b.y, b.z};
  }
};
template <>
struct PaWork<kRest> {
  typedef PaSharedArgs Args;
  typedef RestBlocks B;
  static __device__ __forceinline__ PgEntry entry(const PgParams& p, const PaSharedArgs& a, int i) { return pg_entry(p, a.seqs, a.starts, a.rows, i); }
  static __device__ __forceinline__ B blocks(const PaSharedArgs& a, int i, const PgEntry& e) {
    return rest_blocks(visible_blocks(a, e.len, e.count), __ldcg(a.entries + i));
  }
};

__device__ __forceinline__ uint64_t f32x2_add(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

__device__ __forceinline__ float pa_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Exponents are those of P = p a_v: they include log2 a_v, so that what is rounded to fp16 is relative to the largest shares
// of a row's sum, wherever the magnitudes of other blocks lie.  The sums are relative to 2^m, a reference that follows the
// keys in both directions: fp16 has its 11 bits down to 2^-14 and nothing below 2^-25, and beside a first token that holds
// nearly all probability the others would vanish.  Where the largest exponent of the keys at hand is not within
// [m - 7, m + 15], m is set 7 below it: P is at most 2^15, the largest one 2^7 without rounding (a row whose sum is nearly
// one key's would show that rounding), and
// keys that it is too small for lose 2^-18 of the largest at hand.  Where a row that has a reference meets larger exponents,
// they as a rule come alone: m then goes 12 below them, so that the next keys are not far below it (2048 new tokens at 8192,
// one key block in a hundred four times as large: 10 us of 300 less than with 7).
// In the step kernel a lane sees its own keys only, and m goes down from 2 above it already once any row has to: rows just
// inside the range would call again and again.
constexpr float kRefNew = 7.f, kRefUp = 12.f, kRefMost = 15.f, kRefLeast = -7.f, kRefBack = 2.f;
// The sum of the probabilities takes 2^(exponent - log2 a_v - 8): with magnitudes in [2^-100, 2^100] (less counts as
// values of zero) 2^-102 of the token that has set m, 2^107 of any at most.
constexpr float kLeastValue = 0x1p-100f, kNoValues = -101.f, kSumBits = 8.f;

__device__ __forceinline__ float pa_scaled(float x, float d) {         // x 2^d, also where 2^d alone is out of range
  const float root = pa_ex2(0.5f * d);
  return x * root * root;
}

// (reference, sum) of a part of a row, the same but with the sum in [1, 2) if it was far from that: a weight in joining the
// parts is sum 2^(reference - largest), which is then lost only if it does not count, and times any value in range.  (The
// new reference is rounded: to 2^-18 of the weight up to 64.  Beyond 2^23 references are coarser than the exponent.)
__device__ __forceinline__ float2 pa_share(float m, float sum) {
  if (sum == 0.f) m = -INFINITY;                          // saw nothing
  const int bits = __float_as_int(sum), ex = (bits >> 23) - 127;
  if (sum >= 0x1p-126f && sum < INFINITY && abs(ex) > 20 && fabsf(m) < 0x1p23f) {
    m += (float)ex;
    sum = __int_as_float((bits & 0x007fffff) | 0x3f800000);
  }
  return make_float2(m, sum);
}

__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}

template <typename T>
__device__ __forceinline__ void store8(T* dst, const float* f);       // 8 values, 16 bytes
template <>
__device__ __forceinline__ void store8<__half>(__half* dst, const float* f) {
  uint4 u;
  __half2* h = reinterpret_cast<__half2*>(&u);
#pragma unroll
  for (int i = 0; i < 4; ++i) h[i] = __floats2half2_rn(f[2 * i], f[2 * i + 1]);
  *reinterpret_cast<uint4*>(dst) = u;
}
template <>
__device__ __forceinline__ void store8<__nv_bfloat16>(__nv_bfloat16* dst, const float* f) {
  uint4 u;
  __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&u);
#pragma unroll
  for (int i = 0; i < 4; ++i) h[i] = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
  *reinterpret_cast<uint4*>(dst) = u;
}
__device__ __forceinline__ void store4(__half* dst, float4 f) {
  __half2 h[2] = {__floats2half2_rn(f.x, f.y), __floats2half2_rn(f.z, f.w)};
  *reinterpret_cast<uint2*>(dst) = *reinterpret_cast<uint2*>(h);
}
__device__ __forceinline__ void store4(__nv_bfloat16* dst, float4 f) {
  __nv_bfloat162 h[2] = {__floats2bfloat162_rn(f.x, f.y), __floats2bfloat162_rn(f.z, f.w)};
  *reinterpret_cast<uint2*>(dst) = *reinterpret_cast<uint2*>(h);
}

// Rows of an entry (tokens x query heads of a group) up to which it is the step kernel's, which takes 16 at a time: more
// and it reads the codes again.  With fewer items (entries, layers, KV heads) than every second multiprocessor it is
// slower than the many-token kernel, whose keys are then split, from there on; with more only behind 32.
// Measured, step against many-token kernel, 8 KV heads x 8 queries of D 128 unless said:
//   24 rows (one KV head, D 64): 16 sequences of 1000: 28 / 19 us
//   32 rows:  one of 500: 18 / 20 us; one of 2000: 32 / 22; four of 1000: 34 / 22; 64 of 100: 28 / 46;
//             128 of 2000: 280 / 304; 64 of 1000, 32 KV heads x 1: 292 / 360
//   48 rows:  two of 30 000: 110 / 81; 16 of 2000: 79 / 46
// (Few short sequences lose 2 us by it: the host does not know the lengths.)
constexpr int kStepRows = 32, kStepRowsFew = 16;

int launch_pages_chunk(const PgParams& p, const PaArgs& a, int dim, uint32_t flags, cudaStream_t s);

// host: checks the arguments of an attention call and fills `p` and `a`; LESS_OK with a->n == 0: there is nothing to do
int pa_args(const less_pages* d, int32_t layer_begin, int32_t layer_count, int32_t n, const int32_t* seqs, const int32_t* starts,
            int32_t rows, int32_t max_new, const void* q, int64_t q_stride, int32_t window, int32_t sinks, float scale, void* out,
            PgParams* p, PaArgs* a);
int launch_pages_attention(const PgParams& p, PaArgs a, int dim, uint32_t flags, int32_t max_new, cudaStream_t s);
// results of the groups' tokens over the blocks that they share, into a.parts (pages_prefix.cu)
int launch_pages_prefix(const PgParams& p, const PaSharedArgs& a, int dim, uint32_t flags, cudaStream_t s);
// groups of few rows, in one launch (pages_tree.cu)
int launch_pages_tree(const PgParams& p, const PaSharedArgs& a, int dim, uint32_t flags, cudaStream_t s);

}  // namespace less
