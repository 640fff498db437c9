// The selection of beam search: of the candidates (beam, token) of a group the `keep` largest
//
//   v(b, t) = score_b + l(b, t) - log sum_u exp l(b, u),     ties to the lowest (b, t)
//
// Bound by memory: every logit of a live beam is read once (2 or 4 bytes; an exponential, a sum and two comparisons each).
//   - A row of logits is cut into stretches, a CTA each, where there are too few rows to fill the GPU.  A CTA takes, in one
//     pass, the sum of exponentials relative to a reference (the largest logit of its first tile; moved only
//     where a later one lies more than 2^57 above) and its `keep` largest logits.  Those pass a bar: the keep-th largest of
//     the maxima of 64 (256) groups of threads over the first tile, which at least `keep` elements reach and, of n elements
//     like those of the tile, about keep n / tile.  They go to a list in shared memory, which is cut down to the largest
//     `keep`, and the bar raised, whenever twice as many elements have been seen.
//   - The CTA of a group that arrives last joins: the rows' sums, then the candidates of all beams, by counting for each how
//     many come before it.
// Within a beam the order is that of the logits, which is exact.  Between beams it hangs on the sums.  A term exp2(x) of
// one is off, relative, by 2^-22 (the exponential), |x| 2^-23.4 (x: a product with a rounded factor, for fp32 logits of a
// rounded difference) and 6 * 2^-24 (added to fifteen others; the rest is in 64 bits, rounded once at the end), so a sum
// by at most 6.1e-7 + 1e-7 times the mean of |x| weighted with the terms, which is summed up beside it (a thread's -x, and twice
// its largest x where it has logits above its reference).
// Where two candidates are of different beams and closer than that, the sums of these beams are computed again
// to 1e-10 and the candidates joined once more (a chance of some 1e-4 per kept candidate: of 60 inputs of the large case below
// one; 58 us for a row of 128 256, one CTA's work that waits for memory, so two such rows make 176 us of its 61 us between events).
// References beyond 2^16 take differences before they scale them (32 x 8 beams of 128 256 fp32 logits near 1e6: 78 us instead
// of 61).  A stretch that has more equal logits at its bar than the list holds is gone through again in order: rows that
// begin with thousands of tokens masked with one finite value take 600 us (with -inf 55: that is no candidate).
// Measured: 64 x 8 beams of 128 256 bf16 logits (119 MB of live ones): 55 us, 2.2 TB/s, issue slots half used - some 88
// instructions per warp and 512 bytes - and 465 live rows on 148 multiprocessors of four CTAs; 4 beams of 32 000: 14 - 17 us, a
// chain of waits.  With the rows loaded to registers instead of through a ring of copies 72 us.
#include <float.h>

#include <atomic>

#include "less_internal.cuh"
#include "pages_attn.cuh"

namespace less {

constexpr int BM_THREADS = 256;
constexpr int BM_RING = 8;                                // 16-byte pieces of a thread on their way (a thread's own, so no barriers)
constexpr int BM_FIRST = 4;                               // of them those of the first tile
constexpr int BM_LIST = 1280;                             // candidates that a list holds: more than 9 BM_MOST_KEEP
constexpr int BM_CTAS = 4;                                // on a multiprocessor
constexpr int BM_MOST_BEAMS = 64, BM_MOST_KEEP = 128;
constexpr int BM_JOINED = 8192;                           // candidates of a group that are joined, about
constexpr int BM_DIRECT = 320;                            // as many are compared with one another at once
constexpr float kRefFar = 40.f;                           // a logit that far above the reference moves it
constexpr float kRefPacked = 65536.f;                      // references beyond: differences are taken before they are scaled
// error of a sum: kSumError + kTermError times the mean of |x|
constexpr double kSumError = 6.1e-7, kTermError = 1.0e-7;

struct BmArgs {
  const void* logits;
  int64_t stride;                                         // elements from row to row
  const float* scores;
  const uint8_t* ended;                                   // or null
  int groups, beams, vocab, keep, end_token;
  int splits, per;                                        // stretches of a row, 16-byte pieces of each
  float* out_scores;
  int32_t* out_tokens;
  int32_t* out_parents;
  uint8_t* out_ended;
  int32_t* counters;                                      // [groups] zero between calls
  float4* sums;                                           // [rows][splits] (reference, sum, sum of the terms times |x| or a little more, 0)
  unsigned long long* keys;                               // [rows][splits][keep]
};

// Elements of 16 bytes and what is done with them packed.  NaN counts as -inf throughout: a maximum ignores it.
template <typename T>
struct BmType;
template <>
struct BmType<float> {
  static constexpr int N = 4;
  static constexpr float most = FLT_MAX;
  static __device__ __forceinline__ float below(float x) { return __fsub_rd(x, 87.f); }
  static __device__ __forceinline__ uint32_t pack(float x) { return __float_as_uint(x); }
  static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) { return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b))); }
  static __device__ __forceinline__ uint32_t smaller(uint32_t a, uint32_t b) { return __float_as_uint(fminf(__uint_as_float(a), __uint_as_float(b))); }
  static __device__ __forceinline__ float top(uint32_t m) { return __uint_as_float(m); }
  static __device__ __forceinline__ void unpack(uint32_t u, float* f) { f[0] = __uint_as_float(u); }
  static __device__ __forceinline__ float load(const void* p) { return fmaxf(__ldcg((const float*)p), -INFINITY); }
};
template <>
struct BmType<__half> {
  static constexpr int N = 8;
  static constexpr float most = 65504.f;
  static __device__ __forceinline__ float below(float x) { return __half2float(__float2half_rd(x - 87.f)); }
  static __device__ __forceinline__ uint32_t pack(float x) {
    const __half2 h = __float2half2_rn(x);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) {
    const __half2 h = __hmax2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  static __device__ __forceinline__ uint32_t smaller(uint32_t a, uint32_t b) {
    const __half2 h = __hmin2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  static __device__ __forceinline__ float top(uint32_t m) {
    const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&m));
    return fmaxf(x.x, x.y);
  }
  static __device__ __forceinline__ void unpack(uint32_t u, float* f) {
    const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&u));
    f[0] = x.x;
    f[1] = x.y;
  }
  static __device__ __forceinline__ float load(const void* p) {
    return fmaxf(__half2float(__ushort_as_half(__ldcg((const unsigned short*)p))), -INFINITY);
  }
};
template <>
struct BmType<__nv_bfloat16> {
  static constexpr int N = 8;
  static constexpr float most = 3.38953138925153547590470800371487866880e+38f;
  static __device__ __forceinline__ float below(float x) { return __bfloat162float(__float2bfloat16_rd(__fsub_rd(x, 87.f))); }
  static __device__ __forceinline__ uint32_t pack(float x) {
    const __nv_bfloat162 h = __float2bfloat162_rn(x);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) {
    const __nv_bfloat162 h = __hmax2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  static __device__ __forceinline__ uint32_t smaller(uint32_t a, uint32_t b) {
    const __nv_bfloat162 h = __hmin2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  static __device__ __forceinline__ float top(uint32_t m) { return fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u)); }
  static __device__ __forceinline__ void unpack(uint32_t u, float* f) {
    f[0] = __uint_as_float(u << 16);
    f[1] = __uint_as_float(u & 0xffff0000u);
  }
  static __device__ __forceinline__ float load(const void* p) {
    return fmaxf(__uint_as_float((uint32_t)__ldcg((const unsigned short*)p) << 16), -INFINITY);
  }
};

template <typename T>
__device__ __forceinline__ float bm_top(const uint4& w) {               // the largest; NaN: all are
  typedef BmType<T> B;
  return B::top(B::larger(B::larger(w.x, w.y), B::larger(w.z, w.w)));
}
template <typename T>
__device__ __forceinline__ void bm_unpack(const uint4& w, uint32_t floor, float* f) {    // at least the floor
  typedef BmType<T> B;
  constexpr int N = B::N / 4;
  B::unpack(B::larger(w.x, floor), f);
  B::unpack(B::larger(w.y, floor), f + N);
  B::unpack(B::larger(w.z, floor), f + 2 * N);
  B::unpack(B::larger(w.w, floor), f + 3 * N);
}

// order of a beam's candidates: the logit, then the lower token; 0 = none
__device__ __forceinline__ unsigned long long bm_key(float l, int token) {
  const uint32_t b = __float_as_uint(l + 0.f);            // the two zeros are equal
  const uint32_t o = b & 0x80000000u ? ~b : b | 0x80000000u;
  return (unsigned long long)o << 32 | (0xffffffffu - (uint32_t)token);
}
__device__ __forceinline__ float bm_logit(unsigned long long key) {
  const uint32_t o = (uint32_t)(key >> 32);
  return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ int bm_token(unsigned long long key) { return (int)(0xffffffffu - (uint32_t)key); }

// a beam that takes part: its score is finite
__device__ __forceinline__ bool bm_live(float score) { return fabsf(score) <= FLT_MAX; }

// (value, beam, token) of a candidate of the group; the value as an integer of the same order
struct BmCand {
  long long v;
  unsigned long long at;                                  // what decides between equal values: the beam (6 bits), the larger
                                                          // logit (32; no key's high half is 0), the token (26); ~0 = none
};
__device__ __forceinline__ unsigned long long bm_at(int beam, unsigned long long key, int token) {
  return (unsigned long long)beam << 58 | (unsigned long long)~(uint32_t)(key >> 32) << 26 | (uint32_t)token;
}
__device__ __forceinline__ int bm_beam(const BmCand& x) { return (int)(x.at >> 58); }
constexpr long long kNoCand = (long long)0x8000000000000000ull;
__device__ __forceinline__ long long bm_order(double v) {
  const long long b = __double_as_longlong(v + 0.0);      // the two zeros are equal
  return b ^ (b >> 63 & 0x7fffffffffffffffll);
}
__device__ __forceinline__ double bm_value(long long o) { return __longlong_as_double(o ^ (o >> 63 & 0x7fffffffffffffffll)); }
__device__ __forceinline__ bool bm_before(const BmCand& a, const BmCand& b) { return a.v > b.v || (a.v == b.v && a.at < b.at); }

struct BmShared {
  uint4 ring[BM_RING][BM_THREADS];
  union {
    unsigned long long list[BM_LIST];
    struct {
      BmCand cand[BM_LIST / 2];
      double score[BM_MOST_BEAMS], lse[BM_MOST_BEAMS], err[BM_MOST_BEAMS];   // -inf = no candidates; error of the second
    } j;
  };
  union {
    float best[BM_THREADS];
    BmCand most[BM_THREADS];
    unsigned long long high[BM_THREADS];
    double dsum[BM_THREADS / 32];
  };
  union {
    BmCand top[BM_MOST_KEEP];
    unsigned long long kept[BM_MOST_KEEP];
  };
  float wmax[BM_THREADS / 32];
  float ref[BM_THREADS / 32];
  float bar;
  unsigned long long bar_key;
  BmCand bar_cand;
  unsigned long long again, done;                         // beams whose sums are computed again; that have ended
  int count, last;
};

__device__ __forceinline__ float bm_block_max(BmShared& sh, float x) {
#pragma unroll
  for (int d = 16; d; d >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, d));
  __syncthreads();
  if ((threadIdx.x & 31) == 0) sh.wmax[threadIdx.x >> 5] = x;
  __syncthreads();
  x = sh.wmax[0];
#pragma unroll
  for (int w = 1; w < BM_THREADS / 32; ++w) x = fmaxf(x, sh.wmax[w]);
  return x;
}

// For each of `count` things how many come before it, before(k, i): eight lanes per thing.  Whole block; `put(i, rank)` is one
// lane's.
template <typename Before, typename Put>
__device__ __forceinline__ void bm_rank(int count, Before before, Put put) {
  for (int base = 0; base < count; base += BM_THREADS / 8) {
    const int i = base + (int)threadIdx.x / 8;
    int rank = 0;
    if (i < count)
#pragma unroll 4
      for (int k = threadIdx.x & 7; k < count; k += 8) rank += before(k, i);
#pragma unroll
    for (int d = 1; d < 8; d <<= 1) rank += __shfl_xor_sync(0xffffffffu, rank, d);
    if (i < count && (threadIdx.x & 7) == 0) put(i, rank);
  }
}

// The elements of a row by 16-byte pieces: `head` before the first whole one, `tail` behind the last
template <typename T>
struct BmRow {
  const T* base;
  int head, pieces, tail;
  __device__ __forceinline__ BmRow(const BmArgs& a, int row) {
    constexpr int N = BmType<T>::N;
    base = reinterpret_cast<const T*>(a.logits) + (int64_t)row * a.stride;
    head = min(a.vocab, (int)(((16u - (uint32_t)(reinterpret_cast<uintptr_t>(base) & 15)) & 15u) / sizeof(T)));
    pieces = (a.vocab - head) / N;
    tail = a.vocab - head - pieces * N;
  }
  __device__ __forceinline__ uint4 piece(int i) const { return __ldcg(reinterpret_cast<const uint4*>(base + head) + i); }
  __device__ __forceinline__ int token(int i) const { return head + i * BmType<T>::N; }
  // single elements: those before and behind the pieces, -1 = none
  __device__ __forceinline__ int single(int i, bool front, bool back) const {
    if (i < head) return front ? i : -1;
    return i - head < tail && back ? head + pieces * BmType<T>::N + i - head : -1;
  }
};

// A stretch that has more candidates than the list holds (many equal logits, or ascending ones): again, in order, by tiles
// of a piece per thread.  Of a tile only elements at least as large as the keep-th largest of the threads' maxima count
// (at most keep * N), and only those above the keep-th so far.
template <typename T>
__device__ __noinline__ void bm_crowded(BmShared& sh, const BmArgs& a, const BmRow<T>& row, int p0, int p1, bool front, bool back,
                                        unsigned long long* out) {
  constexpr int N = BmType<T>::N;
  const int tid = threadIdx.x;
  __syncthreads();
  if (tid == 0) sh.count = 0;
  unsigned long long floor = 0;                           // the keep-th so far, once there are as many
  for (int at = p0 - BM_THREADS; at < p1; at += BM_THREADS) {      // the first turn is that of the single elements
    float f[N];
    int token = 0, n = 0;
    if (at < p0) {
      token = row.single(tid, front, back);
      if (token >= 0) {
        f[0] = BmType<T>::load(row.base + token);
        n = 1;
      }
    } else if (at + tid < p1) {
      bm_unpack<T>(row.piece(at + tid), BmType<T>::pack(-INFINITY), f);
      token = row.token(at + tid);
      n = N;
    }
    unsigned long long high = 0;
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < n && f[i] > -INFINITY) {
        const unsigned long long k = bm_key(fminf(f[i], BmType<T>::most), token + i);
        high = k > high ? k : high;
      }
    __syncthreads();
    sh.high[tid] = high;
    if (tid == 0) sh.bar_key = 0;
    __syncthreads();
    int larger = 0;
    for (int i = 0; i < BM_THREADS; ++i) larger += sh.high[i] > high;
    if (high && larger == a.keep - 1) sh.bar_key = high;
    __syncthreads();
    const unsigned long long bar = max(sh.bar_key, floor);
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < n && f[i] > -INFINITY) {
        const unsigned long long k = bm_key(fminf(f[i], BmType<T>::most), token + i);
        if (k >= bar) sh.list[atomicAdd(&sh.count, 1)] = k;       // at most keep * (N + 1) of BM_LIST
      }
    __syncthreads();
    const int count = sh.count;
    unsigned long long mine[(BM_MOST_KEEP * 9 + BM_THREADS - 1) / BM_THREADS];
    int rank[(BM_MOST_KEEP * 9 + BM_THREADS - 1) / BM_THREADS];
#pragma unroll
    for (int j = 0; j < (BM_MOST_KEEP * 9 + BM_THREADS - 1) / BM_THREADS; ++j) {
      const int i = tid + j * BM_THREADS;
      mine[j] = i < count ? sh.list[i] : 0;
      rank[j] = BM_LIST;
      if (mine[j]) {
        rank[j] = 0;
        for (int k = 0; k < count; ++k) rank[j] += sh.list[k] > mine[j];
      }
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < (BM_MOST_KEEP * 9 + BM_THREADS - 1) / BM_THREADS; ++j)
      if (rank[j] < a.keep) sh.list[rank[j]] = mine[j];
    if (tid == 0) sh.count = min(count, a.keep);
    __syncthreads();
    if (count >= a.keep) floor = sh.list[a.keep - 1] + 1;          // keys are of one token each: only larger ones count
  }
  for (int i = tid; i < a.keep; i += BM_THREADS) out[i] = i < sh.count ? sh.list[i] : 0;
}

// 2^f, |f| <= 1/2, by its Taylor polynomial of degree 11 (error below 1e-14)
__device__ __forceinline__ double bm_exp2(double x) {
  if (x < -1020.0) return 0.0;
  const double n = rint(x), z = (x - n) * 0.693147180559945309417232;
  double p = 1.0 / 39916800.0;
  p = fma(p, z, 1.0 / 3628800.0);
  p = fma(p, z, 1.0 / 362880.0);
  p = fma(p, z, 1.0 / 40320.0);
  p = fma(p, z, 1.0 / 5040.0);
  p = fma(p, z, 1.0 / 720.0);
  p = fma(p, z, 1.0 / 120.0);
  p = fma(p, z, 1.0 / 24.0);
  p = fma(p, z, 1.0 / 6.0);
  p = fma(p, z, 0.5);
  p = fma(p, z, 1.0);
  p = fma(p, z, 1.0);
  return p * __hiloint2double(((int)n + 1023) << 20, 0);
}
// Which thread adds which tokens, and the reference, do not depend on where a row lies: equal rows give equal sums.
template <typename T>
__device__ __noinline__ double bm_exact_sum(BmShared& sh, const BmArgs& a, int r) {
  const T* row = reinterpret_cast<const T*>(a.logits) + (int64_t)r * a.stride;
  const int tid = threadIdx.x;
  unsigned long long top = 0;                              // the largest logit: a stretch's first
  for (int s = 0; s < a.splits; ++s) top = max(top, __ldcg(a.keys + ((size_t)r * a.splits + s) * a.keep));
  const float m = bm_logit(top);
  // l - m = k ln 2 / 1024 + z, |z| <= 3.4e-4: 2^(k / 1024) from a table in 64 bits, e^z - 1 as z + z^2 / 2 + z^3 / 6 in 32 (5e-11
  // of e^z; with the roundings of z).  The unit for 64-bit arithmetic is the bound otherwise.
  double* pow2 = reinterpret_cast<double*>(sh.ring);
  for (int k = tid; k < 1024; k += BM_THREADS) pow2[k] = bm_exp2(k / 1024.0);
  __syncthreads();
  double s = 0.0;
  constexpr int N = 4;
  float f[N];
  auto load = [&](int at) {
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = at + i * BM_THREADS < a.vocab ? BmType<T>::load(row + at + i * BM_THREADS) : -INFINITY;
  };
  load(tid);
  for (int at = tid; at < a.vocab; at += N * BM_THREADS) {
    float x[N];
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = fminf(f[i], BmType<T>::most);
    load(at + N * BM_THREADS);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float d = x[i] - m, back = d - x[i], rest = (x[i] - (d - back)) - (m + back);   // d + rest is the difference
      if (d < -680.f) d = -680.f, rest = 0.f;              // below 2^-980 each (-inf among them, where rest is no number)
      const float k = rintf(d * 1477.3197218702985f);
      const float z = fmaf(-k, -0x1.05c61p-39f, fmaf(-k, 0x1.62e43p-11f, d)) + rest;
      const float q = fmaf(z * z, fmaf(z, 0.16666667f, 0.5f), z);
      const double t = pow2[(int)k & 1023];
      const double y = __hiloint2double(__double2hiint(t) + (((int)k >> 10) << 20), __double2loint(t));
      s = fma(y, (double)q, s + y);
    }
  }
#pragma unroll
  for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
  __syncthreads();
  if ((tid & 31) == 0) sh.dsum[tid >> 5] = s;
  __syncthreads();
  s = 0.0;
  for (int w = 0; w < BM_THREADS / 32; ++w) s += sh.dsum[w];
  return (double)m + log(s);
}

// The candidates of a group: its beams' lists, an ended beam's one.  Whole block of the CTA that arrived last.
template <typename T>
__device__ __noinline__ void bm_join(BmShared& sh, const BmArgs& a, int group) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, B = a.beams, K = a.keep;
  const unsigned long long* keys = a.keys + (size_t)group * B * a.splits * K;
  const float4* sums = a.sums + (size_t)group * B * a.splits;
  const float* scores = a.scores + (size_t)group * B;
  const uint8_t* ended = a.ended ? a.ended + (size_t)group * B : nullptr;
  const int per_beam = a.splits * K, total = B * per_beam;
  // (of a beam that is not live: what lies there, which nobody looks at)
  auto key_of = [&](int i) { return __ldcg(keys + i); };
  const unsigned long long first_key = tid < total ? key_of(tid) : 0;   // asked for early
  if (tid == 0) sh.done = 0;
  __syncthreads();
  for (int b = warp; b < B; b += BM_THREADS / 32) {
    const float score = __ldcg(scores + b);
    const bool done = ended && __ldcg(ended + b);
    double c = bm_live(score) ? (double)score : -INFINITY, lse = 0.0, err = 0.0;
    if (done && lane == 0) atomicOr(&sh.done, 1ull << b);
    if (bm_live(score) && !done) {
      float m = -INFINITY;
      for (int s = lane; s < a.splits; s += 32) {
        const float4 x = __ldcg(sums + b * a.splits + s);
        if (x.y > 0.f) m = fmaxf(m, x.x);
      }
#pragma unroll
      for (int d = 16; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
      double sum = 0.0, far = 0.0;
      for (int s = lane; s < a.splits; s += 32) {
        const float4 x = __ldcg(sums + b * a.splits + s);
        if (!(x.y > 0.f)) continue;
        const double back = ((double)x.x - (double)m) * 1.44269504088896340735992, scale = bm_exp2(back);
        sum += (double)x.y * scale;
        if (scale > 0.0) far += ((double)x.z - back * (double)x.y) * scale;
      }
#pragma unroll
      for (int d = 16; d; d >>= 1) {
        sum += __shfl_xor_sync(0xffffffffu, sum, d);
        far += __shfl_xor_sync(0xffffffffu, far, d);
      }
      if (sum > 0.0) {
        lse = (double)m + log(sum);
        err = kSumError + kTermError * far / sum;
      } else {
        c = -INFINITY;
      }
    }
    if (lane == 0) {
      sh.j.score[b] = c;
      sh.j.lse[b] = lse;
      sh.j.err[b] = err;
    }
  }
  if (tid == 0) sh.again = 0;
  __syncthreads();
  // candidate i of the group's lists, whose key is at hand; at = ~0: none
  auto cand = [&](int i, unsigned long long key) {
    BmCand x = {kNoCand, ~0ull};
    const int b = i / per_beam;
    const double c = sh.j.score[b];
    if (c == -INFINITY) return x;
    if (sh.done >> b & 1) {
      if (i == b * per_beam && a.end_token >= 0) x = {bm_order(c), bm_at(b, ~0ull, a.end_token)};   // (its only one)
      return x;
    }
    if (key) x = {bm_order(c + ((double)bm_logit(key) - sh.j.lse[b])), bm_at(b, key, bm_token(key))};
    return x;
  };
  auto differ = [&](const BmCand& x, const BmCand& y) {   // whether the errors of the sums could change the order of two
    const int i = bm_beam(x), j = bm_beam(y);
    const double err = sh.j.err[i] + sh.j.err[j];         // an ended beam has none
    if (i != j && err > 0.0 && bm_value(x.v) - bm_value(y.v) <= err) atomicOr(&sh.again, 1ull << i | 1ull << j);
  };
  double most_err = 0.0;
  for (int b = 0; b < B; ++b) most_err = fmax(most_err, sh.j.err[b]);

  for (bool refined = false;; refined = true) {
    if (tid == 0) sh.count = 0;
    __syncthreads();
    long long bar = kNoCand + 1;
    if (total > BM_DIRECT) {
      // the bar: the keep-th of the best ones of 64 (256) groups of threads, less what the errors of the sums could change
      BmCand best = {kNoCand, ~0ull};
      for (int i = tid; i < total; i += BM_THREADS) {
        const BmCand x = cand(i, i == tid ? first_key : key_of(i));
        if (bm_before(x, best)) best = x;
      }
      const bool wide = K > 32;
      if (!wide) {
#pragma unroll
        for (int d = 1; d < 4; d <<= 1) {
          const BmCand y = {__shfl_xor_sync(0xffffffffu, best.v, d), __shfl_xor_sync(0xffffffffu, best.at, d)};
          if (bm_before(y, best)) best = y;
        }
      }
      const int of = wide ? BM_THREADS : BM_THREADS / 4;
      if (wide || (tid & 3) == 0) sh.most[wide ? tid : tid >> 2] = best;
      if (tid == 0) sh.bar_cand.v = bar;
      __syncthreads();
      if (tid < of) {
        const BmCand mine = sh.most[tid];
        int larger = 0;
#pragma unroll 8
        for (int i = 0; i < of; ++i) larger += bm_before(sh.most[i], mine);
        if (mine.at != ~0ull && larger == K - 1) sh.bar_cand.v = bm_order(bm_value(mine.v) - 2.0 * most_err);
      }
      __syncthreads();
      bar = sh.bar_cand.v;
    }
    for (int i = tid; i < total; i += BM_THREADS) {
      const BmCand x = cand(i, i == tid ? first_key : key_of(i));
      if (x.at != ~0ull && x.v >= bar) {
        const int n = atomicAdd(&sh.count, 1);
        if (n < BM_LIST / 2) sh.j.cand[n] = x;
      }
    }
    __syncthreads();
    const int count = sh.count;
    int found;
    if (count <= BM_LIST / 2) {
      found = min(count, K);
      bm_rank(count, [&](int k, int i) { return bm_before(sh.j.cand[k], sh.j.cand[i]); },
              [&](int i, int rank) { if (rank < K) sh.top[rank] = sh.j.cand[i]; });
      __syncthreads();
      if (!refined) {
        // every two, not neighbours alone: one between them may be of a beam whose sum has a smaller error
        const double reach = 2.0 * most_err;
        for (int i = tid; i < found; i += BM_THREADS)
          for (int k = i + 1; k < found && bm_value(sh.top[i].v) - bm_value(sh.top[k].v) <= reach; ++k) differ(sh.top[i], sh.top[k]);
        if (count > K)                                    // and those that could come in
          for (int i = tid; i < count; i += BM_THREADS) {
            const BmCand x = sh.j.cand[i];
            if (!bm_before(sh.top[K - 1], x)) continue;
            for (int k = K - 1; k >= 0 && bm_value(sh.top[k].v) - bm_value(x.v) <= reach; --k) differ(sh.top[k], x);
          }
      }
    } else {
      // too many near the bar: one after the other, and all sums in 64 bits
      found = 0;
      BmCand last = {0x7fffffffffffffffll, 0};
      if (!refined && tid == 0) sh.again = ~0ull;
      for (; refined && found < K; ++found) {
        BmCand x = {kNoCand, ~0ull};
        for (int i = tid; i < total; i += BM_THREADS) {
          const BmCand y = cand(i, key_of(i));
          if (y.at != ~0ull && bm_before(last, y) && bm_before(y, x)) x = y;
        }
        __syncthreads();
        sh.most[tid] = x;
        __syncthreads();
        for (int d = BM_THREADS / 2; d; d >>= 1) {
          if (tid < d && bm_before(sh.most[tid + d], sh.most[tid])) sh.most[tid] = sh.most[tid + d];
          __syncthreads();
        }
        last = sh.most[0];
        if (last.at == ~0ull) break;
        if (tid == 0) sh.top[found] = last;
      }
    }
    __syncthreads();
    const unsigned long long again = sh.again;
    if (refined || again == 0) {
      for (int i = tid; i < K; i += BM_THREADS) {
        const bool some = i < found;
        const BmCand x = some ? sh.top[i] : BmCand{kNoCand, 0};
        const size_t o = (size_t)group * K + i;
        const int token = some ? (int)(x.at & ((1u << 26) - 1)) : -1;
        a.out_scores[o] = some ? (float)bm_value(x.v) : -INFINITY;
        a.out_tokens[o] = token;
        a.out_parents[o] = group * B + (some ? bm_beam(x) : min(i, B - 1));
        if (a.out_ended) a.out_ended[o] = some && token == a.end_token;
      }
      return;
    }
    for (int b = 0; b < B; ++b) {
      if (!(again >> b & 1) || sh.j.score[b] == -INFINITY || (sh.done >> b & 1)) continue;   // uniform over the block
      const double lse = bm_exact_sum<T>(sh, a, group * B + b);
      if (tid == 0) sh.j.lse[b] = lse;
    }
    __syncthreads();
  }
}

template <typename T>
__global__ void __launch_bounds__(BM_THREADS, BM_CTAS) beam_select_kernel(BmArgs a) {
  constexpr int N = BmType<T>::N;
  extern __shared__ __align__(16) unsigned char bm_smem[];
  BmShared& sh = *reinterpret_cast<BmShared*>(bm_smem);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t ring = (uint32_t)__cvta_generic_to_shared(sh.ring) + tid * 16;
  pg_wait();

  const int r = blockIdx.x / a.splits, split = blockIdx.x - r * a.splits, group = r / a.beams;
  const BmRow<T> row(a, r);
  const int p0 = min(row.pieces, split * a.per), p1 = min(row.pieces, p0 + a.per);
  const bool front = split == 0, back = split == a.splits - 1;
  const float score = __ldcg(a.scores + r);
  const bool done = a.ended && __ldcg(a.ended + r);
  const unsigned char* source = reinterpret_cast<const unsigned char*>(row.base + row.token(p0 + tid));
  auto fetch = [&](int i, int slot) {                     // piece i on its way
    if (i < p1)
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(ring + slot * (BM_THREADS * 16)),
                   "l"(source + (int64_t)(i - p0 - tid) * 16) : "memory");
  };
  auto commit = [] { asm volatile("cp.async.commit_group;" ::: "memory"); };
  if (bm_live(score) && !done) {
    unsigned long long* out = a.keys + ((size_t)r * a.splits + split) * a.keep;
#pragma unroll
    for (int u = 0; u < BM_RING; u += 2) {                  // two pieces at a time
      fetch(p0 + u * BM_THREADS + tid, u);
      fetch(p0 + (u + 1) * BM_THREADS + tid, u + 1);
      commit();
    }
    const int single = row.single(tid, front, back);
    const float lone = single >= 0 ? fminf(BmType<T>::load(row.base + single), BmType<T>::most) : -INFINITY;
    // ---- its first tile: reference and bar ----
    float best = lone;
    asm volatile("cp.async.wait_group %0;" ::"n"((BM_RING - BM_FIRST) / 2) : "memory");
#pragma unroll
    for (int u = 0; u < BM_FIRST; ++u)
      if (p0 + u * BM_THREADS + tid < p1) best = fmaxf(best, bm_top<T>(sh.ring[u][tid]));
    best = fminf(best, BmType<T>::most);
    float ref = bm_block_max(sh, best);
    const bool wide = a.keep > 32;                        // 64 groups of four threads are enough for 32
    if (!wide) {
      best = fmaxf(best, __shfl_xor_sync(0xffffffffu, best, 1));
      best = fmaxf(best, __shfl_xor_sync(0xffffffffu, best, 2));
    }
    const int of = wide ? BM_THREADS : BM_THREADS / 4;
    if (wide || (tid & 3) == 0) sh.best[wide ? tid : tid >> 2] = best;
    if (tid == 0) {
      sh.bar = -INFINITY;
      sh.count = 0;
    }
    __syncthreads();
    if (tid < of) {
      const float mine = sh.best[tid];
      int larger = 0;
      for (int i = 0; i < of; i += 4) {
        const float4 x = *reinterpret_cast<const float4*>(sh.best + i);
        larger += (x.x > mine || (x.x == mine && i < tid)) + (x.y > mine || (x.y == mine && i + 1 < tid)) +
                  (x.z > mine || (x.z == mine && i + 2 < tid)) + (x.w > mine || (x.w == mine && i + 3 < tid));
      }
      if (larger == a.keep - 1) sh.bar = mine;
    }
    __syncthreads();
    float bar = fmaxf(sh.bar, -FLT_MAX);                  // -inf is no candidate

    // ---- the pass ----
    // `floor`: what is less counts as that, 2^-125 of the reference's term or nothing; -inf where the type has no such number
    float limit, floor, care;                             // care: pieces above it need more than adding up (NaN: all)
    double sum = 0.0;
    uint64_t far2 = 0;                                    // terms times x
    float highest = -INFINITY;                            // of the logits added
    auto refer = [&](float to) {                          // nothing seen so far: any reference will do, the next element moves it
      ref = to == -INFINITY ? 0.f : to;
      limit = to == -INFINITY ? -INFINITY : ref + kRefFar;
      floor = fabsf(ref) <= kRefPacked ? BmType<T>::below(ref) : -INFINITY;
      care = floor == -INFINITY ? NAN : limit;
    };
    // Terms are l log2(e) less the rounded ref log2(e).  That rounding, `off` (2^-8 at most, with references of 2^16 at most),
    // is taken out of the sum at the end: 2^-off to the second order, the third below 4e-9.
    auto off = [&] { return floor == -INFINITY ? 0.f : fmaf(ref, 1.4426950408889634f, -(ref * 1.4426950408889634f)); };
    auto back_by = [](float d) {
      const double u = 0.69314718055994531 * (double)d;
      return fma(u, fma(u, 0.5, -1.0), 1.0);
    };
    refer(ref);
    auto push = [&](float l, int token) {
      const int n = atomicAdd(&sh.count, 1);
      if (n < BM_LIST) sh.list[n] = bm_key(l, token);
    };
    if (lone >= bar) push(lone, single);
    if (lone > -INFINITY) {
      // as the terms of pieces are (`add`), whose correction it shares
      const float x = floor == -INFINITY ? (lone - ref) * 1.4426950408889634f :
                                           fmaf(lone, 1.4426950408889634f, -(ref * 1.4426950408889634f)), y = pa_ex2(x);
      sum = y;
      if (y > 0.f) far2 = f32x2_pack(x * y, 0.f);
    }
    const uint64_t scale2 = f32x2_pack(1.4426950408889634f, 1.4426950408889634f);
    auto add = [&](const float* f, uint64_t& part) {
      const float c = -ref * 1.4426950408889634f;
      const uint64_t back2 = f32x2_pack(c, c);
#pragma unroll
      for (int e = 0; e < N; e += 2) {
        const uint64_t x = f32x2_fma(f32x2_pack(f[e], f[e + 1]), scale2, back2);
        float x0, x1;
        f32x2_unpack(x, x0, x1);
        const uint64_t y = f32x2_pack(pa_ex2(x0), pa_ex2(x1));
        far2 = f32x2_fma(y, x, far2);
        part = f32x2_add(part, y);
      }
    };
    auto add_up = [&](uint64_t part) {
      float s0, s1;
      f32x2_unpack(part, s0, s1);
      sum += (double)(s0 + s1);
    };
    int seen = 0, next_cut = 2 * BM_FIRST;                // pieces of a thread so far, and when the list is cut down next
    for (int at = p0; at < p1; at += 2 * BM_THREADS) {
      asm volatile("cp.async.wait_group %0;" ::"n"(BM_RING / 2 - 1) : "memory");
      const int slot = seen & (BM_RING - 1);
      uint4 v[2] = {sh.ring[slot][tid], sh.ring[slot + 1][tid]};
      const float tops[2] = {bm_top<T>(v[0]), bm_top<T>(v[1])}, higher = fmaxf(tops[0], tops[1]);
      if (at + 2 * BM_THREADS <= p1 && higher <= care && bar > floor) {
        float f[2][N];
        uint64_t part[2] = {0, 0};
        const uint32_t low = BmType<T>::pack(floor);
        bm_unpack<T>(v[0], low, f[0]);
        bm_unpack<T>(v[1], low, f[1]);
        add(f[0], part[0]);
        add(f[1], part[1]);
        add_up(f32x2_add(part[0], part[1]));
        highest = fmaxf(highest, higher);
        if (higher >= bar) {
          const int token = row.token(at + tid);
#pragma unroll
          for (int k = 0; k < 2; ++k)
            if (tops[k] >= bar) {
#pragma unroll
              for (int e = 0; e < N; ++e)
                if (f[k][e] >= bar) push(f[k][e], token + k * (BM_THREADS * N) + e);
            }
        }
      } else {
#pragma unroll 1
        for (int k = 0; k < 2; ++k) {
          const int i = at + k * BM_THREADS + tid;
          if (i >= p1) break;
          uint4 w = k ? v[1] : v[0];
          float top = fmaxf(bm_top<T>(w), -INFINITY);
          if (top > limit) {
            top = fminf(top, BmType<T>::most);
            if (limit == -INFINITY) {
              sum = 0.0;
              far2 = 0;
              refer(top);
            } else if (top > ref) {
              // In 64 bits, so that it adds nothing to the errors of the terms so far; their own `off` is taken out, and
              // the new one, which the end takes out, put in.
              const double scale = bm_exp2(((double)ref - (double)top) * 1.44269504088896340735992);
              float s0, s1;
              f32x2_unpack(far2, s0, s1);
              // errors so far are those of x as it was, of either sign (up: as at the end)
              const float up = fmaxf(0.f, (highest - ref) * 1.4426950408889634f);
              far2 = scale > 0.0 ? f32x2_pack((s0 + s1 - 2.f * up * (float)sum) * (float)scale, 0.f) : 0;
              sum *= scale * back_by(off());
              highest = -INFINITY;                        // all so far lie below the new one
              refer(top);
              sum *= back_by(-off());
            }
            const uint32_t most = BmType<T>::pack(BmType<T>::most);
            w = make_uint4(BmType<T>::smaller(w.x, most), BmType<T>::smaller(w.y, most), BmType<T>::smaller(w.z, most),
                           BmType<T>::smaller(w.w, most));
          }
          highest = fmaxf(highest, top);
          float f[N];
          bm_unpack<T>(w, BmType<T>::pack(floor), f);
          uint64_t part = 0;
          if (floor == -INFINITY) {
#pragma unroll
            for (int e = 0; e < N; e += 2) {
              const float x0 = (f[e] - ref) * 1.4426950408889634f, x1 = (f[e + 1] - ref) * 1.4426950408889634f;   // -inf: no term
              const float y0 = pa_ex2(x0), y1 = pa_ex2(x1);
              part = f32x2_add(part, f32x2_pack(y0, y1));
              far2 = f32x2_add(far2, f32x2_pack(y0 > 0.f ? x0 * y0 : 0.f, y1 > 0.f ? x1 * y1 : 0.f));
            }
          } else {
            add(f, part);
          }
          add_up(part);
          if (top >= bar) {
            const int token = row.token(i);
            if (bar > floor) {
#pragma unroll
              for (int e = 0; e < N; ++e)
                if (f[e] >= bar) push(f[e], token + e);
            } else {
#pragma unroll 1
              for (int e = 0; e < N; ++e) {               // as they are in memory
                const float l = fminf(BmType<T>::load(row.base + token + e), BmType<T>::most);
                if (l >= bar) push(l, token + e);
              }
            }
          }
        }
      }
      fetch(at + BM_RING * BM_THREADS + tid, slot);       // (the pieces there have been read)
      fetch(at + (BM_RING + 1) * BM_THREADS + tid, slot + 1);
      commit();
      seen += 2;
      if (seen == next_cut) {
        next_cut *= 2;
        __syncthreads();
        const int count = sh.count;
        if (count > 2 * a.keep && count <= BM_THREADS) {
          bm_rank(count, [&](int k, int i) { return sh.list[k] > sh.list[i]; },
                  [&](int i, int rank) { if (rank < a.keep) sh.kept[rank] = sh.list[i]; });
          __syncthreads();
          for (int i = tid; i < a.keep; i += BM_THREADS) sh.list[i] = sh.kept[i];
          if (tid == 0) {
            sh.bar = bm_logit(sh.kept[a.keep - 1]);
            sh.count = a.keep;
          }
        }
        __syncthreads();
        bar = fmaxf(bar, sh.bar);
      }
    }
    if (limit == -INFINITY) {                             // nothing seen
      sum = 0.0;
      far2 = 0;
      ref = -FLT_MAX;
      floor = -INFINITY;
    }
    // ---- its sum and its largest ----
    const float high = bm_block_max(sh, ref);
    const float behind = (ref - high) * 1.4426950408889634f;
    double scale = ref == high ? 1.0 : bm_exp2(behind);
    scale *= back_by(off());
    float f0, f1;
    f32x2_unpack(far2, f0, f1);
    double all = sum * scale;
    const float up = fmaxf(0.f, (highest - ref) * 1.4426950408889634f);   // terms with x > 0 count with 2 up - x >= x
    float far = scale > 0.0 ? (f0 + f1 + (behind - 2.f * up) * (float)sum) * (float)scale : 0.f;
#pragma unroll
    for (int d = 16; d; d >>= 1) {
      all += __shfl_xor_sync(0xffffffffu, all, d);
      far += __shfl_xor_sync(0xffffffffu, far, d);
    }
    if (lane == 0) {
      sh.dsum[warp] = all;
      sh.ref[warp] = far;
    }
    __syncthreads();
    if (tid == 0) {
      all = 0.0;
      far = 0.f;
      for (int i = 0; i < BM_THREADS / 32; ++i) {
        all += sh.dsum[i];
        far += sh.ref[i];
      }
      a.sums[(size_t)r * a.splits + split] = make_float4(high, (float)all, -far, 0.f);
    }
    const int count = sh.count;
    if (count > BM_LIST) {
      bm_crowded<T>(sh, a, row, p0, p1, front, back, out);
    } else {
      bm_rank(count, [&](int k, int i) { return sh.list[k] > sh.list[i]; },
              [&](int i, int rank) { if (rank < a.keep) out[rank] = sh.list[i]; });
      for (int i = count + tid; i < a.keep; i += BM_THREADS) out[i] = 0;
    }
  }
  asm volatile("cp.async.wait_group 0;" ::: "memory");
  // ---- the last CTA of the group joins ----
  __syncthreads();
  if (tid == 0) {
    __threadfence();                                      // what the block has written
    sh.last = atomicAdd(a.counters + group, 1) == a.beams * a.splits - 1;
    if (sh.last) {
      a.counters[group] = 0;
      __threadfence();
    }
  }
  __syncthreads();
  if (sh.last) bm_join<T>(sh, a, group);
}

struct BmLayout {
  size_t sums, keys, total;
  int splits, per;
};

static bool valid_beams(const less_beams* d) {
  if (d->groups < 1 || d->beams < 1 || d->beams > BM_MOST_BEAMS || d->vocab < 1 || d->vocab > (1 << 26) || d->keep < 1 || d->keep > BM_MOST_KEEP) return false;
  if (d->flags & ~(uint32_t)(LESS_BEAMS_BF16 | LESS_BEAMS_F32) || d->flags == (LESS_BEAMS_BF16 | LESS_BEAMS_F32)) return false;
  if (d->end_token < -1 || d->end_token >= d->vocab) return false;
  return d->groups <= (1 << 20) / d->beams;               // rows
}

// A row is cut so that all CTAs of a call, four on a multiprocessor, run at once, but for no less than 4096 elements each, nor
// into so many lists that joining them shows (64 groups of 8 beams of 128 256: one stretch a row; three 15 us more).  The
// workspace goes by this, and may be asked for without a device: B200's 148 multiprocessors, not the current device's.
static BmLayout bm_layout(const less_beams* d) {
  BmLayout l;
  const int64_t rows = (int64_t)d->groups * d->beams;
  const int pieces = (int)(((int64_t)d->vocab * (d->flags & LESS_BEAMS_F32 ? 4 : 2) + 15) / 16);
  int64_t s = pg_ceil(d->vocab, 4096);
  if (s > BM_CTAS * 148 / rows) s = BM_CTAS * 148 / rows;
  if (s > BM_JOINED / (d->beams * d->keep)) s = BM_JOINED / (d->beams * d->keep);
  l.splits = (int)(s < 1 ? 1 : s);
  l.per = pg_ceil(pieces, l.splits);
  size_t at = ((size_t)d->groups * 4 + 255) / 256 * 256;
  l.sums = at;
  at = (at + (size_t)rows * l.splits * 16 + 255) / 256 * 256;
  l.keys = at;
  l.total = (at + (size_t)rows * l.splits * d->keep * 8 + 255) / 256 * 256;
  return l;
}

template <typename T>
static int launch_select(const BmArgs& a, cudaStream_t s) {
  static std::atomic<unsigned long long> done{0};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return fail_cuda("cudaGetDevice");
  if (dev >= 64 || !(done.load(std::memory_order_relaxed) >> dev & 1)) {
    if (cudaFuncSetAttribute(beam_select_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(BmShared)) != cudaSuccess)
      return fail_cuda("shared memory opt-in of beam_select_kernel");
    if (dev < 64) done.fetch_or(1ull << dev, std::memory_order_relaxed);
  }
  return pg_launch("beam_select_kernel", beam_select_kernel<T>, dim3((unsigned)(a.groups * a.beams * a.splits)), BM_THREADS,
                   sizeof(BmShared), s, a);
}

}  // namespace less

using namespace less;

extern "C" size_t less_beams_workspace_bytes(const less_beams* d) { return d && valid_beams(d) ? bm_layout(d).total : 0; }

extern "C" int less_beam_select(const less_beams* d, const void* logits, int64_t row_stride, const float* scores,
                                const uint8_t* ended, float* out_scores, int32_t* out_tokens, int32_t* out_parents,
                                uint8_t* out_ended, void* stream) {
  if (!d) return LESS_ERR_NULL_POINTER;
  if (!valid_beams(d)) return LESS_ERR_INVALID_CONFIG;
  if (!logits || !scores || !out_scores || !out_tokens || !out_parents || !d->workspace) return LESS_ERR_NULL_POINTER;
  if (ended && d->end_token < 0) return LESS_ERR_INVALID_CONFIG;
  if (row_stride < d->vocab || row_stride > ((int64_t)1 << 40)) return LESS_ERR_INVALID_CONFIG;
  const size_t size = d->flags & LESS_BEAMS_F32 ? 4 : 2;
  if ((uintptr_t)logits & (size - 1) || (uintptr_t)d->workspace & 255) return LESS_ERR_MISALIGNED;
  if (((uintptr_t)scores | (uintptr_t)out_scores | (uintptr_t)out_tokens | (uintptr_t)out_parents) & 3) return LESS_ERR_MISALIGNED;
  const BmLayout l = bm_layout(d);
  if (d->workspace_bytes < l.total) return LESS_ERR_ARENA_TOO_SMALL;
  char* w = (char*)d->workspace;
  BmArgs a = {logits, row_stride, scores, ended, d->groups, d->beams, d->vocab, d->keep, d->end_token, l.splits, l.per,
              out_scores, out_tokens, out_parents, out_ended, (int32_t*)w, (float4*)(w + l.sums), (unsigned long long*)(w + l.keys)};
  cudaStream_t s = (cudaStream_t)stream;
  if (d->flags & LESS_BEAMS_F32) return launch_select<float>(a, s);
  if (d->flags & LESS_BEAMS_BF16) return launch_select<__nv_bfloat16>(a, s);
  return launch_select<__half>(a, s);
}
